// Part of api.cu (included there, inside its namespaces): the operators in 8-bit floating point and the step between two blocks.

bool format_ok(int format) { return format == MIPGEMM_F8_E4M3 || format == MIPGEMM_F8_E5M2; }
bool size_ok(int64_t n) { return n >= 0 && n <= 0x7FFFFF00LL; }
long long f8_blocks(long long n) { return (n + 127) / 128; }

// out[0]: along the rows, or squares; out[1]: along the columns.  Either may have no codes.
int f8_quantize_impl(int type, int format, bool squares, int64_t M, int64_t N, const void* X, int64_t ldx, const mip::F8Codes (&out)[2],
                     void* stream_v) {
    tl_last_path = MIPGEMM_PATH_NONE;
    if (!type_ok(type) || !format_ok(format) || !size_ok(M) || !size_ok(N) || ldx < N) return MIPGEMM_ERR_INVALID_ARG;
    int form = 0;
    for (int side = 0; side < 2; ++side) {
        const mip::F8Codes& o = out[side];
        if (!o.Q && !o.scale) continue;                      // (this side is not wanted)
        if (!o.Q || !o.scale || !aligned_to(o.scale, 4)) return MIPGEMM_ERR_INVALID_ARG;
        if (o.ldq < N || o.lds < (side == 1 ? N : (squares ? f8_blocks(N) : M))) return MIPGEMM_ERR_INVALID_ARG;
        form |= squares ? 4 : 1 << side;
    }
    if (M == 0 || N == 0) return MIPGEMM_OK;
    if (!form || !X || !aligned_to(X, type_size(type))) return MIPGEMM_ERR_INVALID_ARG;
    DeviceState* dev = nullptr;
    const int st = get_device(&dev);
    if (st != MIPGEMM_OK) return st;
    int launches = 0;
    const cudaError_t e = mip::launch_f8_quantize(type, format, form, M, N, X, ldx, out, static_cast<cudaStream_t>(stream_v), &launches);
    g_launches += launches;
    return e == cudaSuccess ? MIPGEMM_OK : cuda_fail(e);
}

int f8_dequantize_impl(int type, int format, int blocks, int64_t M, int64_t N, const mip::F8Codes& in, void* X, int64_t ldx, void* stream_v) {
    tl_last_path = MIPGEMM_PATH_NONE;
    if (!type_ok(type) || !format_ok(format) || blocks < MIPGEMM_F8_ROWS || blocks > MIPGEMM_F8_SQUARES || !size_ok(M) || !size_ok(N) || ldx < N || in.ldq < N ||
        in.lds < (blocks == MIPGEMM_F8_ROWS ? M : (blocks == MIPGEMM_F8_COLUMNS ? N : f8_blocks(N))))
        return MIPGEMM_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return MIPGEMM_OK;
    if (!in.Q || !in.scale || !aligned_to(in.scale, 4) || !X || !aligned_to(X, type_size(type))) return MIPGEMM_ERR_INVALID_ARG;
    DeviceState* dev = nullptr;
    const int st = get_device(&dev);
    if (st != MIPGEMM_OK) return st;
    int launches = 0;
    const cudaError_t e = mip::launch_f8_dequantize(type, format, blocks, M, N, in, X, ldx, static_cast<cudaStream_t>(stream_v), &launches);
    g_launches += launches;
    return e == cudaSuccess ? MIPGEMM_OK : cuda_fail(e);
}

// ---------------------------------------------------------------------------------------
// The product.

struct F8Plan {
    int pair, grid, split;
    int few;                             // 1: the few-token kernel
};

// Few tokens: as plan_stream of the 8-bit layer, K is split over the CTAs of a cluster while that leaves all CTAs resident at
// once (two per SM), each CTA at least two k-blocks, and either a quarter of the SMs would go without or each still gets eight.
F8Plan plan_f8_stream(const mip::F8ProductArgs& a, const DeviceState* dev) {
    const long long tiles = (a.N + 127) / 128, k_blocks = f8_blocks(a.K);
    F8Plan pl{0, 0, 1, 1};
    while (pl.split < 8 && 2 * pl.split * tiles <= 2ll * dev->sm_count && k_blocks / (2 * pl.split) >= 2 &&
           (4 * tiles * pl.split < 3 * dev->sm_count || k_blocks / (2 * pl.split) >= 8))
        pl.split *= 2;
    const Tuning tun = tuning_now();
    if (tun.split_k == 1 || tun.split_k == 2 || tun.split_k == 4 || tun.split_k == 8) pl.split = tun.split_k;
    pl.grid = static_cast<int>(tiles) * pl.split;
    return pl;
}
// Up to so many tokens take it (us here / dense kernel: 16 x 14336 x 4096 11.4 / 15.4, 32 x 11008 x 4096 13.8 / 14.9, and with 64
// tokens 64 x 4096 x 4096 11.4 / 10.4, 64 x 14336 x 4096 20.1 / 16.0).
constexpr long long kFewTokens = 32;
int few_columns(long long M) { return M <= 16 ? 16 : 32; }

F8Plan plan_f8(const mip::F8ProductArgs& a, const DeviceState* dev) {
    const Tuning tun = tuning_now();
    const int k_blocks = static_cast<int>(f8_blocks(a.K));
    F8Plan best{0, 1, 1, 0};
    double best_clk = 1e30;
    for (int pair = 0; pair <= 1; ++pair) {
        if (pair && dev->pair_clusters <= 0) continue;
        if (tun.force_path == MIPGEMM_PATH_DENSE_PAIR && !pair && dev->pair_clusters > 0) continue;
        if (tun.force_path == MIPGEMM_PATH_DENSE && pair) continue;
        const long long side = pair ? 256 : 128, tiles = ((a.M + side - 1) / side) * ((a.N + side - 1) / side);
        const long long slots = pair ? dev->pair_clusters : dev->sm_count;
        for (int split = 1; split <= kMaxSplit; ++split) {
            // K in shares whose partial sums a second kernel adds: only while there are more SMs than tiles (not in lent scratch)
            if (split > 1 && (dev->lent || tiles * (split - 1) >= slots || k_blocks / split < 2)) break;
            const int share = (k_blocks + split - 1) / split;
            if ((k_blocks + share - 1) / share != split) continue;
            // clocks of a k-block (measured: pairs 780, with a scale for each column 1200; single CTAs 480 and 620), but not less than
            // its copies' latency over the stages on their way, which is longer where few row tiles share the weights (512 x 4096 x
            // 14336 bf16: 128 single CTAs 57 us, 64 units of pairs with K in two shares 45; 256 x 4096 x 14336: 28 and, in four shares, 25;
            // from eight row tiles, 1024 x 4096 x 14336: pairs whole 64, in two shares 85); of a tile's outputs, which nothing hides.
            // Of 32 sizes (64 to 4096 rows, both kinds of scales) 24 get a form within 5 % of the best one; furthest off are 1024 x 1024 x
            // 8192 (23.1 us, pairs in four shares 19.1) and, with column scales, 2048 x 2048 x 512 (11.0, single CTAs 9.0).
            const int stages = mip::f8_product_stages(a.type, pair != 0, a.b_vec != 0, split > 1);
            const double latency = ((a.M + side - 1) / side < 8 ? 3600.0 : 2000.0) / stages;
            const double block = std::max(pair ? (a.b_vec ? 1200.0 : 780.0) : (a.b_vec ? 620.0 : 480.0), latency);
            const long long waves = (tiles * split + slots - 1) / slots;
            double clk = static_cast<double>(waves) * (share * block + (a.type == MIPGEMM_TYPE_F32 ? (pair ? 8000.0 : 5500.0) : (pair ? 5000.0 : 4500.0))) + (pair ? 1900.0 : 0.0);
            // (a launch, and the planes written and read at the L2's pace)
            if (split > 1) clk += 5500.0 + 8.0 * split * static_cast<double>(a.M) * a.N / 3500.0;
            if (tun.split_k && split != tun.split_k) clk += kNotAsked;
            if (clk < best_clk) {
                best_clk = clk;
                best = F8Plan{pair, static_cast<int>(std::min(tiles * split, slots)) * (pair ? 2 : 1), split, 0};
            }
        }
    }
    return best;
}

struct F8Entry {
    bool used = false;
    PlanKey key;
    mip::F8ProductParams p;
    F8Plan pl;
};
constexpr int kF8CacheSlots = 256;
F8Entry* g_f8_cache = nullptr;

// as_passed: the operands are the caller's own, not re-pitched copies.
int run_f8_product(const mip::F8ProductArgs& a, DeviceState* dev, cudaStream_t stream, bool as_passed) {
    mip::F8ProductParams p;
    F8Plan pl;
    const bool cacheable = as_passed && plan_cache_enabled();
    PlanKey key;
    bool hit = false;
    if (cacheable) {
        std::memset(&key, 0, sizeof(key));
        const uint64_t words[] = {
            reinterpret_cast<uint64_t>(dev), g_tuning_epoch.load(std::memory_order_acquire),
            static_cast<uint64_t>(a.type) | (static_cast<uint64_t>(a.a_format) << 8) | (static_cast<uint64_t>(a.b_format) << 9) |
                (static_cast<uint64_t>(a.a_order) << 10) | (static_cast<uint64_t>(a.b_order) << 11) | (static_cast<uint64_t>(a.b_vec) << 12) |
                (static_cast<uint64_t>(dev->lent != nullptr) << 13),
            static_cast<uint64_t>(a.M), static_cast<uint64_t>(a.N), static_cast<uint64_t>(a.K), reinterpret_cast<uint64_t>(a.A),
            static_cast<uint64_t>(a.lda), reinterpret_cast<uint64_t>(a.B), static_cast<uint64_t>(a.ldb), reinterpret_cast<uint64_t>(a.R),
            static_cast<uint64_t>(a.ldr), reinterpret_cast<uint64_t>(a.C), static_cast<uint64_t>(a.ldc)};
        static_assert(sizeof(words) <= sizeof(key.w), "plan key too small");
        std::memcpy(key.w, words, sizeof(words));
        const size_t slot = plan_slot(key) % kF8CacheSlots;
        std::lock_guard<std::mutex> lock(g_plan_mutex);
        if (g_f8_cache && g_f8_cache[slot].used && std::memcmp(&g_f8_cache[slot].key, &key, sizeof(key)) == 0) {
            p = g_f8_cache[slot].p;
            pl = g_f8_cache[slot].pl;
            hit = true;
            ++g_plan_hits;
        }
    }
    if (!hit) {
        const Tuning tun = tuning_now();
        pl = plan_f8(a, dev);
        const int k_blocks = static_cast<int>(f8_blocks(a.K));
        int few_stages = 0;
        if (a.M <= kFewTokens && !a.a_order && tun.force_path != MIPGEMM_PATH_DENSE && tun.force_path != MIPGEMM_PATH_DENSE_PAIR) {
            const F8Plan few = plan_f8_stream(a, dev);
            few_stages = mip::f8_stream_stages(few_columns(a.M), (k_blocks + few.split - 1) / few.split);
            if (few_stages) pl = few;
        }
        std::memset(&p, 0, sizeof(p));
        p.M = static_cast<int>(a.M);
        p.N = static_cast<int>(a.N);
        p.K = static_cast<int>(a.K);
        p.type = a.type;
        p.k_blocks = k_blocks;
        p.split = pl.split;
        p.kb_share = (k_blocks + pl.split - 1) / pl.split;
        p.a_mn = a.a_order;
        p.b_mn = a.b_order;
        p.status = dev->status_word;
        int st;
        if (pl.few) {
            p.block_n = few_columns(a.M);
            p.out_n = 128;
            p.stages = few_stages;
            // D float32; the weights are the 128-row operand, the tokens the columns
            p.idesc = (1u << 4) | (static_cast<uint32_t>(a.b_format) << 7) | (static_cast<uint32_t>(a.a_format) << 10) |
                      (static_cast<uint32_t>(a.b_order) << 15) | (static_cast<uint32_t>(p.block_n >> 3) << 17) | (128u >> 4 << 24);
            st = encode_tiled_2d(&p.tmap_a, a.A, a.K, a.M, a.lda, 128, p.M);
        } else {
            const int side = pl.pair ? 256 : 128;
            p.block_n = p.out_n = side;
            p.tiles_m = static_cast<int>((a.M + side - 1) / side);
            p.tiles_n = static_cast<int>((a.N + side - 1) / side);
            p.plane_rows = static_cast<int>(round_up(a.M, 32));
            p.stages = mip::f8_product_stages(a.type, pl.pair != 0, a.b_vec != 0, pl.split > 1);
            if (tun.stages) p.stages = std::min(p.stages, std::max(tun.stages, 2));
            p.a_rows = a.a_order ? mip::kBlockM : std::min(p.M, mip::kBlockM);
            // D float32, the operands' formats, which of them are M/N-contiguous, 128 columns, the tile's rows
            p.idesc = (1u << 4) | (static_cast<uint32_t>(a.a_format) << 7) | (static_cast<uint32_t>(a.b_format) << 10) | (static_cast<uint32_t>(a.a_order) << 15) |
                      (static_cast<uint32_t>(a.b_order) << 16) | (128u >> 3 << 17) | (static_cast<uint32_t>(side >> 4) << 24);
            const size_t size = type_size(a.type);
            p.r_tma = a.R && aligned16(a.R, a.ldr * static_cast<long long>(size)) ? 1 : 0;
            p.c_tma = a.N * size % 16 == 0 && aligned16(a.C, a.ldc * static_cast<long long>(size)) ? 1 : 0;
            st = a.a_order ? encode_tiled_2d(&p.tmap_a, a.A, a.M, a.K, a.lda, 128, 128) : encode_tiled_2d(&p.tmap_a, a.A, a.K, a.M, a.lda, 128, p.a_rows);
            if (st == MIPGEMM_OK && p.r_tma) st = encode_slots(&p.tmap_r, a.R, a.type, a.M, a.N, a.ldr);
            if (st == MIPGEMM_OK && p.c_tma) st = encode_slots(&p.tmap_c, a.C, a.type, a.M, a.N, a.ldc);
        }
        if (st == MIPGEMM_OK)
            st = a.b_order ? encode_tiled_2d(&p.tmap_b0, a.B, a.N, a.K, a.ldb, 128, 128) : encode_tiled_2d(&p.tmap_b0, a.B, a.K, a.N, a.ldb, 128, 128);
        if (st != MIPGEMM_OK) return st;
        p.R = a.R; p.ldr = a.ldr;
        p.C = a.C; p.ldc = a.ldc;
        p.wait_budget_ns = g_wait_budget_ns.load(std::memory_order_relaxed);
        p.debug_flags = g_debug_flags.load(std::memory_order_relaxed);
        if (cacheable) {
            ++g_plan_misses;
            std::lock_guard<std::mutex> lock(g_plan_mutex);
            if (!g_f8_cache) g_f8_cache = new (std::nothrow) F8Entry[kF8CacheSlots];
            if (g_f8_cache) {            // (no memory: calls plan every time)
                F8Entry& e = g_f8_cache[plan_slot(key) % kF8CacheSlots];
                e.used = true;
                e.key = key;
                e.p = p;
                e.pl = pl;
            }
        }
    }
    // (not part of the plan)
    p.sa = a.a_scale; p.lds_a = a.ldas;
    p.sb = a.b_scale;
    // scale of k-block kb and column j: rows of blocks along K (vectors; squares of an N-contiguous B), or along N
    p.sb_k = a.b_vec || a.b_order ? a.ldbs : 1;
    p.sb_n = a.b_vec || a.b_order ? 1 : a.ldbs;
    p.bias = a.bias;
    const int ready = family_ready(dev, pl.few ? kFamilyF8Few : kFamilyF8);
    if (ready != MIPGEMM_OK) return ready;
    cudaError_t e;
    int launches = 1;
    if (pl.few) {
        // (a promise about the weights, not part of the plan; not about re-pitched copies, which the kernel before this one writes)
        const size_t b_bytes = static_cast<size_t>(a.b_order ? a.K - 1 : a.N - 1) * a.ldb + (a.b_order ? a.N : a.K);
        p.b_constant = as_passed && a.M <= 16 && (g_weights_constant.load() || inside_constant_range(a.B, b_bytes));
        e = mip::launch_f8_stream(p, a.b_vec != 0, pl.grid, stream);
    } else if (pl.split > 1) {
        mip::PartialPlanes planes{nullptr, pl.split, p.plane_rows, round_up(a.N, 32), 0};
        Scratch scratch(dev, stream);
        const int st = scratch.reserve(static_cast<size_t>(pl.split) * planes.plane_rows * planes.pitch * 4);
        if (st != MIPGEMM_OK) return st;
        planes.base = scratch.base;
        p.C = scratch.base;
        p.ldc = planes.pitch;
        p.R = nullptr;
        p.r_tma = p.c_tma = 0;
        e = mip::launch_f8_product(p, pl.pair != 0, a.b_vec != 0, true, pl.grid, stream);
        if (e == cudaSuccess) e = mip::launch_f8_finish(a, planes, stream, &launches);
    } else {
        e = mip::launch_f8_product(p, pl.pair != 0, a.b_vec != 0, false, pl.grid, stream);
    }
    g_launches += launches;
    if (e != cudaSuccess) return cuda_fail(e);
    tl_last_path = (pl.few ? MIPGEMM_PATH_SKINNY : (pl.pair ? MIPGEMM_PATH_DENSE_PAIR : MIPGEMM_PATH_DENSE)) | (pl.split > 1 ? MIPGEMM_PATH_SPLITK : 0);
    if (log_enabled())
        std::fprintf(stderr, "mipgemm: f8 product M=%d N=%d K=%d orders=%d%d -> %s stages=%d split=%d r_tma=%d c_tma=%d plan=%s\n", p.M, p.N, p.K,
                     a.a_order, a.b_order, pl.few ? "few tokens" : (pl.pair ? "dense cta-pair" : "dense one-cta"), p.stages, pl.split, p.r_tma, p.c_tma, hit ? "cached" : "new");
    return MIPGEMM_OK;
}

// (a.b_vec arrives as the caller's b_blocks)
int f8_product_impl(const mip::F8ProductArgs& a, void* stream_v) {
    tl_last_path = MIPGEMM_PATH_NONE;
    if (!type_ok(a.type) || !format_ok(a.a_format) || !format_ok(a.b_format) || (a.a_order & ~1) || (a.b_order & ~1)) return MIPGEMM_ERR_INVALID_ARG;
    const bool squares = a.b_vec == MIPGEMM_F8_SQUARES;
    if (!squares && a.b_vec != (a.b_order ? MIPGEMM_F8_COLUMNS : MIPGEMM_F8_ROWS)) return MIPGEMM_ERR_INVALID_ARG;
    if (!size_ok(a.M) || !size_ok(a.N) || !size_ok(a.K)) return MIPGEMM_ERR_INVALID_ARG;
    if (a.lda < (a.a_order ? a.M : a.K) || a.ldb < (a.b_order ? a.N : a.K) || a.ldc < a.N || (a.R && a.ldr < a.N)) return MIPGEMM_ERR_INVALID_ARG;
    if (a.a_scale && a.ldas < a.M) return MIPGEMM_ERR_INVALID_ARG;
    if (a.b_scale && a.ldbs < (squares ? f8_blocks(a.b_order ? a.N : a.K) : a.N)) return MIPGEMM_ERR_INVALID_ARG;
    if (a.M == 0 || a.N == 0) {
        tl_last_path = MIPGEMM_PATH_TRIVIAL;
        return MIPGEMM_OK;
    }
    if (!a.C || (a.K > 0 && (!a.A || !a.B))) return MIPGEMM_ERR_INVALID_ARG;
    for (const void* m : {static_cast<const void*>(a.C), a.R})
        if (!aligned_to(m, type_size(a.type))) return MIPGEMM_ERR_INVALID_ARG;
    for (const float* v : {a.a_scale, a.b_scale, a.bias})
        if (!aligned_to(v, 4)) return MIPGEMM_ERR_INVALID_ARG;
    if (a.R == a.C && a.ldr != a.ldc) return MIPGEMM_ERR_INVALID_ARG;
    DeviceState* dev = nullptr;
    const int st = get_device(&dev);
    if (st != MIPGEMM_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    mip::F8ProductArgs use = a;
    use.b_vec = squares ? 0 : 1;
    if (a.K == 0) {                      // every sum is 0
        int launches = 0;
        const cudaError_t e = mip::launch_f8_finish(use, mip::PartialPlanes{}, stream, &launches);
        g_launches += launches;
        if (e != cudaSuccess) return cuda_fail(e);
        tl_last_path = MIPGEMM_PATH_TRIVIAL;
        return MIPGEMM_OK;
    }
    // operands that the TMA cannot address are re-pitched first
    struct Operand { const void** ptr; long long* ld; long long rows, cols; };
    const Operand ops[2] = {{&use.A, &use.lda, a.a_order ? a.K : a.M, a.a_order ? a.M : a.K}, {&use.B, &use.ldb, a.b_order ? a.K : a.N, a.b_order ? a.N : a.K}};
    Scratch scratch(dev, stream);
    size_t need = 0;
    for (const Operand& o : ops)
        if (!aligned16(*o.ptr, *o.ld)) need += align256(static_cast<size_t>(o.rows) * round_up(o.cols, 16));
    int rc = scratch.reserve(need);
    if (rc != MIPGEMM_OK) return rc;
    mip::RepackPart parts[2];
    int count = 0;
    for (const Operand& o : ops) {
        if (aligned16(*o.ptr, *o.ld)) continue;
        const long long pitch = round_up(o.cols, 16);
        void* dst = scratch.take(static_cast<size_t>(o.rows) * pitch);
        parts[count++] = mip::RepackPart{*o.ptr, *o.ld, dst, pitch, o.rows, o.cols};
        *o.ptr = dst;
        *o.ld = pitch;
    }
    if (count) {
        const cudaError_t e = mip::launch_repack_parts(parts, count, stream);
        ++g_launches;
        if (e != cudaSuccess) return cuda_fail(e);
    }
    rc = run_f8_product(use, dev, stream, need == 0);
    if (rc == MIPGEMM_OK && need) tl_last_path |= MIPGEMM_PATH_REPACK;
    return rc;
}

// ---------------------------------------------------------------------------------------
// The step between two blocks.

bool norm_ok(int kind) { return kind >= MIPGEMM_NORM_NONE && kind <= MIPGEMM_NORM_LAYER; }

// Rates are multiples of 2^-16: `bar` of 65536 values are dropped.  False: no rate.
bool dropout_rate(float drop, uint32_t* bar, float* scale) {
    if (!(drop >= 0.0f) || !(drop < 1.0f)) return false;
    *bar = static_cast<uint32_t>(std::lrint(static_cast<double>(drop) * 65536.0));
    if (*bar > 65535u) return false;
    *scale = static_cast<float>(65536.0 / (65536.0 - *bar));
    return true;
}

// A matrix of a step: there, with its pitch, aligned to its elements; *wide is taken back where 16-byte accesses do not reach it.
struct StepMatrix {
    const void* p;
    long long ld;
};
bool step_matrices_ok(std::initializer_list<StepMatrix> list, int type, long long N, bool* wide) {
    const long long size = static_cast<long long>(type_size(type));
    for (const StepMatrix& m : list) {
        if (!m.p) continue;
        if (m.ld < N || !aligned_to(m.p, type_size(type))) return false;
        if (!aligned16(m.p, m.ld * size)) *wide = false;
    }
    return true;
}
bool step_vectors_ok(std::initializer_list<const void*> list, bool* wide) {
    for (const void* p : list) {
        if (!aligned_to(p, 4)) return false;
        if (!aligned_to(p, 16)) *wide = false;
    }
    return true;
}

int norm_step_impl(int type, mip::StepArgs& a, float drop, void* stream_v) {
    tl_last_path = MIPGEMM_PATH_NONE;
    if (!type_ok(type) || !norm_ok(a.post) || !norm_ok(a.pre) || a.codes < MIPGEMM_CODES_NONE || a.codes > MIPGEMM_CODES_E5M2) return MIPGEMM_ERR_INVALID_ARG;
    if (!size_ok(a.M) || a.N < 0 || a.N > mip::kStepColumns || !(a.eps >= 0.0f)) return MIPGEMM_ERR_INVALID_ARG;
    if (!dropout_rate(drop, &a.mask.bar, &a.mask.scale)) return MIPGEMM_ERR_INVALID_ARG;
    a.wide = a.N % 8 == 0;
    a.wide_vectors = true;
    if (!step_matrices_ok({{a.X, a.ldx}, {a.Z, a.ldz}, {a.gate, a.ldgate}, {a.Y, a.ldy}, {a.H, a.ldh}}, type, a.N, &a.wide) ||
        !step_vectors_ok({a.post_w, a.post_b, a.pre_w, a.pre_b}, &a.wide_vectors))
        return MIPGEMM_ERR_INVALID_ARG;
    a.wide = a.wide && a.wide_vectors;
    if (!aligned_to(a.stats, 4) || !aligned_to(a.q_scale, 4) || !aligned_to(a.mask.counter, 8) || (a.gate && a.gate_rows < 1)) return MIPGEMM_ERR_INVALID_ARG;
    // parts that nothing would read, or that something would miss
    if (!a.Z && (a.post != MIPGEMM_NORM_NONE || a.gate || a.mask.bar)) return MIPGEMM_ERR_INVALID_ARG;
    if (((a.post_w || a.post_b) && a.post == MIPGEMM_NORM_NONE) || ((a.pre_w || a.pre_b) && a.pre == MIPGEMM_NORM_NONE)) return MIPGEMM_ERR_INVALID_ARG;
    if ((a.post_b && a.post != MIPGEMM_NORM_LAYER) || (a.pre_b && a.pre != MIPGEMM_NORM_LAYER)) return MIPGEMM_ERR_INVALID_ARG;
    if ((a.H || a.codes != MIPGEMM_CODES_NONE) && a.pre == MIPGEMM_NORM_NONE) return MIPGEMM_ERR_INVALID_ARG;
    if (a.codes != MIPGEMM_CODES_NONE) {
        if (a.ldq < a.N || (a.codes != MIPGEMM_CODES_S8 && a.ldqs < a.M)) return MIPGEMM_ERR_INVALID_ARG;
        if (!aligned_to(a.Q, 8) || a.ldq % 8 != 0) a.wide = false;
    }
    if (a.M == 0 || a.N == 0) return MIPGEMM_OK;
    if (!a.X && !a.Z) return MIPGEMM_ERR_INVALID_ARG;
    if (a.codes != MIPGEMM_CODES_NONE && (!a.Q || !a.q_scale)) return MIPGEMM_ERR_INVALID_ARG;
    if (!a.Y && !a.H && a.codes == MIPGEMM_CODES_NONE && !a.stats) return MIPGEMM_ERR_INVALID_ARG;
    if ((a.Y && ((a.Y == a.X && a.ldy != a.ldx) || (a.Y == a.Z && a.ldy != a.ldz)))) return MIPGEMM_ERR_INVALID_ARG;
    if (!a.gate) a.gate_rows = 1;        // (the kernels divide by it)
    else if (a.gate_rows > a.M) a.gate_rows = a.M;
    DeviceState* dev = nullptr;
    const int st = get_device(&dev);
    if (st != MIPGEMM_OK) return st;
    const cudaError_t e = mip::launch_norm_step(type, a, dev->sm_count, static_cast<cudaStream_t>(stream_v));
    ++g_launches;
    return e == cudaSuccess ? MIPGEMM_OK : cuda_fail(e);
}

int norm_step_grad_impl(int type, mip::StepGradArgs& a, float drop, void* stream_v) {
    tl_last_path = MIPGEMM_PATH_NONE;
    if (!type_ok(type) || !norm_ok(a.post) || !norm_ok(a.pre)) return MIPGEMM_ERR_INVALID_ARG;
    if (!size_ok(a.M) || a.N < 0 || a.N > mip::kStepColumns) return MIPGEMM_ERR_INVALID_ARG;
    if (!dropout_rate(drop, &a.mask.bar, &a.mask.scale)) return MIPGEMM_ERR_INVALID_ARG;
    a.wide = a.N % 8 == 0;
    a.wide_vectors = true;
    if (!step_matrices_ok({{a.dY, a.lddy}, {a.dH, a.lddh}, {a.Y, a.ldy}, {a.Z, a.ldz}, {a.gate, a.ldgate}, {a.dX, a.lddx}, {a.dZ, a.lddz}, {a.dgate, a.lddgate}},
                          type, a.N, &a.wide) ||
        !step_vectors_ok({a.post_w, a.post_b, a.pre_w}, &a.wide_vectors))
        return MIPGEMM_ERR_INVALID_ARG;
    a.wide = a.wide && a.wide_vectors;
    for (const float* v : {a.stats, static_cast<const float*>(a.dpost_w), static_cast<const float*>(a.dpost_b), static_cast<const float*>(a.dpre_w),
                           static_cast<const float*>(a.dpre_b)})
        if (!aligned_to(v, 4)) return MIPGEMM_ERR_INVALID_ARG;
    if (!aligned_to(a.mask.counter, 8) || (a.gate && a.gate_rows < 1) || (a.dgate && !a.gate)) return MIPGEMM_ERR_INVALID_ARG;
    const bool post = a.post != MIPGEMM_NORM_NONE, pre = a.pre != MIPGEMM_NORM_NONE;
    if ((!post && (a.post_w || a.post_b || a.dpost_w || a.dpost_b)) || (!pre && (a.pre_w || a.dpre_w || a.dpre_b || a.dH))) return MIPGEMM_ERR_INVALID_ARG;
    if ((a.post != MIPGEMM_NORM_LAYER && (a.post_b || a.dpost_b)) || (a.pre != MIPGEMM_NORM_LAYER && a.dpre_b)) return MIPGEMM_ERR_INVALID_ARG;
    if (!a.dX && !a.dZ && !a.dgate && !a.dpost_w && !a.dpost_b && !a.dpre_w && !a.dpre_b) return MIPGEMM_ERR_INVALID_ARG;
    if (a.dX && a.dX == a.dZ) return MIPGEMM_ERR_INVALID_ARG;
    if (a.N == 0) return MIPGEMM_OK;
    if (a.M > 0) {
        if ((pre && (!a.dH || !a.Y)) || (!pre && !a.dY) || ((post || pre) && !a.stats)) return MIPGEMM_ERR_INVALID_ARG;
        if (!a.Z && (post || a.dgate)) return MIPGEMM_ERR_INVALID_ARG;
    }
    for (const StepMatrix& out : {StepMatrix{a.dX, a.lddx}, StepMatrix{a.dZ, a.lddz}})
        for (const StepMatrix& in : {StepMatrix{a.dY, a.lddy}, StepMatrix{a.dH, a.lddh}, StepMatrix{a.Y, a.ldy}, StepMatrix{a.Z, a.ldz}})
            if (out.p && out.p == in.p && out.ld != in.ld) return MIPGEMM_ERR_INVALID_ARG;
    a.sums = (a.dpost_w != nullptr) + (a.dpost_b != nullptr) + (a.dpre_w != nullptr) + (a.dpre_b != nullptr);
    if (a.M == 0 && a.sums == 0) return MIPGEMM_OK;
    if (!a.gate) a.gate_rows = 1;        // (the kernels divide by it)
    else if (a.gate_rows > a.M) a.gate_rows = std::max<long long>(a.M, 1);
    DeviceState* dev = nullptr;
    int st = get_device(&dev);
    if (st != MIPGEMM_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_v);
    if (!post && !pre && !a.dgate && (!a.dX || !a.dZ)) {
        // nothing is summed: dx = s dy, or dz = dropout(gate * dy), are the forward kernel's without norms (16384 x 8192 bf16, dz: 161 -> 130 us)
        mip::StepArgs f = {};
        f.M = a.M; f.N = a.N;
        f.wide = a.wide;
        f.wide_vectors = true;
        f.gate_rows = 1;
        if (a.dX) {
            f.X = a.dY; f.ldx = a.lddy;
            f.x_scale = a.x_scale;
            f.Y = a.dX; f.ldy = a.lddx;
        } else {
            f.Z = a.dY; f.ldz = a.lddy;
            f.gate = a.gate; f.ldgate = a.ldgate; f.gate_rows = a.gate_rows;
            f.mask = a.mask;
            f.Y = a.dZ; f.ldy = a.lddz;
        }
        const cudaError_t e = mip::launch_norm_step(type, f, dev->sm_count, stream);
        ++g_launches;
        return e == cudaSuccess ? MIPGEMM_OK : cuda_fail(e);
    }
    size_t need = a.M > 0 ? mip::plan_norm_step_grad(a, dev->sm_count, mip::kMostWorkers) : 0;
    // (a lent buffer need not hold more than two workers' sums for each SM)
    if (dev->lent && need > dev->lent_bytes) need = mip::plan_norm_step_grad(a, dev->sm_count, mip::kFewWorkers);
    Scratch scratch(dev, stream);
    if ((st = scratch.reserve(need)) != MIPGEMM_OK) return st;
    int launches = 0;
    const cudaError_t e = mip::launch_norm_step_grad(type, a, scratch.base, stream, &launches);
    g_launches += launches;
    return e == cudaSuccess ? MIPGEMM_OK : cuda_fail(e);
}
