// Epilogue shared by the tensor-core kernels of the 8-bit layer: accumulators in tensor memory -> outputs.
//
// Thread = row.  A slot is 32 output columns of 32 rows (64 bytes a row in a 16-bit type, 128 in float32): the warp's
// own swizzled staging buffer.  A matrix that is read (residual, gradient of the output, the sum to add to) arrives in
// the slot by a TMA tile load asked for before the accumulator is ready, is combined in registers, and the result
// goes back to the same 16 bytes, from where a TMA tile store takes it: no global access is narrower than a row of the
// slot, no warp waits for another, and reading a matrix in place is safe (each element is read before the same warp
// writes it).  Matrices the TMA cannot address (16-byte alignment of base and pitch; for stores also whole 16-byte
// pieces per row, because tile stores clip in those) go through the same slot with one row of element accesses per
// instruction.  Scales and bias of a slot's columns are fetched one lane per column one slot ahead and broadcast
// through shared memory.
//
// What bounds it.  An output of an activated layer takes 14 to 28 scheduler clocks for a warp's 32 (a gradient's two 46),
// the exponential, the reciprocal and the conversions from integers among them on quarter- and half-rate units; beside a
// short main loop that is the kernel's time, and what counts is how well the schedulers are fed: one warp each issues
// every fifth clock or so, so there are two or four per scheduler, which take the slots of a tile by turns.  Measured:
// linear 16384 x 4096 x 1024 gelu bf16 81 us, 62 without the activation.  Where the pitch of C is not a multiple of 16
// bytes the element form makes that twice as much and more (linear 11957 x 3640 / 3641 x 112 bf16: 34 / 69 us):
// every row of a slot begins and ends inside a 32-byte sector, and the memory system completes partly written sectors
// one by one.
#pragma once
#include "internal.h"
#include "layer_math.cuh"
#include "ptx.cuh"

namespace mip {

namespace {

constexpr int kSlotCols = 32;
constexpr int slot_bytes(bool wide) { return wide ? 4096 : 2048; }
constexpr int kColBytes = 2 * kSlotCols * 4;        // per warp: two vectors of a slot's columns
// Epilogue warps (a multiple of four: a warp reads one quarter of the accumulator's lanes): 8, or 16 for 16-bit outputs
// behind a short K, where they set the pace.  Behind a long one their staging is better spent on pipeline stages.  (The
// float32 forms' slots are twice as large; the product's conversion warps take the registers of more.)
constexpr int kFewEpiWarps = 8, kManyEpiWarps = 16;
constexpr int product_epi_warps(bool wide) { return wide ? 4 : 8; }
// Slots per warp: two where there is something to wait for or nothing else to do meanwhile; gated forms have half the
// output columns (gradient: two buffers per slot, one per result; the incoming gradient lies in the first), the
// product's pipeline stages need the room.
constexpr int slot_count(int op) { return op == kOpRaw || op == kOpRawGated ? 0 : (op == kOpLinear ? 2 : 1); }
constexpr int slot_stride(int op, bool wide) { return op == kOpGatedGrad ? 2 * slot_bytes(wide) : slot_bytes(wide); }
constexpr int slot_bytes_per_warp(int op, bool wide) { return slot_count(op) * slot_stride(op, wide); }

struct LayerTile {
    int m0, n0;
    int kb0, kb1;        // k-blocks of this unit
    int plane;           // first row of its plane of partial sums
};

__device__ __forceinline__ LayerTile decode_tile(const LayerParams& p, int unit, int rows_per_tile) {
    // the units of a tile (K split) follow one another; tiles: groups of 8 tile columns swept top to bottom, column
    // fastest, so that a group's weights stay in the L2
    LayerTile c;
    int t = unit, ks = 0;
    if (p.split > 1) {
        t = unit / p.split;
        ks = unit - t * p.split;
    }
    const int per_group = 8 * p.tiles_m;
    const int g = t / per_group;
    const int first = g * 8;
    const int gsize = min(8, p.tiles_n - first);
    const int r = t - g * per_group;
    const int tm = r / gsize;
    c.m0 = tm * rows_per_tile;
    c.n0 = (first + (r - tm * gsize)) * p.out_n;
    c.kb0 = ks * p.kb_share;
    c.kb1 = min(p.k_blocks, c.kb0 + p.kb_share);
    c.plane = ks * p.plane_rows;
    return c;
}
__device__ __forceinline__ int layer_units(const LayerParams& p) { return p.tiles_m * p.tiles_n * max(p.split, 1); }

// Shared-memory address of 16 bytes of a slot's row, in the swizzle of a TMA box of 64- or 128-byte rows.
template <bool kWide>
__device__ __forceinline__ uint32_t slot_piece(uint32_t slot, int row, int piece) {
    if (kWide) return slot + static_cast<uint32_t>(row) * 128u + (static_cast<uint32_t>(piece ^ (row & 7)) << 4);
    return slot + static_cast<uint32_t>(row) * 64u + (static_cast<uint32_t>(piece ^ ((row >> 1) & 3)) << 4);
}
__device__ __forceinline__ void lds_v4(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void lds_f4(uint32_t addr, float (&v)[4]) {
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void sts_f32(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi, bool f16) {
    uint32_t r;
    if (f16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void unpack2(uint32_t w, bool f16, float& lo, float& hi) {
    if (f16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        lo = f.x;
        hi = f.y;
    } else {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xFFFF0000u);
    }
}

// Two int32 sums as binary32, rounded to nearest even.  (The conversion instruction.  Halves behind the exponent of 2^23
// and one fused multiply-add give the same float on other pipes, and cost the epilogues 15 %.)
__device__ __forceinline__ uint64_t ints_to_f2(uint32_t a, uint32_t b) {
    return pack_f2(__int2float_rn(static_cast<int>(a)), __int2float_rn(static_cast<int>(b)));
}

// A slot between shared and global memory, one row per instruction (lane = column), element by element: any alignment.
// Sixteen rows' accesses at a time, so that a load's latency is paid once per sixteen rows.
template <bool kWide>
__device__ __forceinline__ uint32_t slot_element(uint32_t slot, int row, int col) {
    constexpr int kPer = kWide ? 4 : 8;
    return slot_piece<kWide>(slot, row, col / kPer) + static_cast<uint32_t>(col % kPer) * (kWide ? 4u : 2u);
}
template <bool kWide>
__device__ __forceinline__ void slot_rows_in(uint32_t slot, const void* src, long long ld, int row0, int col0, int M, int N, int lane) {
    using Raw = std::conditional_t<kWide, uint32_t, uint16_t>;
    const int rows = min(32, M - row0);
    const Raw* at = static_cast<const Raw*>(src) + static_cast<long long>(row0) * ld + col0 + lane;
    const bool in = col0 + lane < N;
    for (int r0 = 0; r0 < rows; r0 += 16) {
        Raw v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            v[r] = Raw(0);
            if (in && r0 + r < rows) v[r] = at[static_cast<long long>(r0 + r) * ld];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (kWide) asm volatile("st.shared.b32 [%0], %1;" ::"r"(slot_element<kWide>(slot, r0 + r, lane)), "r"(static_cast<uint32_t>(v[r])) : "memory");
            else asm volatile("st.shared.b16 [%0], %1;" ::"r"(slot_element<kWide>(slot, r0 + r, lane)), "h"(static_cast<uint16_t>(v[r])) : "memory");
        }
    }
    __syncwarp();
}
template <bool kWide>
__device__ __forceinline__ void slot_rows_out(uint32_t slot, void* dst, long long ld, int row0, int col0, int M, int N, int lane) {
    using Raw = std::conditional_t<kWide, uint32_t, uint16_t>;
    __syncwarp();
    const int rows = min(32, M - row0);
    Raw* at = static_cast<Raw*>(dst) + static_cast<long long>(row0) * ld + col0 + lane;
    const bool in = col0 + lane < N;
    for (int r0 = 0; r0 < rows; r0 += 16) {
        Raw v[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (kWide) {
                uint32_t x;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(slot_element<kWide>(slot, r0 + r, lane)) : "memory");
                v[r] = static_cast<Raw>(x);
            } else {
                uint16_t x;
                asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x) : "r"(slot_element<kWide>(slot, r0 + r, lane)) : "memory");
                v[r] = static_cast<Raw>(x);
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (in && r0 + r < rows) at[static_cast<long long>(r0 + r) * ld] = v[r];
    }
    __syncwarp();
}

// kN accumulator columns of one row: v0 (and, gated, v1) become outputs in the slot.  `col` is the first of them in the
// slot, `cols` the shared-memory address of the slot's column vectors.  The slot's old contents are the residual / the
// gradient of the output.
template <int kOp, int kAct, bool kWide, int kN>
__device__ __forceinline__ void finish_chunk(const uint32_t (&v0)[kN], const uint32_t (&v1)[kN], float as, uint32_t cols, uint32_t slot,
                                             uint32_t slot2, int row, int col, bool has_r, bool f16) {
    constexpr int kPer = kWide ? 4 : 8;             // columns per 16-byte piece
    constexpr int kPieces = kN / kPer;
    const int piece0 = col / kPer;
    struct Inputs {
        float b0[kPer], b1[kPer];
        uint32_t r[4];
    };
    const auto fetch = [&](int g) {
        Inputs in;
        if constexpr (kOp != kOpProduct) {
#pragma unroll
            for (int h = 0; h < kPer; h += 4) {
                lds_f4(cols + (col + g * kPer + h) * 4, reinterpret_cast<float (&)[4]>(in.b0[h]));
                lds_f4(cols + kSlotCols * 4 + (col + g * kPer + h) * 4, reinterpret_cast<float (&)[4]>(in.b1[h]));
            }
        }
        if (kOp != kOpGated) {
            if (has_r) {
                lds_v4(slot_piece<kWide>(slot, row, piece0 + g), in.r);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) in.r[j] = 0u;
            }
        }
        return in;
    };
    const uint64_t as2 = pack_f2(as, as);
#pragma unroll
    for (int g = 0; g < kPieces; ++g) {
        const Inputs in = fetch(g);
        uint64_t r[kPer / 2], y[kPer / 2], y2[kPer / 2];           // two columns each
        if constexpr (kOp != kOpGated) {
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j) {
                if constexpr (kWide) {
                    r[j] = pack_f2(__uint_as_float(in.r[2 * j]), __uint_as_float(in.r[2 * j + 1]));
                } else {
                    float lo, hi;
                    unpack2(in.r[j], f16, lo, hi);
                    r[j] = pack_f2(lo, hi);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
            const int v = g * kPer + 2 * j;
            if constexpr (kOp == kOpProduct) {
                y[j] = add_f2(pack_f2(__uint_as_float(v0[v]), __uint_as_float(v0[v + 1])), r[j]);
            } else {
                const uint64_t s0 = mul_f2(ints_to_f2(v0[v], v0[v + 1]), as2);
                const uint64_t b0 = pack_f2(in.b0[2 * j], in.b0[2 * j + 1]), b1 = pack_f2(in.b1[2 * j], in.b1[2 * j + 1]);
                if constexpr (kOp == kOpLinear) {
                    y[j] = add_f2(activation_f2<kAct, kWide>(fma_f2(s0, b0, b1)), r[j]);
                } else {
                    const uint64_t z1 = mul_f2(mul_f2(ints_to_f2(v1[v], v1[v + 1]), as2), b1);
                    if constexpr (kOp == kOpGated) {
                        y[j] = mul_f2(activation_f2<kAct, kWide>(mul_f2(s0, b0)), z1);
                    } else {
                        uint64_t value, slope;
                        activation_slope_f2<kAct, kWide>(mul_f2(s0, b0), value, slope);
                        y[j] = mul_f2(mul_f2(r[j], z1), slope);
                        y2[j] = mul_f2(r[j], value);
                    }
                }
            }
        }
        const auto put = [&](uint32_t at, const uint64_t (&x)[kPer / 2]) {
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j) {
                float lo, hi;
                unpack_f2(x[j], lo, hi);
                if constexpr (kWide) {
                    o[2 * j] = __float_as_uint(lo);
                    o[2 * j + 1] = __float_as_uint(hi);
                } else {
                    o[j] = pack2(lo, hi, f16);
                }
            }
            st_shared_v4(at, o);
        };
        put(slot_piece<kWide>(slot, row, piece0 + g), y);
        if constexpr (kOp == kOpGatedGrad) put(slot_piece<kWide>(slot2, row, piece0 + g), y2);
    }
}

// Partial sums as they are (32-bit words) to the unit's plane.  A lane has a row's 32 columns and stores them as four whole
// 32-byte sectors, straight from registers: as fast as staging and TMA tile stores (product 848 x 5664 x 18608 bf16 193 /
// 196 us, 1024 x 1024 x 8192 26.8 / 26.9), and the staging's shared memory goes to pipeline stages.
// kHalves: the accumulator holds two projections side by side; kSubs warps take a tile's columns by turns of 32, this one
// every kSubs-th from `sub`.
template <bool kPair, bool kHalves, int kSubs>
__device__ __forceinline__ void raw_epilogue(const LayerParams& p, int sub, uint32_t bar_tfull, uint32_t bar_tempty,
                                             volatile uint32_t* abort_flag, uint32_t tmem_base, int q, int lane, uint32_t cta_rank,
                                             int first_unit, int unit_stride) {
    constexpr int kRowsPerTile = kPair ? 2 * kBlockM : kBlockM;
    const bool leader = cta_rank == 0;
    const int total_units = layer_units(p);
    int t = 0;
    for (int unit = first_unit; unit < total_units; unit += unit_stride, ++t) {
        const LayerTile tc = decode_tile(p, unit, kRowsPerTile);
        const uint32_t acc = t & 1, acc_phase = (t >> 1) & 1;
        const int row0 = tc.m0 + static_cast<int>(cta_rank) * kBlockM + q * 32;
        const int n_here = min(p.out_n, p.N - tc.n0);
        if (!mbar_wait_warp(bar_tfull + 8u * acc, acc_phase, abort_flag, p.wait_budget_ns)) break;
        tc_fence_after();
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * p.block_n;
        // (planes have whole blocks of 32 rows and columns)
        int32_t* const out = static_cast<int32_t*>(p.C) + static_cast<long long>(tc.plane + row0 + lane) * p.ldc + tc.n0;
        for (int c0 = 32 * sub; c0 < p.block_n && row0 < p.M; c0 += 32 * kSubs) {
            const bool second = kHalves && c0 >= p.out_n;
            const int c = second ? c0 - p.out_n : c0;
            if (c >= n_here) continue;
            uint32_t v[32];
            tmem_ld_32x32(t_row + c0, v);
            tmem_ld_wait_for(v);
#pragma unroll
            for (int j = 0; j < 4; ++j) st_global_v8(out + (second ? p.plane_second : 0) + c + 8 * j, &v[8 * j]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (kPair && !leader) mbar_arrive_remote_fenced(bar_tempty + 8u * acc, 0);
            else mbar_arrive(bar_tempty + 8u * acc);
        }
    }
}

// The epilogue role of one warp (e = 0 .. kWarps-1; q = the quarter of the TMEM lanes it may read).  Walks
// the same tiles as the other roles; `slots`, `colvec` and `bar_in` are the shared-memory addresses of the slots, column
// vectors and arrival barriers of all warps.
template <bool kPair, int kOp, bool kWide, int kWarps>
__device__ __forceinline__ void layer_epilogue(const LayerParams& p, uint32_t slots, uint32_t colvec, uint32_t bar_in, uint32_t bar_tfull,
                                               uint32_t bar_tempty, volatile uint32_t* abort_flag, uint32_t tmem_base, int e, int q, int lane,
                                               uint32_t cta_rank, int first_unit, int unit_stride) {
    constexpr bool kGatedForm = kOp == kOpGated || kOp == kOpGatedGrad;
    constexpr int kRowsPerTile = kPair ? 2 * kBlockM : kBlockM;
    constexpr int kBuffers = slot_count(kOp);
    constexpr int kSlotStride = slot_stride(kOp, kWide);
    constexpr int kSlotBytesPerWarp = slot_bytes_per_warp(kOp, kWide);
    constexpr int kSubs = kWarps / 4;
    const int sub = e >> 2;
    const bool leader = cta_rank == 0;
    const int total_units = layer_units(p);
    const uint64_t budget = p.wait_budget_ns;
    const uint32_t my_slots = slots + static_cast<uint32_t>(e) * kSlotBytesPerWarp;
    const uint32_t my_cols = colvec + static_cast<uint32_t>(e) * kColBytes;
    const uint32_t my_bar = bar_in + 8u * static_cast<uint32_t>(e * kBuffers);
    const bool f16 = p.type == kF16;
    const bool has_r = p.R != nullptr;
    const bool r_tma = p.r_tma != 0, c_tma = p.c_tma != 0;
    uint32_t loads = 0, slot_no = 0;                           // tile loads asked for, slots finished
    // slots of a tile this warp finishes, and the column of its i-th
    const auto slots_of = [&](const LayerTile& c) {
        const int n_here = min(p.out_n, p.N - c.n0);
        const bool active = c.m0 + static_cast<int>(cta_rank) * kBlockM + q * 32 < p.M;       // (warp-uniform)
        return active ? ((n_here + kSlotCols - 1) / kSlotCols - sub + kSubs - 1) / kSubs : 0;
    };
    const auto slot_col = [&](int i) { return (sub + i * kSubs) * kSlotCols; };
    // a tile's row scale and a slot's column vectors, one lane per row / column; asked for one slot or tile ahead
    float cv0 = 1.0f, cv1 = 0.0f, as = 1.0f;
    const auto fetch_columns = [&](const LayerTile& c, int i) {
        if (kOp == kOpProduct) return;
        const int col = c.n0 + slot_col(i) + lane;
        const bool in = col < p.N;
        cv0 = (in && p.b0_scale) ? __ldg(p.b0_scale + col) : 1.0f;
        if (kGatedForm) cv1 = (in && p.b1_scale) ? __ldg(p.b1_scale + col) : 1.0f;
        else cv1 = (in && p.bias) ? __ldg(p.bias + col) : 0.0f;
    };
    const auto fetch_row = [&](const LayerTile& c) {
        const int row = c.m0 + static_cast<int>(cta_rank) * kBlockM + q * 32 + lane;
        return (kOp != kOpProduct && p.a_scale && row < p.M) ? __ldg(p.a_scale + row) : 1.0f;
    };
    LayerTile next = {};
    if (first_unit < total_units) {
        next = decode_tile(p, first_unit, kRowsPerTile);
        as = fetch_row(next);
        fetch_columns(next, 0);
    }
    int t = 0;
    for (int unit = first_unit; unit < total_units; unit += unit_stride, ++t) {
        const LayerTile tc = next;
        const bool more = unit + unit_stride < total_units;
        if (more) next = decode_tile(p, unit + unit_stride, kRowsPerTile);
        const uint32_t acc = t & 1, acc_phase = (t >> 1) & 1;
        const int row0 = tc.m0 + static_cast<int>(cta_rank) * kBlockM + q * 32;
        const int n_slots = slots_of(tc);
        const float as_here = as;
        // the slots' first buffers: every store that still reads them has been issued by this warp
        int asked = 0;                                         // of this tile
        const auto ask = [&] {
            const uint32_t b = loads % kBuffers;
            if (elect_one()) {
                mbar_arrive_expect_tx(my_bar + 8u * b, slot_bytes(kWide));
                tma_load_2d(my_slots + b * kSlotStride, &p.tmap_r, my_bar + 8u * b, tc.n0 + slot_col(asked), row0);
            }
            ++asked;
            ++loads;
        };
        if (r_tma) {
            if (n_slots > 0) {
                if (elect_one()) tma_store_wait_read<0>();
                __syncwarp();
                fence_proxy_async_smem();
                __syncwarp();
                while (asked < kBuffers && asked < n_slots) ask();
            }
            // the L2 is asked for what the next tile will read: its loads cannot start before this tile's stores have
            // left their buffers
            const int ahead = more ? slots_of(next) : 0;
            if (elect_one())
                for (int i = 0; i < ahead; ++i)
                    tma_prefetch_l2_2d(&p.tmap_r, next.n0 + slot_col(i), next.m0 + static_cast<int>(cta_rank) * kBlockM + q * 32);
            __syncwarp();
        }
        // the same for a residual that is read element by element: what the buffers hold, before the accumulator is waited for
        const auto fill = [&] {
            slot_rows_in<kWide>(my_slots + (loads % kBuffers) * kSlotStride, p.R, p.ldr, row0, tc.n0 + slot_col(asked), p.M, p.N, lane);
            ++asked;
            ++loads;
        };
        const bool r_rows = has_r && !r_tma;
        if (r_rows && n_slots > 0) {
            if (c_tma && elect_one()) tma_store_wait_read<0>();
            __syncwarp();
            while (asked < kBuffers && asked < n_slots) fill();
        }
        if (n_slots == 0 && more) {
            as = fetch_row(next);
            fetch_columns(next, 0);
        }
        // (the lanes of a warp decide together: none may leave while others still expect it at a warp barrier)
        if (!mbar_wait_warp(bar_tfull + 8u * acc, acc_phase, abort_flag, budget)) break;
        tc_fence_after();
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * p.block_n;
        const uint32_t t_up = t_row + static_cast<uint32_t>(p.block_n >> 1);
        // the accumulator is the MMA warp's again once this warp has read its last columns of it
        const auto release = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (kPair && !leader) mbar_arrive_remote_fenced(bar_tempty + 8u * acc, 0);
                else mbar_arrive(bar_tempty + 8u * acc);
            }
        };
        if (n_slots == 0) release();
        bool gave_up = false;
        for (int sl = 0; sl < n_slots; ++sl, ++slot_no) {
            const int c0 = slot_col(sl);
            const uint32_t b = slot_no % kBuffers;
            const uint32_t slot = my_slots + b * kSlotStride, slot2 = slot + slot_bytes(kWide);
            uint32_t v[kGatedForm ? 16 : 32], v1[16];
            __syncwarp();                                      // tcgen05.ld wants the whole warp: the elected lane is back
            if constexpr (!kGatedForm) tmem_ld_32x32(t_row + c0, v);
            // the slot is free (its last store has been read) or holds the tile that was asked for
            if (!r_tma) {
                if (c_tma && elect_one()) tma_store_wait_read<kBuffers - 1>();
                __syncwarp();
                if (r_rows && asked == sl) fill();
            }
            if (kOp != kOpProduct) {
                __syncwarp();                                  // (the last slot's column vectors have been read)
                sts_f32(my_cols + lane * 4, cv0);
                sts_f32(my_cols + kSlotCols * 4 + lane * 4, cv1);
                __syncwarp();
            }
            if (sl + 1 < n_slots) {
                fetch_columns(tc, sl + 1);
            } else if (more) {
                as = fetch_row(next);
                fetch_columns(next, 0);
            }
            if (r_tma && !mbar_wait_warp(my_bar + 8u * b, (slot_no / kBuffers) & 1u, abort_flag, budget)) {
                gave_up = true;
                break;
            }
            if constexpr (kGatedForm) {
                // (16 columns of both projections at a time: registers for four epilogue warps per scheduler)
#pragma unroll 1
                for (int c = 0; c < kSlotCols; c += 16) {
                    __syncwarp();
                    tmem_ld_32x16(t_row + c0 + c, v);
                    tmem_ld_32x16(t_up + c0 + c, v1);
                    tmem_ld_wait_for16(v, v1);
                    if (sl + 1 == n_slots && c + 16 == kSlotCols) release();
                    with_activation(p.act, [&](auto act) {
                        finish_chunk<kOp, decltype(act)::value, kWide, 16>(v, v1, as_here, my_cols, slot, slot2, lane, c, has_r, f16);
                    });
                }
            } else {
                tmem_ld_wait_for(v);
                if (sl + 1 == n_slots) release();
                with_activation(kOp == kOpProduct ? kActNone : p.act, [&](auto act) {
                    finish_chunk<kOp, decltype(act)::value, kWide, 32>(v, v, as_here, my_cols, slot, slot2, lane, 0, has_r, f16);
                });
            }
            if (c_tma) {
                fence_proxy_async_smem();
                __syncwarp();
                if (elect_one()) {
                    tma_store_2d(&p.tmap_c, slot, tc.n0 + c0, row0);
                    if (kOp == kOpGatedGrad) tma_store_2d(&p.tmap_c2, slot2, tc.n0 + c0, row0);
                    tma_store_commit();
                }
            } else {
                slot_rows_out<kWide>(slot, p.C, p.ldc, row0, tc.n0 + c0, p.M, p.N, lane);
                if (kOp == kOpGatedGrad) slot_rows_out<kWide>(slot2, p.C2, p.ldc2, row0, tc.n0 + c0, p.M, p.N, lane);
            }
            // ask for the tile of a later slot once the buffer it goes to has been read by its store: the one
            // before last (the last store may still be reading its own), unless there is only one buffer
            if (r_tma && (kBuffers == 1 || sl > 0) && asked < n_slots) {
                if (elect_one()) tma_store_wait_read<kBuffers == 1 ? 0 : 1>();
                __syncwarp();
                fence_proxy_async_smem();
                __syncwarp();
                ask();
            }
        }
        if (gave_up) break;
    }
    // unwinding: tiles still on their way into the slots
    for (uint32_t i = slot_no; r_tma && i < loads; ++i) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait(my_bar + 8u * (i % kBuffers), (i / kBuffers) & 1u)) {
            if (globaltimer_ns() - t0 > budget) break;
        }
    }
    if (c_tma && elect_one()) tma_store_wait<0>();
    __syncwarp();
}

}  // namespace

}  // namespace mip
