"""Scratch memory that the library keeps between calls: how much of it there is, and what a call that needs more does."""
import ctypes

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def mg():
    import torch
    from paper_2506_11728_b200 import binding
    binding.mipgemm_set_tuning()
    torch.cuda.synchronize()
    binding.mipgemm_release_staging()
    torch.cuda.empty_cache()
    yield binding
    torch.cuda.synchronize()
    binding.mipgemm_release_staging()
    torch.cuda.empty_cache()


class OwnStream:
    """A stream of its own, destroyed on leaving (torch.cuda.Stream hands out a fixed set of them)."""

    def __enter__(self):
        import torch
        handle = ctypes.c_void_p()
        assert int(torch.cuda.cudart().cudaStreamCreate(ctypes.addressof(handle))) == 0
        self.handle = handle.value
        return self.handle

    def __exit__(self, *exc):
        import torch
        assert int(torch.cuda.cudart().cudaStreamDestroy(self.handle)) == 0


def free_memory():
    import torch
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


class Call:
    """A product of ones whose B has an odd pitch: it is re-pitched into N * (K + 15) bytes of scratch."""
    M = 4

    def __init__(self, mg, N, K=16369):
        import torch
        self.mg, self.N, self.K = mg, N, K
        self.scratch = N * (K + 15)
        self.A = torch.ones(self.M, K + 15, dtype=torch.int8, device="cuda")
        self.B = torch.ones(N, K, dtype=torch.int8, device="cuda")
        self.C = torch.zeros(self.M, N, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()

    def __call__(self, stream):
        return self.mg.mipgemm_s8s8s32(self.M, self.N, self.K, self.A, self.K + 15, self.B, self.K, self.C, self.N, stream=stream)

    def check(self):
        import torch
        torch.cuda.synchronize()
        assert bool((self.C == self.K).all())


def test_release_frees_every_block(mg):
    import torch
    calls = [Call(mg, 4096) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in calls]          # (making them takes memory of its own)
    calls[0](streams[0])
    calls[0].check()
    mg.mipgemm_release_staging()
    before = free_memory()
    for c, s in zip(calls, streams):
        c(s)
    for c in calls:
        c.check()
    assert before - free_memory() >= calls[0].scratch
    mg.mipgemm_release_staging()
    assert before - free_memory() <= 4 << 20


def test_streams_that_come_and_go(mg):
    """A program that makes a stream for each request keeps the scratch of one, not of all that there were."""
    c = Call(mg, 4096)
    with OwnStream() as stream:
        c(stream)
        c.check()
    mg.mipgemm_release_staging()
    before = free_memory()
    for _ in range(50):
        with OwnStream() as stream:
            c.C.zero_()
            free_memory()
            c(stream)
            c.check()
    assert before - free_memory() <= 2 * c.scratch


def test_a_block_in_use_is_not_handed_on(mg):
    """Two streams at once, and the same with the roles changed: neither may read the other's copy of its operand."""
    import torch
    calls = [Call(mg, 4096 + 16 * i) for i in range(2)]
    calls[1].B.fill_(-1)
    streams = [torch.cuda.Stream() for _ in calls]
    for turn in range(6):
        for c in calls:
            c.C.zero_()
        torch.cuda.synchronize()
        for i in range(2):
            s = streams[(i + turn) % 2]
            with torch.cuda.stream(s):
                torch.cuda._sleep(2_000_000)            # (about a millisecond: the second call is made while the first waits)
            calls[i](s)
        torch.cuda.synchronize()
        assert bool((calls[0].C == calls[0].K).all()) and bool((calls[1].C == -calls[1].K).all())


def test_growing_waits_for_no_other_work(mg):
    """Calls are asynchronous, those that need more scratch than there is included: they return while another stream, and
    their own, are busy with what was enqueued before."""
    import torch
    small, large = Call(mg, 1024), Call(mg, 4096)
    other, own = torch.cuda.Stream(), torch.cuda.Stream()
    small(own)
    small.check()
    busy = []
    for s in (other, own):
        with torch.cuda.stream(s):
            torch.cuda._sleep(600_000_000)              # (about 0.3 s)
            busy.append(torch.cuda.Event())
            busy[-1].record()
    large(own)
    assert not any(e.query() for e in busy)
    large.check()


def test_growing_sizes_reach_the_allocator_a_few_times(mg):
    """Slowly growing calls: blocks grow by half, so that the memory in use never passes 1.5 times the largest need."""
    c = Call(mg, 4096)
    free = []
    for N in range(1024, 4097, 64):
        c.N = N
        c.C.zero_()
        c(None)
        free.append(free_memory())
        assert bool((c.C.view(-1)[:c.M * N] == c.K).all())
    assert len(set(free)) <= 8                          # log(4) / log(1.5) = 3.4 growths, and the caching allocator's own
    assert free[0] - free[-1] <= 1.5 * c.scratch + (8 << 20)


def test_no_memory_left_but_what_idle_blocks_hold(mg):
    """Two streams' idle blocks hold what a third stream's call needs: it gets it."""
    import torch
    calls, large = [Call(mg, 16384) for _ in range(2)], Call(mg, 30000)
    assert max(c.scratch for c in calls) < large.scratch < sum(c.scratch for c in calls)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for c, s in zip(calls, streams):
        with torch.cuda.stream(s):
            torch.cuda._sleep(20_000_000)               # (both at once, so that each has a block of its own)
        c(s)
    for c in calls:
        c.check()
    held = torch.empty(free_memory() - (100 << 20), dtype=torch.uint8, device="cuda")
    assert large.scratch > max(c.scratch for c in calls) + free_memory()
    large(streams[2])
    large.check()
    for c, s in zip(calls, streams):                    # the others wait their turn for what is left
        c.C.zero_()
        torch.cuda.synchronize()
        c(s)
        c.check()
    del held
