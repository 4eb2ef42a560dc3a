"""Block tables, slot maps and page lists against their definitions, worked out request by request in Python integers.  All
outputs are whole numbers, so the tolerance is equality, untouched entries included."""
import numpy as np
import pytest
import torch

from paper_2605_06113_b200 import workload as wlm
from paper_2605_06113_b200.binding import BlockCache, Router

import cache_reference as ref
from cache_reference import EMPTY, MOST

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# N, G, B, tokens a block, blocks a pool, columns a row
SHAPES = [(1, 1, 1, 1, 1, 1), (1, 4, 64, 16, 700, 90), (3, 5, 7, 24, 60, 31), (2, 3, 256, 16, 5000, 65), (70, 33, 8, 5, 97, 40),
          (300, 9, 33, 64, 150, 17), (1, 64, 40, 1, 900, 333), (2, 1, 65, 128, 4099, 1030), (1, 2, 9, 100, 3000, 2500),
          (5, 1, 255, 7, 33, 6), (1, 1, 130, 3, 20011, 1000)]
# enough workers for teams of one warp, with one and two slots a lane, and for the smallest teams of wide workers
BATCHES = [(2500, 8, 16, 16, 64, 9), (620, 8, 50, 16, 120, 11), (150, 8, 130, 16, 300, 12)]


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


class Pair:
    """A cache on the GPU and its host copy."""

    def __init__(self, N, G, B, t, P, T, seed=0):
        self.f = ref.Fleets(N, G, B, t, P, T)
        rng = np.random.default_rng(seed)
        for at in self.f.workers():
            rng.shuffle(self.f.free_list[at])
        self.c = BlockCache(_gpu(self.f.table), _gpu(self.f.n_blocks), _gpu(self.f.free_list), _gpu(self.f.n_free), t)

    def same(self, nb=None, nf=None):
        f, c = self.f, self.c
        for name, have, want in (("table", c.table, f.table), ("free_list", c.free_list, f.free_list),
                                 ("n_blocks", c.n_blocks if nb is None else nb[0], f.n_blocks if nb is None else nb[1]),
                                 ("n_free", c.n_free if nf is None else nf[0], f.n_free if nf is None else nf[1])):
            assert np.array_equal(have.cpu().numpy(), want), name

    def update(self, length, step=None, out=False, **kw):
        c, f = self.c, self.f
        short = torch.full((f.N, f.G), -77, dtype=torch.int32, device=DEV)
        nb, nf = (c.n_blocks.clone(), c.n_free.clone()) if out else (None, None)
        c.block_tables(_gpu(length), nb, nf, short, step=None if step is None else _gpu(step), **kw)
        wnb, wnf, wshort = f.update(length, step, commit=not out, **{k: v for k, v in kw.items() if k != "stream"})
        assert np.array_equal(short.cpu().numpy(), wshort)
        self.same((nb, wnb) if out else None, (nf, wnf) if out else None)
        if out:
            self.same()
        return wshort

    def slots(self, length, room, n_new=None, step=None, **kw):
        c, f = self.c, self.f
        cu = torch.full((f.N, f.G, f.B + 1), -7, dtype=torch.int32, device=DEV)
        out = torch.full((f.N, f.G, room), -7, dtype=torch.int64, device=DEV)
        c.slot_map(_gpu(length), cu, out, n_new=None if n_new is None else _gpu(n_new), step=None if step is None else _gpu(step), **kw)
        wcu, wout = f.slots(length, room, n_new, step, **kw)
        assert np.array_equal(cu.cpu().numpy(), wcu)
        assert np.array_equal(out.cpu().numpy(), wout)

    def pages(self, length, step=None, **kw):
        c, f = self.c, self.f
        z = dict(dtype=torch.int32, device=DEV)
        o = [torch.full(s, -7, **z) for s in ((f.N, f.G), (f.N, f.G, f.B), (f.N, f.G, f.B + 1), (f.N, f.G, f.P), (f.N, f.G, f.B))]
        c.page_lists(_gpu(length), *o, step=None if step is None else _gpu(step), **kw)
        for name, have, want in zip(("n_seq", "seq_slot", "indptr", "indices", "last_tokens"), o, f.pages(length, step, **kw)):
            assert np.array_equal(have.cpu().numpy(), want), name


def _walk(rng, f, n, ended, refill, grow):
    """The next lengths: requests end, slots are refilled, the others grow; sizes that use the pool up now and then."""
    most = min(f.T * f.t, int(2.2 * f.P * f.t / f.B) + 2)
    n = np.where((n > 0) & (rng.random(n.shape) >= ended), n + grow, 0)
    return np.where((n == 0) & (rng.random(n.shape) < refill), rng.integers(0, most + 1, n.shape), n)


@pytest.mark.parametrize("shape,stepped", [(s, k) for s in SHAPES for k in (False, True)] + [(s, True) for s in BATCHES])
def test_walks_of_lengths(shape, stepped):
    p = Pair(*shape, seed=sum(shape))
    f = p.f
    rng = np.random.default_rng(17 * sum(shape) + stepped)
    n = np.zeros((f.N, f.G, f.B), np.int64)
    big = f.N * f.G > 1000
    for k, (ended, refill, grow) in enumerate([(0, 0.7, 1), (0.0, 0.0, 1), (0.3, 0.6, 5), (0.01, 0.1, 1), (0.9, 0.2, 40)][:3 if big else 5]):
        n = _walk(rng, f, n, ended, refill, grow)
        step = rng.integers(-5, 10 ** 6, f.N).astype(np.int32) if stepped else None
        length = (np.where(n > 0, n - step[:, None, None], EMPTY) if stepped else n).astype(np.int32)
        if k % 2:
            p.update(length, step, out=True)                     # looked at and dropped
        p.update(length, step)
        n_new = rng.integers(-2, 60, n.shape).astype(np.int32)
        if k == 2:
            n_new = np.where(rng.random(n.shape) < 0.5, MOST, 0).astype(np.int32)
        p.slots(length, f.B, step=step)
        p.slots(length, int(rng.integers(1, 30 * f.B + 2)), n_new, step)
        p.pages(length, step)
        if not big:
            f.check_partition()
    later = (length + (length != EMPTY) * 3).astype(np.int32)    # tables that are behind the lengths, and ahead of them
    p.slots(later, 2 * f.B + 1, n_new, step)
    p.pages(later, step)
    earlier = (np.where(length == EMPTY, EMPTY, length // 2) if not stepped else length - 2 * (length != EMPTY)).astype(np.int32)
    p.slots(earlier, 2 * f.B + 1, n_new, step)
    p.pages(earlier, step)


@pytest.mark.parametrize("N,G", [(1, 1), (2, 64), (40, 64), (700, 8)])
def test_one_request_takes_the_whole_pool_and_gives_it_back(N, G):
    p = Pair(N, G, 24, 16, 1500, 1500, seed=N)
    n = np.zeros((N, G, 24), np.int32)
    n[:, :, 5] = 1500 * 16
    p.update(n)
    p.pages(n)
    p.slots(n, 300, np.full(n.shape, 301, np.int32))
    m = n.copy()
    m[:, :, 5] = 0
    m[:, :, 23] = 1499 * 16 + 1
    p.update(m, out=True)
    p.update(m)                                                  # all of its blocks go to another slot
    m[:, :, 3] = 1
    assert (p.update(m) == 1).all()                              # nothing left for one more
    p.update(np.zeros_like(m))
    p.f.check_partition()


def test_undoing_an_update_restores_tables_and_lists():
    p = Pair(6, 20, 64, 16, 900, 60, seed=3)
    rng = np.random.default_rng(4)
    A = rng.integers(0, 200, (6, 20, 64)).astype(np.int32)
    p.update(A)
    table, free = p.c.table.clone(), p.c.free_list.clone()
    nb, nf = p.c.n_blocks.clone(), p.c.n_free.clone()
    p.update((A + rng.integers(-90, 40, A.shape)).astype(np.int32))
    p.update(A)
    assert torch.equal(nb, p.c.n_blocks) and torch.equal(nf, p.c.n_free)
    held = torch.arange(60, device=DEV) < nb[..., None]
    listed = torch.arange(900, device=DEV) < nf[..., None]
    assert torch.equal(torch.where(held, table, 0), torch.where(held, p.c.table, 0))
    assert torch.equal(torch.where(listed, free, 0), torch.where(listed, p.c.free_list, 0))


@pytest.mark.parametrize("N,G", [(3, 8), (300, 8)])
def test_updates_in_turns_between_two_sets_of_counts(N, G):
    p = Pair(N, G, 50, 16, 700, 40, seed=6)
    rng = np.random.default_rng(7)
    n = np.zeros((N, G, 50), np.int64)
    spare = (torch.empty_like(p.c.n_blocks), torch.empty_like(p.c.n_free))
    for _ in range(6):
        n = _walk(rng, p.f, n, 0.2, 0.6, 3)
        p.c.block_tables(_gpu(n.astype(np.int32)), *spare)
        spare, old = (p.c.n_blocks, p.c.n_free), spare
        p.c.commit(*old)
        p.f.update(n.astype(np.int32))
        p.same()
        p.pages(n.astype(np.int32))
    p.f.check_partition()


@pytest.mark.parametrize("workers", [(1, 3), (900, 7)])
def test_counts_that_cannot_be_leave_the_worker_as_it_was(workers):
    N, G = workers
    for k, (name, value) in enumerate([("n_free", -1), ("n_free", 51), ("n_blocks", -1), ("n_blocks", 11), ("n_blocks", MOST),
                                       ("n_free", MOST), ("n_free", 45), ("n_blocks", -(2 ** 31))]):
        p = Pair(N, G, 12, 4, 50, 10, seed=k)
        n = np.full((N, G, 12), 3, np.int32)
        p.update(n)
        getattr(p.f, name)[N - 1, G - 1, ...] = value
        getattr(p.c, name)[N - 1, G - 1, ...] = value
        n[:, :, 2] = 0
        n[:, :, 7] = 21
        for out in (True, False):
            short = p.update(n, out=out)
            assert short[N - 1, G - 1] == -1 and (short.ravel()[:-1] == 0).all()
        p.slots(n, 40, np.full(n.shape, 3, np.int32))            # counts are clipped to the row
        p.pages(n)


def test_lengths_at_the_ends_of_their_range():
    N, G, B = 5, 2, 10
    edge = np.array([EMPTY, EMPTY + 1, -1, 0, 1, MOST, MOST - 5, 15, 16, 17], np.int32)
    length = np.tile(edge, (N, G, 1))
    step = np.array([0, 1, MOST, -(2 ** 31), -16], np.int32)
    for t in (16, 1, 1 << 20, (1 << 20) - 1):
        p = Pair(N, G, B, t, 4100, 2048, seed=t)
        p.update(length, step)
        p.update(length)
        p.slots(length, 50, np.full((N, G, B), 5, np.int32), step)
        p.slots(length, 10)
        p.pages(length, step)
    # sums of new tokens beyond 2^31 - 1
    p.slots(np.full((N, G, B), MOST, np.int32), 7, np.array([3] + [MOST] * 9, np.int32) * np.ones((N, G, 1), np.int32))


def test_more_new_tokens_than_31_bits_count():
    p = Pair(2, 2, 6, 1 << 20, 4100, 2048, seed=8)
    n = np.array([5, MOST, 7, 9, 3, 1], np.int32) * np.ones((2, 2, 1), np.int32)
    assert (p.update(n) == 0).all()
    for q in ([3, MOST, MOST, 9, 1, 1], [MOST, 0, MOST, MOST, MOST, MOST], [0, MOST, 0, 0, 0, 5]):
        p.slots(n, 41, np.array(q, np.int32) * np.ones((2, 2, 1), np.int32))


def test_cache_slots_beyond_32_bits():
    t = 1 << 20
    p = Pair(2, 3, 4, t, 5000, 2048, seed=9)                      # block 4999 starts at slot 5.2e9
    n = np.array([MOST, 5, t, t + 1], np.int32) * np.ones((2, 3, 1), np.int32)
    p.update(n)
    p.slots(n, 4000, np.full(n.shape, 999, np.int32))
    assert (p.f.table[p.f.table >= 0].astype(np.int64) * t).max() > 2 ** 32


def test_arrays_beyond_32_bits():
    """Tables, free lists, page lists and slot maps of more than 2^31 entries: the last workers' rows are behind that."""
    G, B, T, P, room = 64, 256, 140001, 34000001, 34000001
    z = dict(dtype=torch.int32, device=DEV)
    free = torch.empty((1, G, P), **z)
    free[:, :, P - 1000:] = torch.arange(999, -1, -1, **z)        # the end of the list, where blocks come from
    c = BlockCache(torch.empty((1, G, B, T), **z), torch.zeros((1, G, B), **z), free, torch.full((1, G), P, **z), 16)
    length = torch.zeros((1, G, B), **z)
    length[:, :, 254] = 16 * 900 + 3
    length[:, :, 255] = 16 * 20
    c.block_tables(length)
    assert c.n_blocks[0, :, 254].tolist() == [901] * G and c.n_blocks[0, :, 255].tolist() == [20] * G
    assert torch.equal(c.table[0, :, 254, :901], torch.arange(901, **z).expand(G, 901))
    assert torch.equal(c.table[0, :, 255, :20], torch.arange(901, 921, **z).expand(G, 20))
    cu, slots = torch.zeros((1, G, B + 1), **z), torch.empty((1, G, room), dtype=torch.int64, device=DEV)
    c.slot_map(length, cu, slots)
    assert slots[0, :, :2].tolist() == [[900 * 16 + 2, 921 * 16 - 1]] * G
    slots[:, :, 14723:14725] = -7
    c.slot_map(length, cu, slots, n_new=length)
    assert torch.equal(slots[0, :, :14403], torch.arange(14403, device=DEV).expand(G, 14403))
    assert torch.equal(slots[0, :, 14403:14723], torch.arange(901 * 16, 921 * 16, device=DEV).expand(G, 320))
    assert cu[0, :, -1].tolist() == [14723] * G and bool((slots[:, :, 14723:14725] == -7).all())
    del slots
    o = [torch.zeros(s, **z) for s in ((1, G), (1, G, B), (1, G, B + 1))] + [torch.empty((1, G, P), **z), torch.zeros((1, G, B), **z)]
    c.page_lists(length, *o)
    assert torch.equal(o[3][0, :, :921], torch.arange(921, **z).expand(G, 921)) and o[0].tolist() == [[2] * G]
    c.free_list[:, :, P - 1000:] = -5
    c.block_tables(torch.zeros_like(length))
    assert c.n_free.tolist() == [[P] * G]
    assert torch.equal(c.free_list[0, :, P - 921:], torch.arange(920, -1, -1, **z).expand(G, 921))
    assert bool((c.free_list[:, :, P - 1000:P - 921] == -5).all())


@pytest.mark.parametrize("N,G,B", [(3, 5, 40), (700, 8, 60), (1, 2, 256)])
def test_workers_without_requests_and_requests_without_tokens(N, G, B):
    p = Pair(N, G, B, 16, 300, 20, seed=2)
    nothing = np.full((N, G, B), EMPTY, np.int32)
    step = np.full(N, 7, np.int32)
    some = nothing.copy()
    some[:, ::2, B - 1] = 33                                      # every second worker runs one request, in its last slot
    for length in (nothing, some, np.zeros_like(nothing), nothing - 0 * nothing, np.full_like(nothing, -7), some):
        p.update(length, step)
        p.slots(length, 3, step=step)
        p.pages(length, step)
        for q in (0, -4, 1, MOST):
            p.slots(length, 50, np.full(nothing.shape, q, np.int32), step)
    sparse = np.zeros_like(nothing)
    sparse[:, :, [0, B // 2, B - 1]] = 9                          # new tokens in three slots of many running ones
    full = np.full_like(nothing, 20)
    p.update(full)
    p.slots(full, 100, sparse)
    p.pages(full)


@pytest.mark.parametrize("shape", [(7, 3, 20, 8, 80, 30), (500, 10, 8, 8, 40, 12)])
def test_rows_of_a_batch(shape):
    p = Pair(*shape, seed=11)
    f = p.f
    rng = np.random.default_rng(1)
    n = rng.integers(0, 60, (f.N, f.G, f.B)).astype(np.int32)
    step = rng.integers(0, 9, f.N).astype(np.int32)
    q = rng.integers(0, 9, n.shape).astype(np.int32)
    for first, N in ((2, 3), (0, 1), (f.N - 1, 1), (4, None)):
        rows = dict(first=first, N=f.N - first if N is None else N)
        p.update(n, step, **rows)
        p.slots(n, 37, q, step, **rows)
        p.pages(n, step, **rows)
    p.update(n, step, first=3, N=0)


def test_unaligned_tensors():
    """Arrays that start at any multiple of their elements' size, as slices of a larger buffer do."""
    shape = N, G, B, t, P, T = 3, 5, 23, 16, 301, 40
    rng = np.random.default_rng(2)
    for off in (1, 2, 3):
        p = Pair(*shape, seed=off)

        def shifted(a):
            flat = torch.zeros(a.numel() + 4, dtype=a.dtype, device=DEV)
            v = flat[off:off + a.numel()].view(a.shape)
            v.copy_(a)
            return v

        p.c = BlockCache(shifted(p.c.table), shifted(p.c.n_blocks), shifted(p.c.free_list), shifted(p.c.n_free), t)
        n = rng.integers(0, 300, (N, G, B)).astype(np.int32)
        nb, nf = shifted(p.c.n_blocks), shifted(p.c.n_free)
        p.c.block_tables(shifted(_gpu(n)), nb, nf)
        wnb, wnf, _ = p.f.update(n, commit=False)
        p.same((nb, wnb), (nf, wnf))
        p.update(n)
        cu, out = (shifted(torch.full(s, -7, dtype=d, device=DEV)) for s, d in (((N, G, B + 1), torch.int32), ((N, G, 1001), torch.int64)))
        p.c.slot_map(shifted(_gpu(n)), cu, out, n_new=shifted(_gpu(n)))
        for have, want in zip((cu, out), p.f.slots(n, 1001, n)):
            assert np.array_equal(have.cpu().numpy(), want)
        o = [shifted(torch.full(s, -7, dtype=torch.int32, device=DEV)) for s in ((N, G), (N, G, B), (N, G, B + 1), (N, G, P), (N, G, B))]
        p.c.page_lists(shifted(_gpu(n)), *o)
        for have, want in zip(o, p.f.pages(n)):
            assert np.array_equal(have.cpu().numpy(), want)


def test_lengths_written_by_the_kernel_ahead_and_other_streams():
    shape = N, G, B, t, P, T = 40, 16, 64, 16, 600, 20
    p = Pair(*shape, seed=21)
    rng = np.random.default_rng(3)
    base = rng.integers(0, 130, (N, G, B)).astype(np.int32)
    lens, src = torch.empty((N, G, B), dtype=torch.int32, device=DEV), _gpu(base)
    side = torch.cuda.Stream()
    out = torch.zeros((12, N, G, B), dtype=torch.int64, device=DEV)
    cu = torch.zeros((N, G, B + 1), dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for k in range(12):                                       # nothing waits for the host in between
            torch.add(src, k, out=lens)
            p.c.block_tables(lens)
            p.c.slot_map(lens, cu, out[k])
    side.synchronize()
    for k in range(12):
        p.f.update((base + k).astype(np.int32))
        assert np.array_equal(out[k].cpu().numpy(), p.f.slots((base + k).astype(np.int32), B, fill=0)[1]), k
    p.same()
    explicit = torch.cuda.Stream()
    p.update(base, stream=explicit)
    explicit.synchronize()


def test_captured_and_replayed():
    shape = N, G, B, t, P, T = 20, 16, 64, 16, 500, 30
    p = Pair(*shape, seed=31)
    rng = np.random.default_rng(6)
    base = rng.integers(0, 100, (N, G, B)).astype(np.int32)
    lens, step = _gpu(base), torch.zeros(N, dtype=torch.int32, device=DEV)
    z = dict(dtype=torch.int32, device=DEV)
    cu, out, short = torch.zeros((N, G, B + 1), **z), torch.zeros((N, G, B), dtype=torch.int64, device=DEV), torch.zeros((N, G), **z)
    o = [torch.full(s, -7, **z) for s in ((N, G), (N, G, B), (N, G, B + 1), (N, G, P), (N, G, B))]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step.add_(1)
        p.c.block_tables(lens, short_blocks=short, step=step)
        p.c.slot_map(lens, cu, out, step=step)
        p.c.page_lists(lens, *o, step=step)
    for k in range(1, 30):
        if k == 9:
            base = rng.integers(0, 100, (N, G, B)).astype(np.int32)
            lens.copy_(_gpu(base))
        graph.replay()
        host_step = np.full(N, k, np.int32)
        p.f.update(base, host_step)
        if k in (1, 9, 29):
            torch.cuda.synchronize()
            p.same()
            wcu, wout = p.f.slots(base, B, step=host_step, fill=0)
            running = np.arange(B) < wcu[..., -1:]
            assert np.array_equal(cu.cpu().numpy(), wcu) and np.array_equal(np.where(running, out.cpu().numpy(), 0), wout)
            want = p.f.pages(base, host_step)
            for have, w in zip((o[0], o[1], o[2], o[4]), (want[0], want[1], want[2], want[4])):
                assert np.array_equal(have.cpu().numpy(), w)
            used = np.arange(P) < want[2][..., -1:]
            assert np.array_equal(np.where(used, o[3].cpu().numpy(), -7), want[3])


@pytest.mark.parametrize("name,kw,n_inst,steps", [("c0", dict(hazard=0.05), 1, 40), ("c3", dict(hazard=0.1, G=5, init_active=40), 3, 25)])
def test_beside_the_routing_step(name, kw, n_inst, steps):
    """Route, bring the tables up to date, map the new tokens, list the pages, step after step on the router's own state; the
    free blocks then say which workers an F-score call may choose."""
    cfg = wlm.get_config(name, **kw)
    wl = wlm.make_workload(cfg, n_instances=n_inst)
    r = Router(wl, device=DEV)
    st, out = r.device_state(), r.outputs(n_inst)
    p = Pair(n_inst, cfg.G, cfg.B, 16, 2600, 2100, seed=41)
    p.c = r.block_cache(n_inst, 16, 2600, 2100)
    p.f.free_list[:] = np.arange(2599, -1, -1)
    p.c.table.fill_(-9)
    z = dict(dtype=torch.int32, device=DEV)
    f = p.f
    cu, slots = torch.zeros((n_inst, f.G, f.B + 1), **z), torch.zeros((n_inst, f.G, f.B), dtype=torch.int64, device=DEV)
    o = [torch.zeros(s, **z) for s in ((n_inst, f.G), (n_inst, f.G, f.B), (n_inst, f.G, f.B + 1), (n_inst, f.G, f.P), (n_inst, f.G, f.B))]
    for k in range(steps):
        r.step(st, out)
        p.c.block_tables(st["act_base"], step=st["step"])
        p.c.slot_map(st["act_base"], cu, slots, step=st["step"])
        p.c.page_lists(st["act_base"], *o, step=st["step"])
        base, step = st["act_base"].cpu().numpy(), st["step"].cpu().numpy()
        assert (step == k + 1).all()
        f.update(base, step)
        p.same()
        wcu, wout = f.slots(base, f.B, step=step, fill=0)
        live = np.arange(f.B) < wcu[..., -1:]
        assert np.array_equal(cu.cpu().numpy(), wcu) and np.array_equal(np.where(live, slots.cpu().numpy(), 0), wout)
        want = f.pages(base, step, fill=0)
        assert np.array_equal(o[0].cpu().numpy(), st["nact"].cpu().numpy())
        for j in (0, 1, 2, 4):
            assert np.array_equal(o[j].cpu().numpy(), want[j])
        used = np.arange(f.P) < want[2][..., -1:]
        assert np.array_equal(np.where(used, o[3].cpu().numpy(), 0), want[3])
    f.check_partition()
    p.c.n_free[:, 1] = 0                                          # a worker whose pool is used up takes no request
    s = torch.full((n_inst, 8), 100, **z)
    best = torch.zeros((n_inst, 8), **z)
    F = torch.zeros((n_inst, 8, f.G), dtype=torch.float64, device=DEV)
    load = torch.arange(f.G, dtype=torch.int64, device=DEV).flip(0).mul(1000).expand(n_inst, f.G).contiguous()
    load[:, 1] = -10 ** 6
    r.fscore(s, load, F, cap=p.c.n_free, best_g=best)
    assert not bool((best == 1).any())
    r.close()


def test_range_checked_build():
    """libbr_dbg.so counts indexes outside a row of the tables, lists and outputs: there are none, on teams of every size, with
    runs long and short, counts that cannot be, and rows of outputs that are too small."""
    from paper_2605_06113_b200 import binding, build
    binding.use_library(build.build_debug())
    try:
        hits = binding.lib().br_debug_bounds_hits()
        assert hits >= 0
        rng = np.random.default_rng(9)
        for shape in ((1, 1, 1, 1, 1, 1), (1, 4, 64, 16, 700, 90), (2, 3, 256, 16, 5000, 65), (1300, 8, 33, 5, 97, 40), (5, 1, 130, 7, 33, 6)):
            p = Pair(*shape, seed=13)
            n = np.zeros(p.f.n_blocks.shape, np.int64)
            for k in range(3):
                n = _walk(rng, p.f, n, 0.3, 0.7, 4)
                length = n.astype(np.int32)
                p.update(length, out=k == 1)
                p.slots(length, p.f.B)
                p.slots(length, 1 + 5 * k * p.f.B, rng.integers(0, 50, n.shape).astype(np.int32))
                p.pages(length)
            for value in (MOST, -5):
                p.f.n_blocks[0, 0, 0] = value
                p.c.n_blocks[0, 0, 0] = value
                p.update(length)
                p.slots(length, 9, np.full(n.shape, 3, np.int32))
                p.pages(length)
        assert binding.lib().br_debug_bounds_hits() == hits
    finally:
        binding.use_library(None)


@pytest.mark.parametrize("shape", [(7, 3, 20, 8, 80, 30), (500, 10, 8, 8, 40, 12)])
def test_rows_of_a_batch_updated_elsewhere_and_committed(shape):
    p = Pair(*shape, seed=19)
    f = p.f
    rng = np.random.default_rng(8)
    n = rng.integers(0, 60, (f.N, f.G, f.B)).astype(np.int32)
    p.update(n)
    for first, N in ((2, 3), (0, 1), (f.N - 1, 1), (4, f.N - 4)):
        n = (_walk(rng, f, n.astype(np.int64), 0.3, 0.6, 5)).astype(np.int32)
        spare = (p.c.n_blocks.clone(), p.c.n_free.clone())        # rows outside the update hold the cache's counts
        p.c.block_tables(_gpu(n), *spare, first=first, N=N)
        wnb, wnf, _ = f.update(n, first=first, N=N, commit=False)
        p.same((spare[0], wnb), (spare[1], wnf))
        p.same()                                                  # not taken yet
        p.c.commit(*spare)
        f.n_blocks, f.n_free = wnb, wnf
        p.same()
    rows = (torch.full_like(p.c.n_blocks, -77), torch.full_like(p.c.n_free, -77))
    p.c.block_tables(_gpu(n), *rows, first=1, N=2)
    for t in rows:                                                # rows outside the update are left as they were
        assert bool((t[:1] == -77).all()) and bool((t[3:] == -77).all()) and not bool((t[1:3] == -77).any())
    f.check_partition()


@pytest.mark.parametrize("N,G,end", [(2, 3, 255), (2, 3, 256), (2, 3, 257), (2, 3, 512), (600, 8, 256)])
def test_grants_that_end_at_a_window_with_requests_behind_them_unserved(N, G, end):
    """The last block granted is the last of a window of 256 (or beside it), and what follows asks for a block each, or for many:
    served from the free list, from blocks taken back, and from both."""
    B, T = 28, 700
    sizes = [end - 26, 1, 1, 3, 2, 1, 1, 2, 7, 8]                  # ten requests that take `end` blocks
    behind = [1, 1, 2, 1, 300, 1, 1, 40]                           # nothing is left for these
    after = np.array(sizes + [0] * 4 + behind + [0] * 6, np.int32)
    for before in ([0] * 28,                                       # all from the free list
                   [0] * 22 + [end - 9, 2, 3, 2, 1, 1],            # all of them taken back
                   [0] * 22 + [end - 130, 2, 3, 2, 1, 1],          # some of them
                   [0] * 10 + [end - 9, 2, 3, 2] + [0] * 8 + [1, 1] + [0] * 4):
        p = Pair(N, G, B, 1, end, T, seed=end)
        p.update(np.tile(np.array(before, np.int32), (N, G, 1)))
        n = np.tile(after, (N, G, 1))
        assert (p.update(n, out=True) == sum(behind)).all()
        assert (p.update(n) == sum(behind)).all() and not p.f.n_free.any()
        p.pages(n)
        n[:, :, 0] = 0                                             # and the others get what comes back
        p.update(n)
    p.f.check_partition()


def test_a_worker_without_free_blocks_is_not_chosen():
    """n_free as br_fscore's cap: the worker that the scores favour is chosen without it, the best of the others with it."""
    cfg = wlm.get_config("c0")
    r = Router(wlm.make_workload(cfg, n_instances=2), device=DEV)
    G = cfg.G
    c = r.block_cache(2, 16, 30, 40)
    z = dict(dtype=torch.int32, device=DEV)
    s = torch.tensor([[100, 700, 1, 5000]] * 2, **z)
    F = torch.full((2, 4, G), float("nan"), dtype=torch.float64, device=DEV)
    Lh = torch.randint(0, 10 ** 6, (2, G), dtype=torch.int64, device=DEV, generator=torch.Generator(DEV).manual_seed(3))
    length = torch.zeros((2, G, cfg.B), **z)
    best = torch.full((2, 4), -1, **z)
    r.fscore(s, Lh, F, cap=c.n_free, best_g=best)
    assert torch.equal(best.long(), F.argmax(-1)) and not bool(F.isnan().any())
    favoured = best.clone()
    for i, g in enumerate(best[:, 0].tolist()):
        length[i, g, 5] = 30 * 16                                 # one request takes the worker's whole pool
    c.block_tables(length)
    assert (c.n_free == 0).sum() == 2
    best.fill_(-1)
    r.fscore(s, Lh, F, best_g=best)
    assert torch.equal(best, favoured)
    best.fill_(-1)
    r.fscore(s, Lh, F, cap=c.n_free, best_g=best)
    assert torch.equal(best.long(), F.masked_fill((c.n_free == 0)[:, None, :], -float("inf")).argmax(-1))
    assert bool((best[:, 0] != favoured[:, 0]).all())
    r.close()
