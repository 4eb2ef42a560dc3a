"""The calls on block caches without a GPU: what the library and the binding refuse before anything is launched, and the
definitions that the GPU tests compare with on cases worked out by hand."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_06113_b200 import binding
from paper_2605_06113_b200.binding import BR_EINVAL, BR_OK, BlockCache, BrBlockCache, BrError, BrInstanceBatch

import cache_reference as ref

FAKE = 0x1000                        # never dereferenced: validation fails first, or no instance is in the batch


def _calls(batch, cache, length=FAKE, step=FAKE, a=FAKE, b=FAKE, c=FAKE, room=8):
    L = binding.lib()
    args = (C.byref(batch) if batch else None, C.byref(cache) if cache else None, length, step)
    return [L.br_block_tables(*args, a, b, c), L.br_slot_map(*args, c, room, a, b), L.br_page_lists(*args, a, b, c, a, b)]


def _cache(**kw):
    c = BrBlockCache(G=4, B=64, block_tokens=16, pool_blocks=100, table_blocks=10, table=FAKE, n_blocks=FAKE, free_list=FAKE,
                     n_free=FAKE)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_library_refuses_bad_arguments_without_touching_the_gpu():
    none = BrInstanceBatch(n_instances=0, first_instance=0, n_steps=1, stream=None)
    some = BrInstanceBatch(n_instances=2, first_instance=0, n_steps=1, stream=None)
    assert _calls(none, _cache()) == [BR_OK] * 3                                 # an empty batch is a no-op
    assert _calls(none, _cache(), step=None) == [BR_OK] * 3
    assert _calls(none, _cache(), c=None) == [BR_OK, BR_OK, BR_EINVAL]           # short_blocks and n_new may be NULL
    assert _calls(none, _cache(G=64, B=256, block_tokens=1 << 20, pool_blocks=1 << 28, table_blocks=1 << 22)) == [BR_OK] * 3
    assert _calls(None, _cache()) == _calls(some, None) == [BR_EINVAL] * 3
    for kw in (dict(length=None), dict(a=None), dict(b=None), dict(length=FAKE + 2), dict(step=FAKE + 1), dict(a=FAKE + 2),
               dict(b=FAKE + 2), dict(c=FAKE + 3)):
        assert _calls(some, _cache(), **kw) == [BR_EINVAL] * 3, kw
    for kw in (dict(G=0), dict(G=65), dict(B=0), dict(B=257), dict(block_tokens=0), dict(block_tokens=(1 << 20) + 1),
               dict(pool_blocks=0), dict(pool_blocks=(1 << 28) + 1), dict(table_blocks=0), dict(table_blocks=(1 << 22) + 1),
               dict(table=None), dict(n_blocks=None), dict(free_list=None), dict(n_free=None), dict(table=FAKE + 2),
               dict(n_blocks=FAKE + 1), dict(free_list=FAKE + 2), dict(n_free=FAKE + 2), dict(G=-1), dict(B=-8)):
        assert _calls(some, _cache(**kw)) == [BR_EINVAL] * 3, kw
        assert _calls(none, _cache(**kw)) == [BR_EINVAL] * 3, kw
    for n, first in ((-1, 0), (1, -1), (1 << 29, 0), (1, (1 << 29) - 1), ((1 << 31) - 1, (1 << 31) - 1)):
        b = BrInstanceBatch(n_instances=n, first_instance=first, n_steps=1, stream=None)
        assert _calls(b, _cache()) == [BR_EINVAL] * 3, (n, first)
    for room in (0, -1, (1 << 30) + 1):
        assert _calls(some, _cache(), room=room)[1] == BR_EINVAL
    assert _calls(some, _cache(), a=FAKE, b=FAKE + 4)[1] == BR_EINVAL            # slots are 64-bit


def _buffers(N, G, B, P, room=16):
    z = dict(dtype=torch.int32)
    return dict(cu=torch.zeros((N, G, B + 1), **z), slots=torch.zeros((N, G, room), dtype=torch.int64), n_seq=torch.zeros((N, G), **z),
                seq_slot=torch.zeros((N, G, B), **z), indptr=torch.zeros((N, G, B + 1), **z), indices=torch.zeros((N, G, P), **z),
                last_tokens=torch.zeros((N, G, B), **z))


def test_binding_refuses_tensors_of_another_type_shape_layout_or_device():
    N, G, B, T, P = 2, 3, 5, 7, 11
    z = dict(dtype=torch.int32)
    good = dict(table=torch.zeros((N, G, B, T), **z), n_blocks=torch.zeros((N, G, B), **z), free_list=torch.zeros((N, G, P), **z),
                n_free=torch.zeros((N, G), **z), block_tokens=16)
    for name, bad in (("table", torch.zeros((N, G, B, T), dtype=torch.int64)), ("table", torch.zeros((N, G, B), **z)),
                      ("table", torch.zeros((N, G, T, B), **z).transpose(2, 3)), ("n_blocks", torch.zeros((N, G, B + 1), **z)),
                      ("free_list", torch.zeros((N, G + 1, P), **z)), ("free_list", torch.zeros((N, G, P, 1), **z)),
                      ("n_free", torch.zeros((N, G), dtype=torch.float32)), ("n_free", torch.zeros((N, G), device="meta", **z))):
        with pytest.raises(ValueError):
            BlockCache(**{**good, name: bad})
    cache = BlockCache(**good)
    length, step, o = torch.zeros((N, G, B), **z), torch.zeros((N,), **z), _buffers(N, G, B, P)
    pages = (o["n_seq"], o["seq_slot"], o["indptr"], o["indices"], o["last_tokens"])
    strided = torch.zeros((N, G, 2 * B), **z)[:, :, ::2]
    for wrong in (length.long(), length[:1], strided, length.float()):
        with pytest.raises(ValueError):
            cache.block_tables(wrong, N=0)
        with pytest.raises(ValueError):
            cache.slot_map(wrong, o["cu"], o["slots"], N=0)
        with pytest.raises(ValueError):
            cache.page_lists(wrong, *pages, N=0)
        with pytest.raises(ValueError):
            cache.slot_map(length, o["cu"], o["slots"], n_new=wrong, N=0)
        with pytest.raises(ValueError):
            cache.block_tables(length, n_blocks_out=wrong, N=0)
    for call in (lambda **k: cache.block_tables(length, **k), lambda **k: cache.slot_map(length, o["cu"], o["slots"], **k),
                 lambda **k: cache.page_lists(length, *pages, **k)):
        for bad in (dict(step=torch.zeros((N + 1,), **z)), dict(step=step.long()), dict(N=N + 1), dict(N=-1), dict(first=-1),
                    dict(first=N, N=1), dict(first=N + 1)):
            with pytest.raises(ValueError):
                call(**bad)
        call(N=0)
        call(first=N)
        call(N=0, step=step, stream=C.c_void_p(0))
    for slots in (o["slots"].int(), o["slots"][:, :, ::2], o["slots"][:1], torch.zeros((N, G), dtype=torch.int64)):
        with pytest.raises(ValueError):
            cache.slot_map(length, o["cu"], slots, N=0)
    with pytest.raises(ValueError):
        cache.slot_map(length, o["seq_slot"], o["slots"], N=0)
    for k in range(5):
        with pytest.raises(ValueError):
            cache.page_lists(length, *[p if j != k else p.long() for j, p in enumerate(pages)], N=0)
    with pytest.raises(ValueError):
        cache.block_tables(length, short_blocks=torch.zeros((N, G, 1), **z), N=0)
    with pytest.raises(ValueError):
        cache.block_tables(length, n_free_out=torch.zeros((N, G), dtype=torch.int64), N=0)
    for call in (lambda **k: cache.block_tables(length, **k), lambda **k: cache.slot_map(length, o["cu"], o["slots"], **k),
                 lambda **k: cache.page_lists(length, *pages, **k)):
        with pytest.raises(ValueError, match="on a GPU"):                        # host memory never reaches a kernel
            call()
        with pytest.raises(ValueError, match="on a GPU"):
            call(N=1, first=1, stream=0)
    with pytest.raises(ValueError, match="at most"):
        cache.slot_map(length, o["cu"], torch.empty((N, G, 2 ** 32 + 5), dtype=torch.int64, device="meta"), N=0)
    with pytest.raises(ValueError):
        BlockCache(**{**good, "block_tokens": 2 ** 31})
    with pytest.raises(BrError):                                                 # no room for a single token
        cache.slot_map(length, o["cu"], torch.zeros((N, G, 0), dtype=torch.int64), N=0)
    with pytest.raises(BrError):
        BlockCache(**{**good, "block_tokens": 0}).block_tables(length, N=0)
    BlockCache.empty(0, G, B, 16, P, T, device="cpu").block_tables(torch.zeros((0, G, B), **z))


def test_counts_are_taken_by_commit_and_not_by_assignment():
    c = BlockCache.empty(2, 3, 4, 16, 5, 6, device="cpu")
    nb, nf = torch.ones_like(c.n_blocks), torch.ones_like(c.n_free)
    for name in ("table", "n_blocks", "free_list", "n_free"):
        with pytest.raises(AttributeError):
            setattr(c, name, nb)
    before = c._packed
    for bad in ((nb.long(), nf), (nb, nf[:1]), (nf, nb)):
        with pytest.raises(ValueError):
            c.commit(*bad)
    assert c._packed == before
    c.commit(nb, nf)
    assert c.n_blocks is nb and c.n_free is nf and c._packed != before


def test_new_cache_gives_out_blocks_from_zero():
    c = BlockCache.empty(2, 3, 4, 16, 5, 6, device="cpu")
    assert c.free_list.tolist() == [[[4, 3, 2, 1, 0]] * 3] * 2 and c.n_free.tolist() == [[5] * 3] * 2
    assert int(c.n_blocks.sum()) == 0


def test_definition_on_a_worker_worked_out_by_hand():
    # blocks of 4 tokens, a pool of 8: requests of 9, 0, 3 and 4 tokens
    f = ref.Fleets(1, 1, 4, t=4, P=8, T=4)
    L = np.array([[[9, ref.EMPTY, 3, 4]]], np.int32)
    _, _, short = f.update(L)
    assert f.table[0, 0].tolist() == [[0, 1, 2, -9], [-9] * 4, [3, -9, -9, -9], [4, -9, -9, -9]]
    assert f.n_blocks[0, 0].tolist() == [3, 0, 1, 1] and f.n_free[0, 0] == 3 and short[0, 0] == 0
    cu, out = f.slots(L, 5, n_new=np.array([[[2, 5, 0, 9]]], np.int32))
    assert cu[0, 0].tolist() == [0, 2, 2, 2, 6] and out[0, 0].tolist() == [7, 8, 16, 17, 18]     # the last one has no room
    n, slot, indptr, indices, last = f.pages(L)
    assert n[0, 0] == 3 and slot[0, 0].tolist() == [0, 2, 3, -1] and indptr[0, 0].tolist() == [0, 3, 4, 5, 5]
    assert indices[0, 0].tolist() == [0, 1, 2, 3, 4, -7, -7, -7] and last[0, 0].tolist() == [1, 3, 4, 0]
    # the first shrinks to 4 tokens, the second grows to 13: blocks 1, 2 are taken back, then 5 and 6 come off the list
    M = np.array([[[4, 13, 3, ref.EMPTY]]], np.int32)
    f.update(M)
    assert f.n_blocks[0, 0].tolist() == [1, 4, 1, 0] and f.table[0, 0, 1].tolist() == [1, 2, 4, 5]
    assert f.n_free[0, 0] == 2 and f.free_list[0, 0].tolist()[:2] == [7, 6]
    # 17 tokens pass the row of four columns, 9 are too many for the two blocks left, so 8 behind them wait too
    short = f.update(np.array([[[17, 13, 15, 8]]], np.int32))[2]
    assert short[0, 0] == 4 + 3 + 2 and f.n_blocks[0, 0].tolist() == [1, 4, 1, 0]
    f.update(L)
    assert f.n_blocks[0, 0].tolist() == [3, 0, 1, 1] and f.table[0, 0, 0].tolist()[:3] == [0, 1, 2]
    f.check_partition()


def test_definition_undoes_what_it_did():
    rng = np.random.default_rng(5)
    f = ref.Fleets(1, 1, 9, t=5, P=60, T=12)
    f.update(rng.integers(0, 30, (1, 1, 9)).astype(np.int32))
    for _ in range(50):
        A = rng.integers(0, 30, (1, 1, 9)).astype(np.int32)
        f.update(A)
        before = (f.n_blocks.copy(), f.n_free.copy(), [f.table[0, 0, b, :n].tolist() for b, n in enumerate(f.n_blocks[0, 0])],
                  f.free_list[0, 0, :f.n_free[0, 0]].tolist())
        if f.update(rng.integers(0, 30, (1, 1, 9)).astype(np.int32))[2][0, 0]:
            continue
        f.update(A)
        assert np.array_equal(f.n_blocks, before[0]) and np.array_equal(f.n_free, before[1])
        assert [f.table[0, 0, b, :n].tolist() for b, n in enumerate(f.n_blocks[0, 0])] == before[2]
        assert f.free_list[0, 0, :f.n_free[0, 0]].tolist() == before[3]
    f.check_partition()


def test_count_outputs_go_together():
    """Counts in place for one array and elsewhere for the other would leave a cache whose n_blocks and n_free disagree."""
    some = BrInstanceBatch(n_instances=0, first_instance=0, n_steps=1, stream=None)
    c = _cache(n_blocks=FAKE, n_free=2 * FAKE)
    L = binding.lib()
    for nb, nf, want in ((FAKE, 2 * FAKE, BR_OK), (3 * FAKE, 4 * FAKE, BR_OK), (FAKE, 4 * FAKE, BR_EINVAL), (3 * FAKE, 2 * FAKE, BR_EINVAL)):
        assert L.br_block_tables(C.byref(some), C.byref(c), FAKE, None, nb, nf, None) == want, (nb, nf)
    cache = BlockCache.empty(2, 3, 4, 16, 5, 6, device="cpu")
    length, nb, nf = torch.zeros_like(cache.n_blocks), torch.empty_like(cache.n_blocks), torch.empty_like(cache.n_free)
    for mixed in (dict(n_blocks_out=nb), dict(n_free_out=nf), dict(n_blocks_out=cache.n_blocks, n_free_out=nf),
                  dict(n_blocks_out=nb, n_free_out=cache.n_free)):
        with pytest.raises(ValueError, match="go together"):
            cache.block_tables(length, N=0, **mixed)
    for both in (dict(), dict(n_blocks_out=nb, n_free_out=nf), dict(n_blocks_out=cache.n_blocks, n_free_out=cache.n_free),
                 dict(n_blocks_out=cache.n_blocks), dict(n_free_out=cache.n_free)):
        cache.block_tables(length, N=0, **both)


def test_definition_with_one_of_the_counts_in_place_deals_blocks_out_twice():
    """Why they go together: with entries kept out of use nothing notices, and two requests share blocks."""
    f = ref.Fleets(1, 1, 2, t=1, P=10, T=4)
    f.n_free[:] = 4                                                              # blocks 9 to 6; the others are out of use
    f.n_blocks = f.update(np.array([[[2, 0]]], np.int32), commit=False)[0]       # (beside the old n_free)
    assert f.update(np.array([[[2, 2]]], np.int32))[2][0, 0] == 0
    assert f.table[0, 0, 0].tolist()[:2] == f.table[0, 0, 1].tolist()[:2] == [6, 7]


def test_calls_use_the_memory_that_the_tensors_have_now(monkeypatch):
    """A tensor of the cache may be given other memory after the handle was made (resized, reloaded, moved into a pool)."""
    N, G, B, T, P = 2, 3, 4, 6, 5
    cache = BlockCache.empty(N, G, B, 16, P, T, device="cpu")
    length, o = torch.zeros_like(cache.n_blocks), _buffers(N, G, B, P)
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda batch, packed, *args: seen.append(BrBlockCache.from_buffer_copy(packed)) or BR_OK

    monkeypatch.setattr(binding, "_lib", Library())
    calls = (lambda: cache.block_tables(length, N=0), lambda: cache.slot_map(length, o["cu"], o["slots"], N=0),
             lambda: cache.page_lists(length, o["n_seq"], o["seq_slot"], o["indptr"], o["indices"], o["last_tokens"], N=0))
    names = ("table", "n_blocks", "free_list", "n_free")
    for name in names:
        held = getattr(cache, name)
        for change in (lambda: held.set_(held.clone()), lambda: setattr(held, "data", held.data.clone())):
            old = held.data_ptr()
            keep = held.untyped_storage()                                        # (so that the new memory is elsewhere)
            change()
            assert held.data_ptr() != old and keep.data_ptr() == old
            for call in calls:
                call()
                assert [getattr(seen[-1], n) for n in names] == [getattr(cache, n).data_ptr() for n in names], name
                assert (seen[-1].G, seen[-1].B, seen[-1].block_tokens, seen[-1].pool_blocks, seen[-1].table_blocks) == (G, B, 16, P, T)
    count = len(seen)
    cache.free_list.data = torch.zeros((N, G, P - 1), dtype=torch.int32)
    for call in calls:
        with pytest.raises(ValueError, match="free_list"):
            call()
    assert len(seen) == count


def test_block_size_is_a_whole_number():
    c = BlockCache.empty(2, 3, 4, 16, 5, 6, device="cpu")
    arrays = (c.table, c.n_blocks, c.free_list, c.n_free)
    for t in (16.5, 0.99, float("nan"), float("inf"), "16", None):
        with pytest.raises(ValueError, match="block_tokens"):
            BlockCache(*arrays, t)
    for t in (16, 16.0, np.int64(16), torch.tensor(16)):
        assert BlockCache(*arrays, t).block_tokens == 16


def test_commit_takes_both_counts_or_none():
    cache = BlockCache.empty(2, 3, 4, 16, 5, 6, device="cpu")
    nb, nf = torch.zeros_like(cache.n_blocks), torch.zeros_like(cache.n_free)
    own, before = (cache.n_blocks, cache.n_free), cache._packed
    for mixed in ((nb, own[1]), (own[0], nf)):
        with pytest.raises(ValueError, match="go together"):
            cache.commit(*mixed)
    assert cache._packed == before and cache.n_blocks is own[0] and cache.n_free is own[1]
    cache.commit(*own)                                                           # what it has already
    assert cache._packed == before
    cache.commit(nb, nf)
    assert cache.n_blocks is nb and cache.n_free is nf
