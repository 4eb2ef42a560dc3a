"""What the calls on block caches compute, request by request in Python integers, written from their definitions."""
import numpy as np

EMPTY = -(2 ** 31)
MOST = 2 ** 31 - 1


def tokens_of(length, step):
    """Tokens of one worker's requests: length + step, 0 for a free slot, at most 2^31 - 1."""
    return [0 if int(v) == EMPTY else min(MOST, max(0, int(v) + step)) for v in length]


def block_tables(tokens, t, table, n_blocks, free_list, n_free):
    """One worker, in place on table [B, T] and free_list [P]; returns the new counts and the blocks still lacking."""
    B, T = table.shape
    P = free_list.shape[0]
    held = [int(v) for v in n_blocks]
    if not 0 <= n_free <= P or any(not 0 <= h <= T for h in held) or sum(held) + n_free > P:
        return held, n_free, -1
    free = [int(v) for v in free_list[:n_free]]
    need = [-(-n // t) for n in tokens]
    taken = []
    for b in range(B):
        if need[b] < held[b]:
            taken += [int(v) for v in table[b, need[b]:held[b]]]
            held[b] = need[b]
    stock, lacking, stuck = len(taken) + len(free), 0, False
    for b in range(B):
        more = need[b] - held[b]
        if more <= 0:
            continue
        if need[b] > T:
            lacking += more
            continue
        stuck = stuck or more > stock
        if stuck:
            lacking += more
            continue
        for c in range(held[b], need[b]):
            table[b, c] = taken.pop(0) if taken else free.pop()
        stock -= more
        held[b] = need[b]
    while taken:
        free.append(taken.pop())
    if len(free) > n_free:
        free_list[n_free:len(free)] = free[n_free:]
    return held, len(free), min(MOST, lacking)


def slot_map(tokens, n_new, t, table, n_blocks, out):
    """One worker: writes out [room] and returns the prefix sums."""
    cu = [0]
    for b, n in enumerate(tokens):
        q = int(n > 0) if n_new is None else min(max(int(n_new[b]), 0), n)
        for p in range(n - q, n)[:max(0, len(out) - cu[-1])]:
            held = min(max(int(n_blocks[b]), 0), table.shape[1])
            out[cu[-1] + p - (n - q)] = int(table[b, p // t]) * t + p % t if p // t < held else -1
        cu.append(cu[-1] + q)
    return [min(MOST, v) for v in cu]


def page_lists(tokens, t, table, n_blocks, indices):
    """One worker: writes indices [P] and returns (n_seq, seq_slot, indptr, last_tokens)."""
    B = len(tokens)
    slot, indptr, last = [], [0], []
    for b, n in enumerate(tokens):
        if n == 0:
            continue
        need, held = -(-n // t), min(max(int(n_blocks[b]), 0), table.shape[1])
        k = min(need, held)
        for c in range(k):
            if indptr[-1] + c < len(indices):
                indices[indptr[-1] + c] = table[b, c]
        slot.append(b)
        indptr.append(indptr[-1] + k)
        last.append(0 if k == 0 else t if need > held else n - (need - 1) * t)
    m = len(slot)
    return m, slot + [-1] * (B - m), indptr + [indptr[-1]] * (B - m), last + [0] * (B - m)


class Fleets:
    """The host copy of a cache, updated by the definitions."""

    def __init__(self, N, G, B, t, P, T, fill=-9):
        self.N, self.G, self.B, self.t, self.P, self.T = N, G, B, t, P, T
        self.table = np.full((N, G, B, T), fill, np.int32)
        self.n_blocks = np.zeros((N, G, B), np.int32)
        self.free_list = np.tile(np.arange(P - 1, -1, -1, dtype=np.int32), (N, G, 1))
        self.n_free = np.full((N, G), P, np.int32)

    def workers(self, first=0, N=None):
        return [(i, g) for i in range(first, self.N if N is None else first + N) for g in range(self.G)]

    def _tokens(self, length, step, at):
        return tokens_of(length[at], 0 if step is None else int(step[at[0]]))

    def update(self, length, step=None, first=0, N=None, commit=True):
        """Returns (n_blocks, n_free, short_blocks) after the update; keeps the counts if `commit`."""
        nb, nf = self.n_blocks.copy(), self.n_free.copy()
        short = np.full((self.N, self.G), -77, np.int32)
        for at in self.workers(first, N):
            nb[at], nf[at], short[at] = block_tables(self._tokens(length, step, at), self.t, self.table[at], self.n_blocks[at],
                                                     self.free_list[at], int(self.n_free[at]))
        if commit:
            self.n_blocks, self.n_free = nb, nf
        return nb, nf, short

    def slots(self, length, room, n_new=None, step=None, first=0, N=None, fill=-7):
        out = np.full((self.N, self.G, room), fill, np.int64)
        cu = np.full((self.N, self.G, self.B + 1), fill, np.int32)
        for at in self.workers(first, N):
            cu[at] = slot_map(self._tokens(length, step, at), None if n_new is None else n_new[at], self.t, self.table[at],
                              self.n_blocks[at], out[at])
        return cu, out

    def pages(self, length, step=None, first=0, N=None, fill=-7):
        n_seq = np.full((self.N, self.G), fill, np.int32)
        slot, last = (np.full((self.N, self.G, self.B), fill, np.int32) for _ in range(2))
        indptr = np.full((self.N, self.G, self.B + 1), fill, np.int32)
        indices = np.full((self.N, self.G, self.P), fill, np.int32)
        for at in self.workers(first, N):
            n_seq[at], slot[at], indptr[at], last[at] = page_lists(self._tokens(length, step, at), self.t, self.table[at],
                                                                   self.n_blocks[at], indices[at])
        return n_seq, slot, indptr, indices, last

    def check_partition(self):
        """Every block of every worker is held once or free once."""
        for at in self.workers():
            held = [int(v) for b in range(self.B) for v in self.table[at][b, :self.n_blocks[at][b]]]
            assert sorted(held + [int(v) for v in self.free_list[at][:self.n_free[at]]]) == list(range(self.P)), at
