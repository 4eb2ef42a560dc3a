"""Thin ctypes binding of libbr.so: the same calls as include/br.h, argument
marshalling only.  Device memory and streams come from PyTorch; every step of the
routing path runs inside the library's CUDA kernels.  There is no fallback: if the
library is missing or a call fails, an exception is raised."""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbr.so")

BR_OK, BR_EINVAL, BR_ERANGE, BR_ECUDA, BR_ENOMEM, BR_ESTATE, BR_ELIMIT = 0, -1, -2, -3, -4, -5, -6
STATIC_STAGE_BYTES = 8 << 20
MAX_SLOT_ROOM = 1 << 30
ST_QUEUE_OVERFLOW, ST_ITER_CAP, ST_BAD_STATE = 1, 2, 4
EMPTY = -(2 ** 31)


class BrParams(C.Structure):
    _fields_ = [
        ("B", C.c_int32), ("W", C.c_int32), ("R_max", C.c_int32), ("S_greedy", C.c_int32),
        ("alpha", C.c_double), ("beta", C.c_double), ("gamma", C.c_double),
        ("delta_T", C.c_int32), ("gate", C.c_float), ("c_floor", C.c_float),
        ("score_mode", C.c_int32), ("term_mode", C.c_int32), ("term_cdf", C.c_void_p),
        ("arr_cdf", C.c_void_p), ("arr_len", C.c_int32), ("arr_period", C.c_int32),
        ("arr_inst_stride", C.c_int32),
        ("len_tab", C.c_void_p), ("len_tab_log2", C.c_int32),
        ("burst_every", C.c_int32), ("burst_size", C.c_int32),
        ("s_max", C.c_int32), ("threads", C.c_int32), ("inst_per_block", C.c_int32),
        ("pred_mode", C.c_int32), ("out_tab", C.c_void_p), ("out_tab_log2", C.c_int32),
    ]


class BrWorkerState(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("load", "nact", "occ", "act_base", "act_id", "act_chat0", "act_kref", "act_end",
                 "step", "seed", "next_id")]


class BrWaitingQueue(C.Structure):
    _fields_ = [("s", C.c_void_p), ("id", C.c_void_p), ("n", C.c_void_p), ("o", C.c_void_p)]


class BrInstanceBatch(C.Structure):
    _fields_ = [("n_instances", C.c_int32), ("first_instance", C.c_int32),
                ("n_steps", C.c_int32), ("stream", C.c_void_p)]


class BrBlockCache(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("G", "B", "block_tokens", "pool_blocks", "table_blocks")] + \
               [(n, C.c_void_p) for n in ("table", "n_blocks", "free_list", "n_free")]


class BrLoadOut(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("load", "trace", "status", "counters", "fscore",
                                          "phase_cycles")]


EXPORTS = ["br_create", "br_step", "br_graph_capture", "br_graph_step", "br_step_host",
           "br_step_host_static", "br_debug_bounds_hits", "br_debug_bounds_selftest", "br_debug_step_registers",
           "br_fscore", "br_best_subset", "br_bypass_dispatch", "br_survival_chat", "br_block_tables",
           "br_slot_map", "br_page_lists", "br_destroy", "br_strerror", "br_version"]

_lib = None


class BrError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        msg = lib().br_strerror(status).decode()
        super().__init__(f"{where}: status {status} ({msg})")


def lib():
    """Loads libbr.so.  Raises if it has not been built (python -m paper_2605_06113_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: build the CUDA library first "
                               "(python paper_2605_06113_b200/build.py)")
        L = C.CDLL(LIB_PATH)
        step_args = [C.c_void_p] * 7       # structures go by address: byref() of one, or its packed bytes
        L.br_create.argtypes = [C.c_int32, C.c_int32, C.POINTER(BrParams), C.POINTER(C.c_void_p)]
        L.br_step.argtypes = step_args
        L.br_graph_capture.argtypes = step_args
        L.br_graph_step.argtypes = [C.c_void_p]
        L.br_step_host.argtypes = step_args + [C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.br_step_host_static.argtypes = step_args + [C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.br_fscore.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.br_best_subset.argtypes = [C.c_void_p, C.POINTER(BrInstanceBatch), C.c_void_p, C.c_int32,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.br_bypass_dispatch.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                         C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.br_survival_chat.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                       C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
        L.br_block_tables.argtypes = [C.c_void_p] * 7
        L.br_slot_map.argtypes = [C.c_void_p] * 5 + [C.c_int32] + [C.c_void_p] * 2
        L.br_page_lists.argtypes = [C.c_void_p] * 9
        L.br_debug_bounds_hits.argtypes = []
        L.br_debug_bounds_selftest.argtypes = [C.c_void_p]
        L.br_debug_step_registers.argtypes = [C.c_int32] * 5 + [C.POINTER(C.c_int32)]
        L.br_destroy.argtypes = [C.c_void_p]
        L.br_strerror.restype = C.c_char_p
        L.br_strerror.argtypes = [C.c_int]
        for n in EXPORTS:
            if n != "br_strerror":
                getattr(L, n).restype = C.c_int
        _lib = L
    return _lib


def use_library(path: Optional[str] = None) -> None:
    """Makes lib() load another build of the library (the range-checked libbr_dbg.so); None goes
    back to libbr.so.  Contexts created earlier keep the library they were created with only as
    long as the caller keeps using them through it: close them first."""
    global _lib, LIB_PATH
    _lib = None
    LIB_PATH = os.path.join(_HERE, "libbr.so") if path is None else path


# The same structures as packed bytes, which the library only reads: filling ctypes fields by name takes
# longer than the rest of an eager one-instance step.
_pack_batch = struct.Struct("@iiiP").pack
_pack_state = struct.Struct("@11P").pack
_pack_queue = struct.Struct("@4P").pack
_pack_out = struct.Struct("@6P").pack
_pack_cache = struct.Struct("@5i4x4P").pack


def _addr(t) -> int:
    return 0 if t is None else t.data_ptr() if not isinstance(t, np.ndarray) else t.ctypes.data


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        return t.ctypes.data
    return t.data_ptr()


def _to_torch(a: np.ndarray, device):
    """numpy -> torch on `device`, keeping the bit pattern of unsigned types."""
    import torch
    if a.dtype == np.uint64:
        return torch.from_numpy(a.view(np.int64).copy()).to(device)
    if a.dtype == np.uint32:
        return torch.from_numpy(a.view(np.int32).copy()).to(device)
    return torch.from_numpy(np.ascontiguousarray(a)).to(device)


_STATE_DTYPES = dict(load=np.int64, nact=np.int32, occ=np.uint64, act_base=np.int32,
                     act_id=np.uint32, act_chat0=np.float32, act_kref=np.uint8, step=np.int32,
                     seed=np.uint64, next_id=np.uint32, wq_s=np.int32, wq_id=np.uint32, wq_n=np.int32,
                     act_end=np.int32, wq_o=np.int32)


class Router:
    """br_create / br_step / br_destroy for one fleet shape, fed from a generated workload."""

    def __init__(self, wl, device="cuda:0", threads: int = 0, **overrides):
        import torch
        self.torch = torch
        self.wl = wl
        cfg = wl.cfg
        self.cfg = cfg
        self.device = torch.device(device)
        self._data_ptr, self._null = torch.Tensor.data_ptr, torch.empty(0)      # the empty tensor's address is NULL
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.len_tab = _to_torch(wl.len_tab, self.device)
        self.arr_cdf = _to_torch(wl.arr_cdf, self.device)
        self.term_cdf = _to_torch(wl.term_cdf, self.device)
        self.out_tab = _to_torch(wl.out_tab, self.device) if wl.out_tab is not None else None
        p = BrParams(
            B=cfg.B, W=cfg.W, R_max=cfg.R_max, S_greedy=cfg.S_greedy, alpha=cfg.alpha,
            beta=cfg.beta, gamma=cfg.gamma, delta_T=cfg.delta_T, gate=cfg.gate, c_floor=cfg.c_floor,
            score_mode=cfg.score_mode, term_mode=cfg.term_mode, term_cdf=self.term_cdf.data_ptr(),
            arr_cdf=self.arr_cdf.data_ptr(), arr_len=wl.arr_cdf.shape[1], arr_period=wl.arr_period,
            arr_inst_stride=wl.arr_inst_stride, len_tab=self.len_tab.data_ptr(),
            len_tab_log2=int(wl.len_tab.size).bit_length() - 1, burst_every=cfg.burst_every,
            burst_size=cfg.burst_size, s_max=int(max(cfg.len_clip[1], cfg.ctx_clip[1])),
            threads=threads, pred_mode=cfg.pred_mode,
            out_tab=self.out_tab.data_ptr() if self.out_tab is not None else None,
            out_tab_log2=int(wl.out_tab.size).bit_length() - 1 if wl.out_tab is not None else 0)
        for k, v in overrides.items():
            setattr(p, k, v)
        self.params = p
        h = C.c_void_p()
        rc = lib().br_create(cfg.G, cfg.H, C.byref(p), C.byref(h))
        if rc != BR_OK:
            raise BrError(rc, "br_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            lib().br_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- buffers -----------------------------------------------------------
    def device_state(self, state: Optional[Dict[str, np.ndarray]] = None) -> Dict[str, "object"]:
        st = self.wl.state if state is None else state
        return {k: _to_torch(np.ascontiguousarray(v, dtype=_STATE_DTYPES[k]), self.device)
                for k, v in st.items()}

    def outputs(self, N: int, n_steps: int = 1, fscore: bool = False, device=None):
        t = self.torch
        dev = self.device if device is None else device
        cfg = self.cfg
        o = dict(
            assign=t.empty((n_steps, N, cfg.W), dtype=t.int32, device=dev),
            load=t.empty((n_steps, N, cfg.G), dtype=t.int64, device=dev),
            trace=t.empty((n_steps, N, 3), dtype=t.int64, device=dev),
            status=t.zeros((n_steps, N), dtype=t.int32, device=dev),
            counters=t.zeros((n_steps, N, 4), dtype=t.int32, device=dev),
        )
        if fscore:
            o["fscore"] = t.zeros((n_steps, N, cfg.W, cfg.G), dtype=t.float64, device=dev)
        return o

    def _structs(self, st, out, N, first, n_steps, stream):
        ws = BrWorkerState(**{k: _ptr(st.get(k)) for k in
                              ("load", "nact", "occ", "act_base", "act_id", "act_chat0", "act_kref", "act_end",
                               "step", "seed", "next_id")})
        wq = BrWaitingQueue(s=_ptr(st["wq_s"]), id=_ptr(st["wq_id"]), n=_ptr(st["wq_n"]), o=_ptr(st.get("wq_o")))
        lo = BrLoadOut(load=_ptr(out["load"]), trace=_ptr(out["trace"]), status=_ptr(out.get("status")),
                       counters=_ptr(out.get("counters")), fscore=_ptr(out.get("fscore")),
                       phase_cycles=_ptr(out.get("phase_cycles")))
        b = BrInstanceBatch(n_instances=N, first_instance=first, n_steps=n_steps, stream=stream)
        return b, ws, wq, lo

    def _stream(self, stream):
        if stream is None:
            if self._raw_stream is not None and self.device.index is not None:
                return self._raw_stream(self.device.index)        # without building a stream object
            return self.torch.cuda.current_stream(self.device).cuda_stream
        if isinstance(stream, C.c_void_p):
            return stream.value
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream

    def block_cache(self, N: int, block_tokens: int, pool_blocks: int, table_blocks: int) -> "BlockCache":
        """A new paged cache for the workers of N fleets of this shape."""
        return BlockCache.empty(N, self.cfg.G, self.cfg.B, block_tokens, pool_blocks, table_blocks, device=self.device)

    # ---- the calls of include/br.h -------------------------------------------
    def step(self, st, out, term_probs=None, N=None, first=0, n_steps=1, stream=None):
        if N is None:
            N = st["step"].shape[0] - first
        sget, oget, null = st.get, out.get, self._null
        arrays = (sget("load", null), sget("nact", null), sget("occ", null), sget("act_base", null),
                  sget("act_id", null), sget("act_chat0", null), sget("act_kref", null), sget("act_end", null),
                  sget("step", null), sget("seed", null), sget("next_id", null),
                  st["wq_s"], st["wq_id"], st["wq_n"], sget("wq_o", null),
                  null if term_probs is None else term_probs, out["assign"],
                  out["load"], out["trace"], oget("status", null), oget("counters", null),
                  oget("fscore", null), oget("phase_cycles", null))
        try:
            a = list(map(self._data_ptr, arrays))
        except TypeError:                      # a None or a numpy array among them
            a = list(map(_addr, arrays))
        rc = lib().br_step(self._h, _pack_batch(N, first, n_steps, self._stream(stream) or 0), _pack_state(*a[:11]),
                           _pack_queue(*a[11:15]), a[15], a[16], _pack_out(*a[17:]))
        if rc != BR_OK:
            raise BrError(rc, "br_step")

    def prepare(self, st, out, term_probs=None, N=None, first=0, n_steps=1, stream=None):
        """Marshals the arguments of br_step once; the returned callable repeats the same call
        (same buffers, same stream) without rebuilding the argument structures."""
        N = st["step"].shape[0] - first if N is None else N
        b, ws, wq, lo = self._structs(st, out, N, first, n_steps, self._stream(stream))
        fn, h = lib().br_step, self._h
        args = (h, C.byref(b), C.byref(ws), C.byref(wq), _ptr(term_probs), _ptr(out["assign"]), C.byref(lo))
        keep = (b, ws, wq, lo, st, out, term_probs)

        def call(_fn=fn, _args=args, _keep=keep):
            rc = _fn(*_args)
            if rc != BR_OK:
                raise BrError(rc, "br_step")
        return call

    def graph_capture(self, st, out, term_probs=None, N=None, first=0, n_steps=1, stream=None):
        N = st["step"].shape[0] - first if N is None else N
        b, ws, wq, lo = self._structs(st, out, N, first, n_steps, self._stream(stream))
        rc = lib().br_graph_capture(self._h, C.byref(b), C.byref(ws), C.byref(wq), _ptr(term_probs),
                                    _ptr(out["assign"]), C.byref(lo))
        if rc != BR_OK:
            raise BrError(rc, "br_graph_capture")

    def graph_step(self):
        rc = lib().br_graph_step(self._h)
        if rc != BR_OK:
            raise BrError(rc, "br_graph_step")

    def step_host(self, st, out, term_probs=None, N=None, stream=None):
        """st / out / term_probs are host tensors or numpy arrays (pinned for async copies)."""
        N = st["step"].shape[0] if N is None else N
        b, ws, wq, lo = self._structs(st, out, N, 0, 1, self._stream(stream))
        up, down = C.c_int64(), C.c_int64()
        rc = lib().br_step_host(self._h, C.byref(b), C.byref(ws), C.byref(wq), _ptr(term_probs),
                                _ptr(out["assign"]), C.byref(lo), C.byref(up), C.byref(down))
        if rc != BR_OK:
            raise BrError(rc, "br_step_host")
        return up.value, down.value

    def step_host_static(self, st, out, term_probs=None, N=None, stream=None):
        """br_step_host_static: like step_host, but the device staging is the library's built-in
        array, so nothing is allocated; raises BrError(BR_ELIMIT) if the batch does not fit."""
        N = st["step"].shape[0] if N is None else N
        b, ws, wq, lo = self._structs(st, out, N, 0, 1, self._stream(stream))
        up, down = C.c_int64(), C.c_int64()
        rc = lib().br_step_host_static(self._h, C.byref(b), C.byref(ws), C.byref(wq), _ptr(term_probs),
                                       _ptr(out["assign"]), C.byref(lo), C.byref(up), C.byref(down))
        if rc != BR_OK:
            raise BrError(rc, "br_step_host_static")
        return up.value, down.value

    def fscore(self, s, Lh, F, cap=None, best_g=None, N=None, first=0, stream=None):
        n, n_req = s.shape[:2]                         # (trailing dimensions of one are fine)
        b = _pack_batch(n - first if N is None else N, first, 1, self._stream(stream) or 0)
        rc = lib().br_fscore(self._h, b, _addr(s), n_req, _addr(Lh), _addr(cap), _addr(F), _addr(best_g))
        if rc != BR_OK:
            raise BrError(rc, "br_fscore")


    def bypass_dispatch(self, s, virtual_load, inflight, inflight_cap, worker_out, N=None, first=0, stream=None):
        n, n_req = s.shape[:2]                         # (trailing dimensions of one are fine)
        b = _pack_batch(n - first if N is None else N, first, 1, self._stream(stream) or 0)
        rc = lib().br_bypass_dispatch(self._h, b, _addr(s), n_req, _addr(virtual_load), _addr(inflight),
                                      _addr(inflight_cap), _addr(worker_out))
        if rc != BR_OK:
            raise BrError(rc, "br_bypass_dispatch")

    def survival_chat(self, hist_sorted, hist_prefix, age, c_hat, p_fin=None, mu_rem=None, stream=None):
        rc = lib().br_survival_chat(self._h, self._stream(stream), _ptr(hist_sorted), _ptr(hist_prefix),
                                    int(hist_sorted.numel()), _ptr(age), int(age.numel()), _ptr(c_hat),
                                    _ptr(p_fin), _ptr(mu_rem))
        if rc != BR_OK:
            raise BrError(rc, "br_survival_chat")

    def best_subset(self, win, margins, lim, best_mask, best_F=None, N=None, first=0, stream=None):
        N = win.shape[0] - first if N is None else N
        b = BrInstanceBatch(n_instances=N, first_instance=first, n_steps=1, stream=self._stream(stream))
        rc = lib().br_best_subset(self._h, C.byref(b), _ptr(win), int(win.shape[1]), _ptr(margins), _ptr(lim),
                                  _ptr(best_mask), _ptr(best_F))
        if rc != BR_OK:
            raise BrError(rc, "br_best_subset")


class BlockCache:
    """The paged caches of a batch of fleets (br_block_tables / br_slot_map / br_page_lists).

    ``table`` [N, G, B, columns], ``n_blocks`` [N, G, B], ``free_list`` [N, G, pool] and ``n_free`` [N, G] are int32 tensors of
    one device, contiguous, owned by the caller; ``block_tokens`` is the size of a cache block.  ``BlockCache.empty`` makes
    the tensors of a new cache.  Every call takes the request lengths [N, G, B] as int32, plain or, with ``step`` [N], as the
    router keeps them (``st["act_base"], step=st["step"]``), and works on the rows ``first`` to ``first + N``.  A tensor of
    another type, shape, layout or device is refused with ValueError.  Calls use the memory that the cache's tensors have
    when they are made (a captured graph that of its capture)."""

    def __init__(self, table, n_blocks, free_list, n_free, block_tokens):
        import torch
        self.torch, self._int32, self._int64 = torch, torch.int32, torch.int64
        if table.dim() != 4 or free_list.dim() != 3:
            raise ValueError("BlockCache: table is [N, G, B, columns] and free_list [N, G, pool]")
        self.device = table.device
        self.N, self.G, self.B, self.columns = table.shape
        try:
            whole = int(block_tokens)
        except (TypeError, ValueError, OverflowError):
            whole = None
        if whole != block_tokens or whole is None:
            raise ValueError(f"block_tokens: needs a whole number of tokens, got {block_tokens!r}")
        self.pool, self.block_tokens = free_list.shape[2], whole
        if not all(-2 ** 31 <= v < 2 ** 31 for v in (self.pool, self.columns, self.block_tokens)):
            raise ValueError("BlockCache: sizes are 32-bit numbers")
        self._fleet, self._worker, self._slot = (self.N,), (self.N, self.G), (self.N, self.G, self.B)
        self._cu = (self.N, self.G, self.B + 1)
        self._list = (*self._worker, self.pool)
        self._table, self._free_list = table, free_list
        self._index = table.get_device()                     # -1: not on a GPU
        self._take(n_blocks, n_free)
        self._whole = None, b""
        if self._index < 0:
            self._current_stream = lambda index: 0
        else:
            self._current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
                (lambda index: torch.cuda.current_stream(index).cuda_stream)
        # (with one GPU it is the current one)
        self._several = self._index >= 0 and torch.cuda.device_count() > 1
        self._current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)

    # (read-only: the calls use the tensors that the handle was made with, or the counts of the last commit)
    table, free_list = property(lambda self: self._table), property(lambda self: self._free_list)
    n_blocks, n_free = property(lambda self: self._n_blocks), property(lambda self: self._n_free)

    def _take(self, n_blocks, n_free):
        self._refuse((self._table, "table", (*self._slot, self.columns)), (n_blocks, "n_blocks", self._slot),
                     (self._free_list, "free_list", self._list), (n_free, "n_free", self._worker))
        self._keep(n_blocks, n_free)

    def _keep(self, n_blocks, n_free):
        self._n_blocks, self._n_free = n_blocks, n_free
        self._addresses = self._table.data_ptr, n_blocks.data_ptr, self._free_list.data_ptr, n_free.data_ptr
        self._at = tuple(address() for address in self._addresses)
        self._packed = _pack_cache(self.G, self.B, self.block_tokens, self.pool, self.columns, *self._at)

    def commit(self, n_blocks, n_free):
        """Takes the counts that an update wrote to other tensors as the cache's own, all rows of them: those outside the
        update's ``first`` to ``first + N`` were not written and have to hold the cache's counts already (copy them in
        ahead of such an update).  The old tensors are free again, but for graphs captured with them."""
        self._refuse((n_blocks, "n_blocks", self._slot), (n_free, "n_free", self._worker))
        if (n_blocks.data_ptr() == self._n_blocks.data_ptr()) != (n_free.data_ptr() == self._n_free.data_ptr()):
            raise ValueError("n_blocks and n_free go together: one of them is the cache's own and the other is not")
        self._keep(n_blocks, n_free)

    @classmethod
    def empty(cls, N, G, B, block_tokens, pool_blocks, table_blocks, device="cuda:0"):
        """A new cache: no request holds a block, and the blocks are given out from number 0 up."""
        import torch
        z = dict(dtype=torch.int32, device=device)
        free = torch.arange(pool_blocks - 1, -1, -1, **z).expand(N, G, pool_blocks).contiguous()
        return cls(torch.zeros((N, G, B, table_blocks), **z), torch.zeros((N, G, B), **z), free,
                   torch.full((N, G), pool_blocks, **z), block_tokens)

    def _is(self, t, shape):
        return t.dtype is self._int32 and t.shape == shape and t.get_device() == self._index and t.is_contiguous()

    def _refuse(self, *arrays):
        for t, name, shape in arrays:
            if t is not None and (t.dtype is not self._int32 or t.shape != shape or t.device != self.device or not t.is_contiguous()):
                raise ValueError(f"{name}: needs a contiguous int32 tensor {list(shape)} on {self.device}, "
                                 f"got {t.dtype} {list(t.shape)} on {t.device}")

    def _batch(self, N, first, stream):
        table, n_blocks, free_list, n_free = self._addresses
        if (table(), n_blocks(), free_list(), n_free()) != self._at:             # a tensor of the cache was given other memory
            self._take(self._n_blocks, self._n_free)
        whole = N is None and first == 0
        if whole:
            N = self.N
        else:
            if N is None:
                N = self.N - first
            if first < 0 or N < 0 or first + N > self.N:
                raise ValueError(f"rows {first} to {first + N}: the cache has {self.N}")
        if self._index < 0 and N:
            raise ValueError(f"the cache is on {self.device}: the calls need tensors on a GPU")
        if stream is None:
            stream = self._current_stream(self._index)
        elif isinstance(stream, C.c_void_p):
            stream = stream.value or 0
        elif hasattr(stream, "cuda_stream"):
            stream = stream.cuda_stream
        if not whole:
            return _pack_batch(N, first, 1, stream)
        packed = self._whole                                 # the batch of all rows on the stream of the last call
        if packed[0] != stream:
            packed = self._whole = stream, _pack_batch(N, 0, 1, stream)
        return packed[1]

    def _call(self, name, batch, *args):
        if self.N == 0:
            return                                           # (empty tensors have no address)
        fn = getattr(_lib or lib(), name)
        if self._several and self._current_device() != self._index:
            with self.torch.cuda.device(self.device):       # the launch goes to the tensors' device
                rc = fn(batch, self._packed, *args)
        else:
            rc = fn(batch, self._packed, *args)
        if rc != BR_OK:
            raise BrError(rc, name)

    def block_tables(self, length, n_blocks_out=None, n_free_out=None, short_blocks=None, step=None, N=None, first=0,
                     stream=None):
        """Brings tables and free lists in line with the lengths; the new counts go to ``n_blocks_out`` and ``n_free_out``
        (default: the cache's own, in place), rows ``first`` to ``first + N`` of them.  With other tensors the cache stays as
        it was until ``commit`` takes them, which takes all rows.  One of the two in place and the other elsewhere is refused
        with ValueError: the counts would not belong together."""
        nb = self._n_blocks if n_blocks_out is None else n_blocks_out
        nf = self._n_free if n_free_out is None else n_free_out
        ok, slot, worker = self._is, self._slot, self._worker
        if not (ok(length, slot) and ok(nb, slot) and ok(nf, worker) and (step is None or ok(step, self._fleet)) and
                (short_blocks is None or ok(short_blocks, worker))):
            self._refuse((length, "length", slot), (nb, "n_blocks_out", slot), (nf, "n_free_out", worker),
                         (step, "step", self._fleet), (short_blocks, "short_blocks", worker))
        batch, at = self._batch(N, first, stream), self._at
        nb = at[1] if n_blocks_out is None else nb.data_ptr()
        nf = at[3] if n_free_out is None else nf.data_ptr()
        if (nb == at[1]) != (nf == at[3]):
            raise ValueError("n_blocks_out and n_free_out go together: both the cache's own or both other tensors")
        self._call("br_block_tables", batch, length.data_ptr(), None if step is None else step.data_ptr(), nb, nf,
                   None if short_blocks is None else short_blocks.data_ptr())

    def slot_map(self, length, cu, slots, n_new=None, step=None, N=None, first=0, stream=None):
        """Cache slots of the newest ``n_new`` tokens of each request (default: one of each running request) into ``slots``
        [N, G, room] int64, with prefix sums ``cu`` [N, G, B + 1]."""
        ok, slot = self._is, self._slot
        if not (ok(length, slot) and ok(cu, self._cu) and (n_new is None or ok(n_new, slot)) and
                (step is None or ok(step, self._fleet))):
            self._refuse((length, "length", slot), (cu, "cu", self._cu), (n_new, "n_new", slot), (step, "step", self._fleet))
        shape = slots.shape
        room = shape[2] if len(shape) == 3 else -1
        if room > MAX_SLOT_ROOM:
            raise ValueError(f"slots: room for {room} tokens a worker; at most {MAX_SLOT_ROOM}")
        if slots.dtype is not self._int64 or shape != (self.N, self.G, room) or slots.get_device() != self._index or \
                not slots.is_contiguous():
            raise ValueError(f"slots: needs a contiguous int64 tensor [{self.N}, {self.G}, room] on {self.device}, "
                             f"got {slots.dtype} {list(slots.shape)} on {slots.device}")
        self._call("br_slot_map", self._batch(N, first, stream), length.data_ptr(),
                   None if step is None else step.data_ptr(), None if n_new is None else n_new.data_ptr(), room,
                   cu.data_ptr(), slots.data_ptr())

    def page_lists(self, length, n_seq, seq_slot, indptr, indices, last_tokens, step=None, N=None, first=0, stream=None):
        """The running requests packed, with their blocks one after another."""
        ok, slot = self._is, self._slot
        if not (ok(length, slot) and ok(n_seq, self._worker) and ok(seq_slot, slot) and ok(indptr, self._cu) and
                ok(indices, self._list) and ok(last_tokens, slot) and (step is None or ok(step, self._fleet))):
            self._refuse((length, "length", slot), (n_seq, "n_seq", self._worker), (seq_slot, "seq_slot", slot),
                         (indptr, "indptr", self._cu), (indices, "indices", self._list), (last_tokens, "last_tokens", slot),
                         (step, "step", self._fleet))
        self._call("br_page_lists", self._batch(N, first, stream), length.data_ptr(),
                   None if step is None else step.data_ptr(), n_seq.data_ptr(), seq_slot.data_ptr(), indptr.data_ptr(),
                   indices.data_ptr(), last_tokens.data_ptr())


def state_to_numpy(st) -> Dict[str, np.ndarray]:
    """Device (or host) torch state -> numpy with the boundary's unsigned types restored."""
    out = {}
    for k, v in st.items():
        a = v.detach().cpu().numpy() if not isinstance(v, np.ndarray) else v
        want = _STATE_DTYPES[k]
        if a.dtype != want and a.dtype.itemsize == np.dtype(want).itemsize:
            a = a.view(want)
        out[k] = a
    return out
