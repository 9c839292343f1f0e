"""A paged key/value cache on the GPU and attention over it (``include/sim_kv.h``): one ``KVCache`` per pool.

The tensors are torch's; every step runs in the library's CUDA kernels.  Calls are enqueued on torch's current
stream, or on ``stream`` (a cudaStream_t as an int); one cache is used on one stream at a time.  The cache, its plans and the
tensors given to a call on ``stream`` may be dropped while work on them is still to come; the stream has to exist until they are.
Lists of
sequences and offsets are int32 CUDA tensors.  What only the device can see (an unknown sequence, no page left)
is reported by ``check()``.
"""
from __future__ import annotations

import ctypes
import math

from . import _lib as L


def _dtypes():
    import torch
    return {torch.bfloat16: 0, torch.float16: 1}


class AttentionPlan:
    """How the attention of one batch is divided (``KVCache.plan``); holds what the calls with it read."""

    def __init__(self, cache, batch, seqs, cu_q, cu_group, buffer, made_on, stream, captured):
        self.cache, self.batch, self.seqs, self.cu_q, self.cu_group, self._buffer = cache, batch, seqs, cu_q, cu_group, buffer
        self._ref = ctypes.byref(batch)
        self.n_q, self.heads = batch.n_q, batch.q_heads
        self._stream = stream       # whose next plan may have the buffer, None: no other plan
        self._read_on = {made_on}   # streams that the allocator knows of
        self._captured = captured   # what it reads lives as long as the graph that reads it

    def _read_elsewhere(self, stream, capturing):
        """Before it is read on a stream that is not the one it was made on, or in a graph: what it reads outlives the plan."""
        self._stream = None
        held = [x for x in (self._buffer, self.seqs, self.cu_q, self.cu_group) if x is not None]
        if capturing:
            if not self._captured:
                self.cache._in_graphs.append(held)
                self._captured = True
        elif stream not in self._read_on:
            self.cache._record(stream, held)
            self._read_on.add(stream)

    def __del__(self):
        if self._stream is not None and len(self.cache._spare) < 2:
            self.cache._spare.append((self._stream, self._buffer))


class KVCache:
    """``n_pages`` pages of ``page_size`` tokens, each with the keys and values of all layers and kv heads; up to
    ``max_seqs`` sequences of up to ``max_pages`` pages.  ``pool`` [n_pages, n_layers, 2, n_kv_heads, page_size,
    head_dim], ``table`` [max_seqs, max_pages], ``length`` [max_seqs] and ``ref`` [n_pages] are its state.

    With ``bits=4`` keys and values of the type ``dtype`` are quantised as they are written: each 32 of a token's head (the last ones:
    fewer) are held as their lowest, a step and 4 bits each, in 20 bytes (5 bits a value if head_dim is a multiple of 32); ``pool`` is then
    uint8 [n_pages, n_layers, 2, n_kv_heads, page_size, 20 ceil(head_dim / 32)], in strips of 16 tokens (``include/sim_kv.h``).  A value
    read back, or attended to, is the 16-bit float nearest to lowest + code step: half a step and a rounding from the one written, together at
    most a step, which is at most a 15th of the distance from the lowest of its 32 to the highest (or 15 times the type's smallest float)."""

    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, max_seqs: int, max_pages: int,
                 n_layers: int = 1, dtype=None, device="cuda", bits: int = 16):
        import torch
        if bits not in (4, 16):
            raise ValueError("bits must be 4 or 16")
        ints = dict(dtype=torch.int32, device=device)
        dtype = dtype or torch.bfloat16
        kind, last = (dtype, head_dim) if bits == 16 else (torch.uint8, 20 * -(-head_dim // 32))
        self._set(torch.empty(n_pages, n_layers, 2, n_kv_heads, page_size, last, dtype=kind, device=device),
                  torch.full((max_seqs, max_pages), -1, **ints), torch.zeros(max_seqs, **ints), torch.zeros(n_pages, **ints), head_dim, dtype)

    @classmethod
    def wrap(cls, pool, table, length, ref, head_dim: int | None = None, dtype=None) -> "KVCache":
        """A cache over tensors that exist (laid out as above, on one CUDA device); nothing is copied.  A uint8 pool is
        one of 4 bits, which does not say its ``head_dim`` and ``dtype``."""
        self = cls.__new__(cls)
        self._set(pool, table, length, ref, head_dim, dtype)
        return self

    def _set(self, pool, table, length, ref, head_dim=None, dtype=None):
        import torch
        packed = pool.dtype == torch.uint8
        if pool.dim() != 6 or pool.shape[2] != 2 or (not packed and pool.dtype not in _dtypes()) or not pool.is_cuda:
            raise ValueError("pool must be a CUDA tensor [n_pages, n_layers, 2, n_kv_heads, page_size, head_dim] of bfloat16 or float16, "
                             "or of uint8 for 4 bits")
        n_pages, n_layers, _, heads, page, dim = pool.shape
        if packed:
            if head_dim is None or dtype not in _dtypes() or dim != 20 * -(-head_dim // 32):
                raise ValueError("a pool of 4 bits needs its dtype, bfloat16 or float16, and a head_dim with 20 ceil(head_dim / 32) bytes a token")
            dim = head_dim
        elif head_dim not in (None, dim) or dtype not in (None, pool.dtype):
            raise ValueError(f"the pool is {pool.dtype} with head_dim {dim}")
        else:
            dtype = pool.dtype
        if table.dim() != 2 or length.shape != table.shape[:1] or ref.shape != (n_pages,):
            raise ValueError("table must be [max_seqs, max_pages], length [max_seqs] and ref [n_pages]")
        for x in (pool, table, length, ref):
            if not x.is_contiguous() or x.device != pool.device or (x is not pool and x.dtype != torch.int32):
                raise ValueError("pool, table, length and ref must be contiguous, on one device, the last three int32")
        self.pool, self.table, self.length, self.ref = pool, table, length, ref
        self.device, self.dtype, self.bits = pool.device, dtype, 4 if packed else 16
        self.status = torch.zeros(1, dtype=torch.int32, device=pool.device)
        self._kv = L.sim_kv(pool.data_ptr(), table.data_ptr(), length.data_ptr(), ref.data_ptr(), self.status.data_ptr(), None,
                            _dtypes()[dtype] | (L.SIM_KV_4BIT if packed else 0), n_pages, n_layers, heads, page, dim, table.shape[0], table.shape[1])
        self._ref = ctypes.byref(self._kv)
        self._lib = L.lib()
        size = self._lib.sim_kv_scratch_bytes(self._ref)
        if size == 0:
            raise ValueError("sizes outside the cache's limits (see include/sim_kv.h)")
        self._scratch = torch.empty(size, dtype=torch.uint8, device=pool.device)
        self._kv.scratch = self._scratch.data_ptr()
        self._index, self._dim, self._heads, self._n_pages = pool.device.index, dim, heads, n_pages
        self._torch, self._i32 = torch, torch.int32
        self._sizes = {}  # bytes of a plan and its workspace by the batch's sizes
        self._spare = []  # streams and buffers of plans that are gone: the workspace of the next ones
        self._streams = set()  # where the cache has been used
        self._in_graphs = []  # what plans made outside of a graph have left to its replays
        torch.cuda.current_stream(self.device).synchronize()  # the first call may be on any stream

    def _empty(self, stream, shape, dtype):
        """A tensor whose memory belongs to the stream that the call runs on."""
        torch = self._torch
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=self.device)):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _stream(self, stream):
        torch = self._torch
        if torch._C._cuda_getDevice() != self._index:
            raise ValueError(f"the cache is on {self.device}, which is not the current device")
        st = torch._C._cuda_getCurrentRawStream(self._index) if stream is None else int(stream)
        if st not in self._streams:
            self._record(st, (self.pool, self.table, self.length, self.ref, self.status, self._scratch))
            self._streams.add(st)
        return st

    def _lend(self, stream, *tensors):
        if stream is not None:
            self._record(int(stream), [x for x in tensors if x is not None])

    def _capturing(self, stream):
        torch = self._torch
        if stream is None:
            return torch.cuda.is_current_stream_capturing()
        with torch.cuda.stream(torch.cuda.ExternalStream(int(stream), device=self.device)):
            return torch.cuda.is_current_stream_capturing()

    def _record(self, stream, tensors):
        """Their memory is used on that stream: the allocator gives it to others only after the work enqueued there."""
        on = self._torch.cuda.ExternalStream(stream, device=self.device)
        for x in tensors:
            x.record_stream(on)

    def _fail(self, rc):
        raise L.SimError(rc, L.sim_last_error(None))

    def _ints(self, name, x, n):
        if x.dtype is not self._i32 or x.shape != (n,) or x.get_device() != self._index or not x.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor of {n} values on {self.device}")
        return x.data_ptr()

    def _rows(self, name, x, n, heads):
        token, head, last = x.stride() if x.dim() == 3 else (0, 0, 0)
        if last != 1 or x.dtype is not self.dtype or x.shape != (n, heads, self._dim) or x.get_device() != self._index:
            raise ValueError(f"{name} must be {self.dtype} [{n}, {heads}, {self._dim}] on {self.device}, the last dimension contiguous")
        if x.requires_grad and self._torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which these calls do not have: detach it, or call under torch.no_grad()")
        return x.data_ptr(), token, head

    def check(self) -> None:
        """Raise if a call has been refused, in part or as a whole, since the last check.  Waits for the device, calls on
        all streams and in replayed graphs included."""
        self._torch.cuda.synchronize(self.device)
        code = int(self.status.item())
        if code != L.SIM_OK:
            self.status.zero_()
            self._torch.cuda.current_stream(self.device).synchronize()  # later calls may be on any stream
        if code == L.SIM_E_NOMEM:
            raise L.SimError(code, "too few free pages: that call changed nothing")
        if code == L.SIM_E_INVAL:
            raise L.SimError(code, "a sequence out of range, repeated, or without room: that entry was left out")
        if code != L.SIM_OK:
            raise L.SimError(code, "an internal wait ran out")

    # ---- pages --------------------------------------------------------------------------------------------------

    def extend(self, seqs, cu_new, n_new: int, stream: int | None = None):
        """Room for cu_new[i + 1] - cu_new[i] tokens at the end of seqs[i] (``n_new`` in all); returns their slots
        (int64, -1 where refused).  A shared last page is copied first."""
        n, st = seqs.shape[0], self._stream(stream)
        slots = self._empty(stream, (n_new,), self._torch.int64)
        rc = self._lib.sim_kv_extend(self._ref, n, self._ints("seqs", seqs, n), self._ints("cu_new", cu_new, n + 1), n_new,
                                     slots.data_ptr(), st)
        if rc:
            self._fail(rc)
        self._lend(stream, seqs, cu_new)
        return slots

    def write(self, slots, k, v, layer: int = 0, stream: int | None = None) -> None:
        """Keys and values [n_new, n_kv_heads, head_dim] of one layer into their slots; quantised in a cache of 4 bits."""
        n = slots.shape[0]
        if slots.dtype is not self._torch.int64 or slots.get_device() != self._index or slots.dim() != 1 or not slots.is_contiguous():
            raise ValueError(f"slots must be a contiguous int64 tensor on {self.device}")
        st = self._stream(stream)
        rc = self._lib.sim_kv_write(self._ref, layer, n, slots.data_ptr(), *self._rows("k", k, n, self._heads),
                                    *self._rows("v", v, n, self._heads), st)
        if rc:
            self._fail(rc)
        self._lend(stream, slots, k, v)

    def read(self, seqs, cu, n: int, layer: int = 0, first=None, stream: int | None = None):
        """Cached keys and values of one layer, each [n, n_kv_heads, head_dim], in order: rows cu[i] .. cu[i + 1] - 1 are the
        tokens of seqs[i] from first[i] on (0 by default).  Rows of an entry that is refused are zeros."""
        m, st = seqs.shape[0], self._stream(stream)
        if not 0 <= n < 1 << 31:  # before the tensors are made; ctypes would cut it off
            raise ValueError("n must be in [0, 2^31)")
        k, v = (self._empty(stream, (n, self._heads, self._dim), self.dtype) for _ in range(2))
        at = self._heads * self._dim, self._dim
        rc = self._lib.sim_kv_read(self._ref, layer, m, self._ints("seqs", seqs, m), self._ints("cu", cu, m + 1),
                                   None if first is None else self._ints("first", first, m), n, k.data_ptr(), *at, v.data_ptr(), *at, st)
        if rc:
            self._fail(rc)
        self._lend(stream, seqs, cu, first)
        return k, v

    def fork(self, src, dst, tokens=None, stream: int | None = None) -> None:
        """dst[i] (empty) becomes the first tokens[i] tokens of src[i], on the same pages."""
        n, st = src.shape[0], self._stream(stream)
        rc = self._lib.sim_kv_fork(self._ref, n, self._ints("src", src, n), self._ints("dst", dst, n),
                                   None if tokens is None else self._ints("tokens", tokens, n), st)
        if rc:
            self._fail(rc)
        self._lend(stream, src, dst, tokens)

    def copy(self, src, dst, stream: int | None = None) -> None:
        """dst[i] (empty) becomes src[i], on pages of its own."""
        n, st = src.shape[0], self._stream(stream)
        rc = self._lib.sim_kv_copy(self._ref, n, self._ints("src", src, n), self._ints("dst", dst, n), st)
        if rc:
            self._fail(rc)
        self._lend(stream, src, dst)

    def free(self, seqs, keep=None, stream: int | None = None) -> None:
        """seqs[i] keeps its first keep[i] tokens (none by default) and gives the other pages back."""
        n, st = seqs.shape[0], self._stream(stream)
        rc = self._lib.sim_kv_free(self._ref, n, self._ints("seqs", seqs, n),
                                   None if keep is None else self._ints("keep", keep, n), st)
        if rc:
            self._fail(rc)
        self._lend(stream, seqs, keep)

    def compact(self, stream: int | None = None):
        """Move the pages in use to the lowest numbers; returns each page's new number (int32, -1: was free)."""
        st = self._stream(stream)
        to = self._empty(stream, (self._n_pages,), self._i32)
        rc = self._lib.sim_kv_compact(self._ref, to.data_ptr(), st)
        if rc:
            self._fail(rc)
        return to

    # ---- attention ----------------------------------------------------------------------------------------------

    def plan(self, seqs, cu_q, n_q: int, heads: int, cu_group=None, stream: int | None = None) -> AttentionPlan:
        """Divide a batch's attention: entry i has the query tokens cu_q[i] .. cu_q[i + 1] - 1 (``n_q`` in all), the
        last ones of sequence seqs[i].  Entries cu_group[g] .. cu_group[g + 1] - 1 may share a prefix: pages that
        all of them begin with are read once.  Valid until lengths or tables change; what a captured ``attend`` reads of
        it is kept as long as the cache."""
        n, st = seqs.shape[0], self._stream(stream)
        ng = 0 if cu_group is None else max(cu_group.shape[0] - 1, 0)
        b = L.sim_kv_batch(n, n_q, heads, ng, self._ints("seqs", seqs, n), self._ints("cu_q", cu_q, n + 1),
                           None if cu_group is None else self._ints("cu_group", cu_group, ng + 1), None, None)
        sizes = self._sizes.get((n, n_q, heads, ng))
        if sizes is None:
            size = self._lib.sim_kv_plan_bytes(self._ref, ctypes.byref(b))
            sizes = (size + 255) // 256 * 256, self._lib.sim_kv_workspace_bytes(self._ref, ctypes.byref(b))
            if len(self._sizes) > 1000:
                self._sizes.clear()
            self._sizes[n, n_q, heads, ng] = sizes
        size, buffer, mine = sizes[0] + sizes[1] + 16, None, None
        capturing = self._capturing(stream)
        if stream is None and not capturing:  # a graph's buffers are its own
            mine = st
            while buffer is None and self._spare:
                of, buffer = self._spare.pop()
                if of != st or buffer.shape[0] < size:
                    buffer = None
        if buffer is None:
            buffer = self._empty(stream, (size,), self._torch.uint8)
        b.plan = buffer.data_ptr()
        b.workspace = b.plan + sizes[0]
        plan = AttentionPlan(self, b, seqs, cu_q, cu_group, buffer, st, mine, capturing)
        rc = self._lib.sim_kv_plan(self._ref, plan._ref, st)
        if rc:
            self._fail(rc)
        self._lend(stream, seqs, cu_q, cu_group)
        return plan

    def attend(self, q, plan: AttentionPlan, layer: int = 0, scale: float | None = None, out=None, lse=None, stream: int | None = None):
        """softmax(scale q k^T) v of queries [n_q, heads, head_dim] over the keys that each sees, and the log of the
        sum of exponentials [n_q, heads] (float32); scale is head_dim ** -0.5 by default.  There is no backward pass:
        tensors that require a gradient are refused, here and in ``write``, unless gradients are switched off."""
        torch, st, dim = self._torch, self._stream(stream), self._dim
        if plan.cache is not self:
            raise ValueError("the plan is another cache's")
        if plan._stream != st or torch.cuda.is_current_stream_capturing():
            plan._read_elsewhere(st, self._capturing(stream))
        rows = self._rows("q", q, plan.n_q, plan.heads)
        if out is None:
            out = self._empty(stream, (plan.n_q, plan.heads, dim), self.dtype)
            to = out.data_ptr(), plan.heads * dim, dim
        else:
            to = self._rows("out", out, plan.n_q, plan.heads)
        if lse is None:
            lse = self._empty(stream, (plan.n_q, plan.heads), torch.float32)
        elif lse.dtype is not torch.float32 or lse.get_device() != self._index or lse.shape != (plan.n_q, plan.heads) or not lse.is_contiguous():
            raise ValueError(f"lse must be a contiguous float32 tensor [{plan.n_q}, {plan.heads}] on {self.device}")
        rc = self._lib.sim_kv_attend(self._ref, plan._ref, layer, *rows, 1.0 / math.sqrt(dim) if scale is None else scale,
                                     *to, lse.data_ptr(), st)
        if rc:
            self._fail(rc)
        self._lend(stream, q, out, lse)
        return out, lse
