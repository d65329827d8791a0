"""Device-memory plumbing around the C ABI: one layer's cache, factors and workspaces
(``Layer``: the low-rank cache; ``DenseLayer``: an uncompressed layer's 8-bit cache), and rotary
positions (``Rope``).

PyTorch provides device memory and the stream; every computation runs in the
library's HIP kernels.
"""
from __future__ import annotations

from typing import Optional

import numpy as np

from . import starkv as S


def to_dev(bits: np.ndarray, device="cuda"):
    """uint16 / int32 / uint8 numpy array -> device tensor with the same bytes."""
    import torch
    a = np.ascontiguousarray(bits)
    if a.dtype == np.uint16:
        a = a.view(np.int16)
    return torch.from_numpy(a.copy()).to(device)


class PagePool:
    """Host-side page allocator of a paged cache (continuous batching).

    Keeps the free pool pages and, per sequence slot, the pages it holds; the block
    table lives on the device (the plan reads it) with a host copy that ``sync``
    uploads.  Pages are handed out lowest-free-first unless ``rng`` shuffles the
    free list (tests use that to scatter sequences over the pool)."""

    def __init__(self, n_pages: int, page_tokens: int, batch: int, capacity: int,
                 device="cuda", rng: Optional[np.random.Generator] = None):
        import torch
        self.n_pages, self.page_tokens, self.batch = n_pages, page_tokens, batch
        self.capacity = capacity
        self.per_seq = -(-capacity // page_tokens)
        free = np.arange(n_pages, dtype=np.int32)
        if rng is not None:
            free = rng.permutation(free).astype(np.int32)
        self.free = list(free[::-1])                 # pop() hands out free[0] first
        self.host = np.full((batch, self.per_seq), -1, np.int32)
        self.table = torch.full((batch, self.per_seq), -1, dtype=torch.int32, device=device)

    def ensure(self, b: int, n_tokens: int) -> None:
        """Give sequence b pages for its first n_tokens tokens."""
        need = -(-n_tokens // self.page_tokens)
        if n_tokens > self.capacity:
            raise ValueError(f"sequence {b}: {n_tokens} tokens exceed the capacity")
        for j in range(need):
            if self.host[b, j] < 0:
                if not self.free:
                    raise MemoryError("page pool exhausted")
                self.host[b, j] = self.free.pop()

    def release(self, b: int) -> None:
        """Return all pages of sequence b to the pool."""
        for j in range(self.per_seq):
            if self.host[b, j] >= 0:
                self.free.append(int(self.host[b, j]))
                self.host[b, j] = -1

    def pages_in_use(self) -> int:
        return int((self.host >= 0).sum())

    def sync(self) -> None:
        """Upload the host table (stream-ordered before later library calls)."""
        import torch
        self.table.copy_(torch.from_numpy(self.host))


class Layer:
    """Plan + cache + workspaces of one attention layer (contiguous, or paged when
    page_tokens > 0: then ``pool`` is the layer's PagePool)."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, capacity, key_rank, value_rank,
                 qmode, rope_theta, q_dtype, out_dtype, d_model=0, device="cuda",
                 max_ctx: Optional[int] = None, page_tokens: int = 0, n_pages: int = 0,
                 page_rng: Optional[np.random.Generator] = None):
        import torch
        self.pool = None
        if page_tokens:
            self.pool = PagePool(n_pages, page_tokens, batch, capacity, device, page_rng)
        self.cfg = S.make_config(batch, n_q_heads, n_kv_heads, head_dim, capacity, key_rank,
                                 value_rank, qmode, rope_theta, d_model=d_model,
                                 q_dtype=q_dtype, out_dtype=out_dtype, page_tokens=page_tokens,
                                 n_pages=n_pages,
                                 block_table=self.pool.table if self.pool else None)
        self.plan = S.starkv_plan_create(self.cfg)
        self.device = device
        self.batch, self.n_q, self.head_dim = batch, n_q_heads, head_dim
        self.capacity = capacity
        self.out_dtype = out_dtype
        self.cache = torch.zeros(S.starkv_cache_bytes(self.plan), dtype=torch.uint8, device=device)
        self.max_ctx = capacity if max_ctx is None else max_ctx
        self.dec_ws = torch.empty(max(S.starkv_decode_workspace_bytes(self.plan, self.max_ctx), 256),
                                  dtype=torch.uint8, device=device)
        self.app_ws = None
        self.out = torch.empty((batch, n_q_heads, head_dim),
                               dtype=torch.float32 if out_dtype == S.DT_F32 else torch.int16,
                               device=device)

    def _app_ws(self, n_new: int):
        import torch
        need = S.starkv_append_workspace_bytes(self.plan, n_new)
        if need == 0:
            return None
        if self.app_ws is None or self.app_ws.numel() < need:
            self.app_ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self.app_ws

    def append(self, x_or_latents, pos, A_all=None, stream=None):
        n_new = int(x_or_latents.shape[1])
        ws = self._app_ws(n_new)
        S.starkv_append(self.plan, self.cache, x_or_latents, A_all, pos, n_new, ws, stream=stream)

    def decode(self, q, B_k, B_v, ctx_len, max_ctx: Optional[int] = None, out=None, stream=None):
        mc = self.max_ctx if max_ctx is None else max_ctx
        out = self.out if out is None else out
        S.starkv_decode_attn(self.plan, self.cache, q, B_k, B_v, ctx_len, mc, out, self.dec_ws,
                             stream=stream)
        return out

    def decode_absorbed(self, q, B_k, W_abs, ctx_len, max_ctx: Optional[int] = None, out=None,
                        stream=None):
        """Attention-block output [B][d_out] with the value up-projection absorbed into the
        output projection; W_abs [d_out][H_q * r_v] fp16 bits (int16 tensor)."""
        import torch
        mc = self.max_ctx if max_ctx is None else max_ctx
        d_out = int(W_abs.shape[0])
        if out is None:
            out = torch.empty((self.batch, d_out),
                              dtype=torch.float32 if self.out_dtype == S.DT_F32 else torch.int16,
                              device=self.device)
        S.starkv_decode_attn_absorbed(self.plan, self.cache, q, B_k, W_abs, d_out, ctx_len, mc,
                                      out, self.dec_ws, stream=stream)
        return out

    def out_float(self, out=None):
        """Output bit patterns -> float64 numpy."""
        import torch
        o = (self.out if out is None else out).cpu()
        if self.out_dtype == S.DT_F32:
            return o.to(torch.float64).numpy()
        if self.out_dtype == S.DT_BF16:
            return o.view(torch.bfloat16).to(torch.float64).numpy()
        return o.view(torch.float16).to(torch.float64).numpy()


# ------------------------------------------------------------------- uncompressed layers

_types = {}              # library dtype -> the torch types that may hold it


def _types_of(dtype):
    """The torch type of a library dtype and the integer of the same width, for bit patterns."""
    if not _types:
        import torch
        _types.update({S.DT_F16: (torch.float16, torch.int16),
                       S.DT_BF16: (torch.bfloat16, torch.int16),
                       S.DT_F32: (torch.float32, torch.int32)})
    return _types[dtype]


def _array(name, t, shape, dtype, device):
    """Checks a [B][n][H][d] array; returns its strides for the library (None: packed)."""
    if t.dtype not in _types_of(dtype):
        raise TypeError(f"{name}: {t.dtype}, expected {_types_of(dtype)[0]}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the layer on {device}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.is_contiguous():
        return None
    b, n, h, d = t.stride()
    if d != 1 and shape[3] > 1:
        raise ValueError(f"{name}: channels must be contiguous")
    return S.starkv_strides(b, n, h)


def _vector(name, t, shape, dtype, device):
    """Checks a packed array of int32 (dtype "int32") or float32."""
    if str(t.dtype)[6:] != dtype:
        raise TypeError(f"{name}: {t.dtype}, expected {dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the layer on {device}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous array of shape {tuple(shape)}")


def _run(device, stream, fn, *args):
    """fn(*args, stream=...) with the arrays' device current; on torch's current stream there unless
    one is given (its handle alone: the stream object would cost 2 us a call)."""
    import torch
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(device.index)
    if torch.cuda.current_device() == device.index:
        fn(*args, stream=stream)
    else:
        with torch.cuda.device(device):
            fn(*args, stream=stream)


def _cuda(device):
    import torch
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"a GPU is needed, got {device}")
    return device if device.index is not None else torch.device("cuda", torch.cuda.current_device())


class Rope:
    """Rotary positions: ``rope(x, positions)`` rotates x [B][n][H][d] (or [n][H][d]) at
    positions [B][n] (or [n]), int32.  ``out`` may be x itself; ``inverse`` applies the transposed
    map, the gradient with respect to x."""

    def __init__(self, head_dim, theta, rotary_dim=None, layout=S.ROPE_HALF,
                 scaling=S.ROPE_PLAIN, factor=1.0, original_ctx=0, turns_low=0.0, turns_high=0.0,
                 gain=0.0, dtype=S.DT_BF16):
        self.cfg = S.make_rope_config(head_dim, theta, rotary_dim, layout, scaling, factor,
                                      original_ctx, turns_low, turns_high, gain, dtype)
        self.plan = S.starkv_rope_plan_create(self.cfg)

    def __call__(self, x, positions, out=None, inverse=False, stream=None):
        import torch
        if x.device.type != "cuda" or x.dim() not in (3, 4):
            raise ValueError("x: a GPU array [B][n][H][d] or [n][H][d] is needed")
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        a, o, pos = x, out, positions
        if x.dim() == 3:
            a, o, pos = x.unsqueeze(0), out.unsqueeze(0), positions.unsqueeze(0)
        shape = (*a.shape[:3], self.cfg.head_dim)
        xs = _array("x", a, shape, self.cfg.dtype, x.device)
        os_ = _array("out", o, shape, self.cfg.dtype, x.device)
        _vector("positions", pos, shape[:2], "int32", x.device)
        if 0 in shape:
            return out
        _run(x.device, stream, S.starkv_rope, self.plan, a, xs, o, os_, pos, shape[0], shape[1],
             shape[2], int(inverse))
        return out


class DenseLayer:
    """Plan, 8-bit cache and workspaces of one uncompressed attention layer.

    ``block_table`` (int32 [batch][n_kv_heads][blocks]) names the pool block of every block of
    every KV head; without one the layer makes a table that gives each head its own run of
    blocks.  Arrays of queries, keys, values and outputs are [B][n][H][d] (or [B][H][d] for one
    token) with contiguous channels and any other strides."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, capacity, code=S.CODE_INT8,
                 block_tokens=64, dtype=S.DT_BF16, softmax_scale=0.0, n_blocks=None,
                 block_table=None, device="cuda"):
        import torch
        self.batch, self.n_q, self.n_kv, self.head_dim = batch, n_q_heads, n_kv_heads, head_dim
        self.capacity, self.block_tokens, self.dtype = capacity, block_tokens, dtype
        self.device = _cuda(device if block_table is None else block_table.device)
        self.blocks = -(-capacity // max(block_tokens, 1))
        shape = (batch, n_kv_heads, self.blocks)
        if block_table is None:
            n = batch * n_kv_heads * self.blocks
            block_table = torch.arange(n, dtype=torch.int32, device=self.device).view(shape)
        _vector("block_table", block_table, shape, "int32", self.device)
        self.table = block_table
        if n_blocks is None:
            n_blocks = batch * n_kv_heads * self.blocks
        self.cfg = S.make_dense_config(batch, n_q_heads, n_kv_heads, head_dim, capacity, n_blocks,
                                       block_table, code, block_tokens, dtype, softmax_scale)
        self.plan = S.starkv_dense_plan_create(self.cfg)
        self.cache = torch.empty(S.starkv_dense_cache_bytes(self.plan), dtype=torch.uint8,
                                 device=self.device)
        self._ws = {}

    def new_weights(self):
        """Zeroed block weights, to be gathered by ``attend`` and used by ``evict``."""
        import torch
        return torch.zeros((self.batch, self.n_kv, self.blocks), dtype=torch.float32,
                           device=self.device)

    def _lengths(self, name, t):
        _vector(name, t, (self.batch,), "int32", self.device)

    def append(self, k, v, pos, n_new=None, stream=None):
        """Tokens k, v [B][n][H_kv][d] at positions pos[b] ..; n_new: how many of the n in each
        sequence (int32 [B], default all)."""
        if k.dim() == 3:
            k, v = k.unsqueeze(1), v.unsqueeze(1)
        shape = (self.batch, k.shape[1], self.n_kv, self.head_dim)
        ks = _array("k", k, shape, self.dtype, self.device)
        vs = _array("v", v, shape, self.dtype, self.device)
        self._lengths("pos", pos)
        if n_new is not None:
            self._lengths("n_new", n_new)
        if shape[1] == 0:
            return
        _run(self.device, stream, S.starkv_dense_append, self.plan, self.cache, k, ks, v, vs, pos,
             shape[1], n_new)

    def read(self, ctx_len, start, k_out, v_out, stream=None):
        """Rows start[b] .. of the cache into k_out, v_out [B][n][H_kv][d] (16 or 32 bits)."""
        import torch
        dtype = {torch.float32: S.DT_F32, torch.float16: S.DT_F16,
                 torch.bfloat16: S.DT_BF16}.get(k_out.dtype)
        if dtype is None:
            raise TypeError(f"k_out: {k_out.dtype}")
        shape = (self.batch, k_out.shape[1], self.n_kv, self.head_dim)
        ks = _array("k_out", k_out, shape, dtype, self.device)
        vs = _array("v_out", v_out, shape, dtype, self.device)
        self._lengths("ctx_len", ctx_len)
        self._lengths("start", start)
        if shape[1] == 0:
            return
        _run(self.device, stream, S.starkv_dense_read, self.plan, self.cache, ctx_len, start,
             shape[1], k_out, ks, v_out, vs, dtype)

    def workspace(self, n_q=1, weights=False):
        """The workspace that ``attend`` uses for n_q query tokens.  It is kept, so a captured
        call may be replayed as long as the layer lives; calls that share it must not overlap."""
        import torch
        key = (n_q, bool(weights))
        if key not in self._ws:
            need = S.starkv_dense_workspace_bytes(self.plan, n_q, self.capacity, weights)
            self._ws[key] = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._ws[key]

    def attend(self, q, ctx_len, q_len=None, max_ctx=None, weights=None, out=None, ws=None,
               stream=None):
        """Attention of the last query tokens q [B][n][H_q][d] over the first ctx_len[b] tokens;
        q_len: how many of the n in each sequence (other rows of ``out`` stay as they are)."""
        import torch
        if out is None:
            make = torch.empty if q_len is None else torch.zeros
            out = make(q.shape, dtype=q.dtype, device=self.device)
        a, o = (q.unsqueeze(1), out.unsqueeze(1)) if q.dim() == 3 else (q, out)
        shape = (self.batch, a.shape[1], self.n_q, self.head_dim)
        qs = _array("q", a, shape, self.dtype, self.device)
        os_ = _array("out", o, shape, self.dtype, self.device)
        self._lengths("ctx_len", ctx_len)
        if q_len is not None:
            self._lengths("q_len", q_len)
        if weights is not None:
            _vector("weights", weights, (self.batch, self.n_kv, self.blocks), "float32",
                    self.device)
        if shape[1] == 0:
            return out
        if ws is None:
            ws = self.workspace(shape[1], weights is not None)
        _run(self.device, stream, S.starkv_dense_attn, self.plan, self.cache, a, qs, shape[1],
             q_len, ctx_len, self.capacity if max_ctx is None else max_ctx, o, os_, weights, ws)
        return out

    def evict(self, weights, ctx_len, keep, sink=0, recent=0, table_out=None, weights_out=None,
              ctx_out=None, stream=None):
        """Shortens every sequence to about ``keep`` finished blocks per KV head (see
        starkv_dense_evict); in place where no output is given.  Returns (table, weights,
        ctx_len)."""
        shape = (self.batch, self.n_kv, self.blocks)
        _vector("weights", weights, shape, "float32", self.device)
        self._lengths("ctx_len", ctx_len)
        if table_out is not None:
            _vector("table_out", table_out, shape, "int32", self.device)
        if weights_out is not None:
            _vector("weights_out", weights_out, shape, "float32", self.device)
        if ctx_out is not None:
            self._lengths("ctx_out", ctx_out)
        _run(self.device, stream, S.starkv_dense_evict, self.plan, weights, ctx_len, keep, sink,
             recent, table_out, weights_out, ctx_out)
        return (self.table if table_out is None else table_out,
                weights if weights_out is None else weights_out,
                ctx_len if ctx_out is None else ctx_out)
