"""A decoding tenant over PyTorch tensors: operator lists, the paged 4-bit cache, and sessions that run them.

``OpList`` writes down a tenant's operators (``include/gacer.h`` has their definitions) over tensors that the caller owns;
``TokenSession`` loads one or several lists into a gacer context and enqueues or runs them; ``Cache`` holds the tensors of a
paged cache.  ``harness.Session`` takes such lists beside its own tenants (``extra=``), so that a decoding tenant runs in
the same regulated rounds as the others.  No arithmetic happens here; every operator runs inside libgacer.so.

Activations are ``[batch, tokens, features]`` or ``[batch, features]``, contiguous, in the list's dtype.
"""
import ctypes as C

import torch

from . import binding as B

_ACT = {"none": B.GACER_ACT_NONE, "relu": B.GACER_ACT_RELU, "relu6": B.GACER_ACT_RELU6, "gelu": B.GACER_ACT_GELU}


def _need(ok, why):
    if not ok:
        raise ValueError(why)


class Cache:
    """The tensors of one layer's paged 4-bit cache (``gacer_cache``): codes uint8 ``[pages, kv_heads, page_tokens, D/2]`` for keys and
    ``[pages, kv_heads, page_tokens/32, D, 16]`` for values, scales int32 ``[pages, kv_heads, page_tokens, D/64]``, and the page table
    int32 ``[batch, pages per sequence]``, whose entries outside the pool mean "no page"."""

    def __init__(self, k_codes, v_codes, k_scales, v_scales, page_table):
        pages, heads, page, half = k_codes.shape
        dim = half * 2
        _need(tuple(v_codes.shape) == (pages, heads, page // 32, dim, 16), "v_codes must be [pages, kv_heads, page_tokens/32, D, 16]")
        for name, t in (("k_scales", k_scales), ("v_scales", v_scales)):
            _need(tuple(t.shape) == (pages, heads, page, dim // B.GACER_CACHE_GROUP) and t.dtype == torch.int32, f"{name} must be int32 [pages, kv_heads, page_tokens, D/64]")
        _need(k_codes.dtype == torch.uint8 and v_codes.dtype == torch.uint8, "codes must be uint8")
        _need(page_table.dim() == 2 and page_table.dtype == torch.int32, "page_table must be int32 [batch, pages]")
        for t in (k_codes, v_codes, k_scales, v_scales, page_table):
            _need(t.is_cuda and t.is_contiguous() and t.device == k_codes.device, "the cache's tensors must be contiguous and on one GPU")
        self.k_codes, self.v_codes, self.k_scales, self.v_scales, self.page_table = k_codes, v_codes, k_scales, v_scales, page_table
        self.pages, self.kv_heads, self.page_tokens, self.head_dim = pages, heads, page, dim

    @classmethod
    def allocate(cls, pages, kv_heads, head_dim, page_table, page_tokens=64, device="cuda"):
        """An empty pool of ``pages`` pages."""
        _need(head_dim in (64, 128), "the cache holds heads of 64 or 128 features")
        z = dict(device=device)
        return cls(torch.zeros(pages, kv_heads, page_tokens, head_dim // 2, dtype=torch.uint8, **z),
                   torch.zeros(pages, kv_heads, page_tokens // 32, head_dim, 16, dtype=torch.uint8, **z),
                   torch.zeros(pages, kv_heads, page_tokens, head_dim // B.GACER_CACHE_GROUP, dtype=torch.int32, **z),
                   torch.zeros(pages, kv_heads, page_tokens, head_dim // B.GACER_CACHE_GROUP, dtype=torch.int32, **z), page_table)


class OpList:
    """One tenant: operators in execution order over the caller's tensors, which the list keeps alive."""

    def __init__(self, dtype, batch):
        _need(dtype in (torch.float32, torch.bfloat16), "a tenant computes in float32 or bfloat16")
        self.dtype, self.batch = dtype, int(batch)
        self.ops, self._descs, self._tensors, self._index, self._keep = [], [], [], {}, []
        self.input = self.output = None
        self.device = None

    @property
    def tensors(self):
        """Logical shapes (n, c, h, w) of the tenant's tensors."""
        return [shape for _, shape in self._tensors]

    def activations(self):
        """The tenant's tensors as [n, h, w, c] views."""
        return [t.view(n, h, w, c) for t, (n, c, h, w) in self._tensors]

    # -- tensors ---------------------------------------------------------------------------------------------------------------
    def _shape(self, t):
        _need(t.dim() in (2, 3), "activations are [batch, features] or [batch, tokens, features]")
        return (t.shape[0], t.shape[-1], t.shape[1] if t.dim() == 3 else 1, 1)

    def _register(self, t):
        _need(t.dtype == self.dtype, f"expected {self.dtype}, got {t.dtype}")
        _need(t.is_cuda and t.is_contiguous(), "activations must be contiguous and on the GPU")
        if self.device is None:
            self.device = t.device
        _need(t.device == self.device, "the tensors of a tenant are on one GPU")
        self._tensors.append((t, self._shape(t)))
        return len(self._tensors) - 1

    def _read(self, t):
        """Index of a tensor that an operator reads; the first one that no operator has written is the tenant's input, others that none
        has written are not allowed (every input of a tenant is its one input tensor or an earlier operator's output)."""
        key = (t.data_ptr(), self._shape(t))
        if key not in self._index:
            _need(self.input is None, "the tensor is neither the tenant's input nor written by an earlier operator")
            self._index[key] = self.input = self._register(t)
        return self._index[key]

    def _write(self, t):
        i = self._register(t)
        self._index[(t.data_ptr(), self._shape(t))] = i
        self.output = i
        return i

    def _array(self, t, dtype, shape, what):
        if t is None:
            return None
        _need(t.dtype == dtype and tuple(t.shape) == tuple(shape), f"{what} must be {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")
        _need(t.is_cuda and t.is_contiguous() and (self.device is None or t.device == self.device), f"{what} must be contiguous and on the tenant's GPU")
        self._keep.append(t)
        return t.data_ptr()

    def _op(self, kind, in0=-1, out=-1, in1=-1, res=-1, w=None, bias=None, scale=None, shift=None, cin=0, cout=0, act="none", alpha=1.0, desc=None):
        if desc is not None:
            self._descs.append(desc)
            w = C.addressof(desc)
        self.ops.append(B.gacer_op(kind, in0, in1, res, out, w, bias, scale, shift, cin, cout, 1, 1, 1, 0, 1, _ACT[act], alpha))

    # -- operators of any tenant that a decoder layer needs ----------------------------------------------------------------------
    def gemm(self, x, weight, out, bias=None, act="none", res=None):
        """out = act(x @ weight.T + bias + res), position by position; weight ``[out features, in features]`` in the list's dtype."""
        i, r = self._read(x), -1 if res is None else self._read(res)
        w = self._array(weight, self.dtype, (out.shape[-1], x.shape[-1]), "weight")
        b = self._array(bias, torch.float32, (out.shape[-1],), "bias")
        self._op(B.GACER_GEMM, i, self._write(out), res=r, w=w, bias=b, cin=x.shape[-1], cout=out.shape[-1], act=act)

    def layernorm(self, x, gamma, beta, out, eps=1e-5, res=None):
        """LayerNorm over the features of x + res."""
        i, r = self._read(x), -1 if res is None else self._read(res)
        g, b = (self._array(t, torch.float32, (x.shape[-1],), what) for t, what in ((gamma, "gamma"), (beta, "beta")))
        self._op(B.GACER_LAYERNORM, i, self._write(out), res=r, scale=g, shift=b, alpha=eps)

    # -- operators of a decoding tenant ------------------------------------------------------------------------------------------
    def qknorm_rope(self, qkv, out, positions, table, *, heads, kv_heads, head_dim, gamma_q=None, gamma_k=None, eps=1e-6, rotary_dims=None,
                    sections=None, interleaved=False):
        """RMS norm of every query and key head, then rotation (GACER_QKNORM_ROPE).  ``positions`` int32 ``[batch, tokens, axes]``, ``table``
        float32 ``[positions, rotary_dims/2, 2]`` (cosine, sine), both None with ``rotary_dims=0``; ``sections``: pairs per axis (default: all on
        one axis).  ``out`` may be ``qkv`` itself."""
        r = head_dim if rotary_dims is None else rotary_dims
        sections = [r // 2] if sections is None else list(sections)
        _need(1 <= len(sections) <= 3, "one to three axes")
        i = self._read(qkv)
        n, _, t, _ = self._shape(qkv)
        p = self._array(positions if r else None, torch.int32, (n, t, len(sections)), "positions")
        _need(not r or (table is not None and table.dim() == 3), "table must be [positions, rotary_dims/2, 2]")
        tab = self._array(table if r else None, torch.float32, (table.shape[0] if r else 0, r // 2, 2), "table")
        gq, gk = (self._array(g, torch.float32, (head_dim,), what) for g, what in ((gamma_q, "gamma_q"), (gamma_k, "gamma_k")))
        d = B.gacer_rope(heads, kv_heads, head_dim, r, int(bool(interleaved)), len(sections), (C.c_int * 3)(*sections), table.shape[0] if r else 0, tab, p)
        self._op(B.GACER_QKNORM_ROPE, i, self._write(out), scale=gq, shift=gk, alpha=eps, desc=d)

    def _cache(self, cache, start, count, heads=0, kv_heads=None, head_dim=None, window=0):
        _need(kv_heads in (None, cache.kv_heads) and head_dim in (None, cache.head_dim), "heads do not match the cache's")
        _need(cache.page_table.shape[0] == self.batch, "the page table has a row per sequence")
        if self.device is None:                      # a list that begins with a cache read
            self.device = cache.k_codes.device
        _need(cache.k_codes.device == self.device, "the cache must be on the tenant's GPU")
        st = self._array(start, torch.int32, (self.batch,), "start")
        ct = self._array(count, torch.int32, (self.batch,), "count")
        _need(st is not None, "start is missing")
        self._keep.append(cache)
        return B.gacer_cache(heads, cache.kv_heads, cache.head_dim, cache.page_tokens, cache.pages, cache.page_table.shape[1], window,
                             cache.k_codes.data_ptr(), cache.v_codes.data_ptr(), cache.k_scales.data_ptr(), cache.v_scales.data_ptr(),
                             cache.page_table.data_ptr(), st, ct)

    def cache_write(self, qkv, cache, start, count=None, *, heads, kv_heads=None, head_dim=None):
        """Keys and values of the new tokens into the cache (GACER_CACHE_WRITE): token t of sequence b at position ``start[b] + t``, for
        t < ``count[b]``."""
        i = self._read(qkv)
        self._op(B.GACER_CACHE_WRITE, i, desc=self._cache(cache, start, count, heads, kv_heads, head_dim))

    def cache_read(self, out, cache, start, count=None):
        """``out[b, t] = [keys | values]`` of the cached token ``start[b] + t`` (GACER_CACHE_READ)."""
        d = self._cache(cache, start, count)
        self._op(B.GACER_CACHE_READ, out=self._write(out), desc=d)

    def cache_attention(self, qkv, out, cache, start, count=None, *, heads, kv_heads=None, head_dim=None, scale=None, window=0):
        """Causal attention of the new tokens' queries over the cache (GACER_CACHE_ATTENTION); ``scale`` defaults to 1/sqrt(head_dim)."""
        i = self._read(qkv)
        d = self._cache(cache, start, count, heads, kv_heads, head_dim, window)
        self._op(B.GACER_CACHE_ATTENTION, i, self._write(out), alpha=cache.head_dim ** -0.5 if scale is None else scale, desc=d)

    def sample(self, logits, tokens, u, *, logp=None, temperature=None, top_k=None, top_p=None, min_p=None):
        """One token per row of logits (GACER_SAMPLE): ``tokens`` int32, ``u`` (random numbers in [0, 1)), ``logp``, ``temperature``,
        ``top_p``, ``min_p`` float32, ``top_k`` int32, each with a value per row."""
        i = self._read(logits)
        rows = (logits.numel() // logits.shape[-1],)
        f = torch.float32
        d = B.gacer_sampling(self._array(u, f, rows, "u"), self._array(temperature, f, rows, "temperature"), self._array(top_k, torch.int32, rows, "top_k"),
                             self._array(top_p, f, rows, "top_p"), self._array(min_p, f, rows, "min_p"), self._array(tokens, torch.int32, rows, "tokens"),
                             self._array(logp, f, rows, "logp"))
        self._op(B.GACER_SAMPLE, i, desc=d)

    # -- descriptor ----------------------------------------------------------------------------------------------------------------
    def descriptor(self, stream=0):
        """The tenant's ``gacer_tenant``; the list must outlive the call that loads it, and its tensors the session."""
        _need(self.ops, "an empty operator list")
        if self.input is None:                       # only cache reads: a tenant still names an input
            self._tensors.append((torch.empty(self.batch, dtype=self.dtype, device=self.device), (self.batch, 1, 1, 1)))
            self.input = len(self._tensors) - 1
        tens = (B.gacer_tensor * len(self._tensors))()
        for i, (t, (n, c, h, w)) in enumerate(self._tensors):
            tens[i] = B.gacer_tensor(n, c, h, w, t.data_ptr(), 0, 0, 0)
        ops = (B.gacer_op * len(self.ops))(*self.ops)
        self._arrays = (tens, ops)
        out = self.input if self.output is None else self.output
        return B.gacer_tenant(len(ops), ops, len(tens), tens, self.input, out, B.GACER_BF16 if self.dtype == torch.bfloat16 else B.GACER_F32,
                              self.batch, C.c_void_p(stream))


class TokenSession:
    """One gacer context with the given operator lists loaded as its tenants."""

    def __init__(self, lists, streams=None):
        if not torch.cuda.is_available():
            raise RuntimeError("a GPU is required: the library has no CPU fallback")
        self.lists = list(lists)
        self.device = self.lists[0].device
        _need(all(l.device == self.device for l in self.lists), "the lists of a session are on one GPU")
        self.ctx = C.c_void_p()
        with torch.cuda.device(self.device):
            B.check(self.ctx, B.gacer_create(C.byref(self.ctx)))
            self.streams = list(streams) if streams is not None else [None] * len(self.lists)
            descs = (B.gacer_tenant * len(self.lists))(*[l.descriptor(s.cuda_stream if s is not None else 0) for l, s in zip(self.lists, self.streams)])
            B.check(self.ctx, B.gacer_load_tenants(self.ctx, descs, len(self.lists)))

    def enqueue(self, tenant=0, stream=None):
        """One round of a tenant on ``stream`` (default: PyTorch's current one), without waiting (gacer_enqueue)."""
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        st = B.gacer_enqueue(self.ctx, tenant, s.cuda_stream)
        if st:
            B.check(self.ctx, st)

    def run(self, mode=B.GACER_MODE_SEQUENTIAL, rounds=1):
        """Rounds of all tenants on their own streams (gacer_run); returns when they have finished."""
        ms = (C.c_float * rounds)()
        with torch.cuda.device(self.device):
            B.check(self.ctx, B.gacer_run(self.ctx, mode, rounds, ms))
        return list(ms)

    def close(self):
        if self.ctx:
            torch.cuda.synchronize(self.device)
            with torch.cuda.device(self.device):
                B.gacer_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
