"""The binding's calls over a paged key-value cache (include/rbs.h, last section).

The buffers that live as long as a cache does (its pages, their bookkeeping, a
rotation's weights) sit in objects that check them once, when made, and keep
their C structs: a decode step's calls are short, and the checks of all of
their tensors would take longer than the kernels.  The tensors that change from
call to call are checked at every call, as in the other calls.

stream: where a call goes, the current stream by default.  What a call makes
itself (outputs that are not given, the workspace) is that stream's memory, which
nothing else uses before the stream's earlier work is done; outputs may be dropped
once the current stream's work that uses them has been queued.
"""

from __future__ import annotations

import ctypes
import math
import threading
from dataclasses import dataclass, field

import torch

from . import _lib as L

RBS_CACHE_BF16, RBS_CACHE_FP8 = 0, 1
RBS_PAGES_FEW, RBS_PAGES_ROW, RBS_PAGES_TOKENS, RBS_PAGES_STACK = 1, 2, 4, 8
RBS_MAX_ROWS = 4096


class rbs_cache(ctypes.Structure):
    _fields_ = [
        ("n_pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("format", ctypes.c_int32),
        ("stride_page", ctypes.c_int64),
        ("stride_head", ctypes.c_int64),
        ("stride_tok", ctypes.c_int64),
        ("K", ctypes.c_void_p),
        ("V", ctypes.c_void_p),
        ("amax", ctypes.c_void_p),
    ]


class rbs_pages(ctypes.Structure):
    _fields_ = [
        ("n_rows", ctypes.c_int32),
        ("max_pages", ctypes.c_int32),
        ("n_pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("page_table", ctypes.c_void_p),
        ("free_pages", ctypes.c_void_p),
    ]


class rbs_rope(ctypes.Structure):
    _fields_ = [
        ("q_weight", ctypes.c_void_p),
        ("k_weight", ctypes.c_void_p),
        ("inv_freq", ctypes.c_void_p),
        ("rot_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("factor", ctypes.c_float),
    ]


def declare(lib):
    """Argument types of the paged calls (called by load())."""
    P, I32, F32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    SP = ctypes.POINTER(L.rbs_shape)
    lib.rbs_pages_extend.argtypes = [ctypes.POINTER(rbs_pages), P, P, P, I32, P, P, P, P, P, P, P]
    lib.rbs_pages_extend.restype = ctypes.c_int
    lib.rbs_pages_release.argtypes = [ctypes.POINTER(rbs_pages), P, P, P, P, P]
    lib.rbs_pages_release.restype = ctypes.c_int
    lib.rbs_qk_norm_rope.argtypes = [SP, SP, ctypes.POINTER(rbs_rope), P, P, P, P, P, P, ctypes.POINTER(rbs_cache), P, P]
    lib.rbs_qk_norm_rope.restype = ctypes.c_int
    lib.rbs_decode_workspace_bytes.argtypes = []
    lib.rbs_decode_workspace_bytes.restype = SZ
    lib.rbs_paged_decode.argtypes = [SP, ctypes.POINTER(rbs_cache), P, P, I32, P, F32, P, P, P, P]
    lib.rbs_paged_decode.restype = ctypes.c_int
    lib.rbs_paged_decode_packed.argtypes = [SP, ctypes.POINTER(rbs_cache), P, P, I32, P, I32, P, F32, P, P, P, P]
    lib.rbs_paged_decode_packed.restype = ctypes.c_int


def _handle(device: int, stream):
    # (The stream object that torch.cuda.current_stream() makes costs 2.7 us, as much as a launch.)
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else L._stream(stream)


def _on(device: int, stream, call, *args):
    """call(*args, stream handle) with `device` current: a launch goes to the
    current device, and the default stream is that device's."""
    if device == torch._C._cuda_getDevice():
        return call(*args, _handle(device, stream))
    with torch.cuda.device(device):
        return call(*args, _handle(device, stream))


def _elsewhere(dev: int, *tensors) -> bool:
    """Whether one of the tensors (None skipped) is not on GPU dev, or dev is none."""
    for x in tensors:
        if x is not None and x.get_device() != dev:
            return True
    return dev < 0


def _rows(name, t, sizes):
    """The strides of a bf16 (head, token, dimension) tensor of these sizes."""
    if isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.shape == sizes:
        strides = t.stride()
        if strides[2] == 1 and strides[0] and strides[1]:
            return strides[:2]
    return L._heads_tokens(name, t, *sizes)


def _int_row(name, t, n):
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.shape == (n,) and t.is_contiguous()):
        L._check_tensor(name, t, torch.int32, (n,))


def _strided(shape, q, kv=None):
    """L._with_strides, short where the shape leaves the strides to the tensors."""
    if shape.q_stride_head == shape.q_stride_tok == shape.kv_stride_head == shape.kv_stride_tok == 0:
        return L.rbs_shape(shape.n_tokens, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.block_size, *q,
                           *((0, 0) if kv is None else kv))
    return L._with_strides(shape, q=q, kv=kv)


def _one_dimensional(name, t, dtype, n=None):
    if isinstance(t, torch.Tensor) and t.dim() == 1 and n is None:
        n = t.numel()
    L._check_tensor(name, t, dtype, (n,) if n is not None else (-1,))


@dataclass(frozen=True, eq=False)
class PagedCache:
    """Keys and values of a paged cache: K and V [n_pages][H_kv][page_size][d]
    views of any strides the library takes (for [n_pages][page_size][H_kv][d]
    buffers, their transpose(1, 2)), bf16, or uint8 E4M3 codes with amax (fp32
    [2 H_kv]: the magnitudes of each K head, then each V head, that map to 448)."""
    K: torch.Tensor
    V: torch.Tensor
    amax: torch.Tensor | None = None
    c: rbs_cache = field(init=False, repr=False)
    device: int = field(init=False, repr=False)

    def __post_init__(self):
        K, V = self.K, self.V
        if not isinstance(K, torch.Tensor) or K.dim() != 4:
            raise ValueError("K must be a [n_pages][H_kv][page_size][d] tensor")
        dtype = torch.bfloat16 if self.amax is None else torch.uint8
        L._check_tensor("K", K, dtype, tuple(K.shape), contiguous=False)
        L._check_tensor("V", V, dtype, tuple(K.shape), contiguous=False)
        if V.stride() != K.stride():
            raise ValueError(f"V strides {V.stride()} differ from K strides {K.stride()}; the library takes one set")
        n_pages, hkv, page_size, d = K.shape
        if self.amax is not None:
            L._check_tensor("amax", self.amax, torch.float32, (2 * hkv,))
        s = K.stride()
        if K.numel() == 0 or min(s[i] for i in range(3) if K.shape[i] > 1 or i == 2) < d:
            raise ValueError(f"K's places overlap or it holds none (shape {tuple(K.shape)}, strides {s})")
        dev = L._on_gpu(("K", K), ("V", V), ("amax", self.amax))
        # A dimension of one page or head has no stride of its own.
        page, head = (s[i] if K.shape[i] > 1 else n for i, n in ((0, hkv * page_size * d), (1, page_size * d)))
        c = rbs_cache(n_pages, page_size, hkv, d, RBS_CACHE_BF16 if self.amax is None else RBS_CACHE_FP8, page, head,
                      s[2], K.data_ptr(), V.data_ptr(), L._ptr(self.amax))
        object.__setattr__(self, "c", c)
        object.__setattr__(self, "device", dev)

    @classmethod
    def allocate(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int = 128, amax=None,
                 device="cuda") -> "PagedCache":
        dtype = torch.bfloat16 if amax is None else torch.uint8
        K = torch.empty((n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device)
        return cls(K, torch.empty_like(K), amax)

    @property
    def page_size(self) -> int:
        return self.K.shape[2]


@dataclass(frozen=True, eq=False)
class Pages:
    """The bookkeeping of a cache's pages (int32 device tensors): the page table
    [n_rows][max_pages], the stack of free pages [n_pages] and how many it
    holds [1], the rows' lengths [n_rows] (negative: unused; a request is
    admitted to a row by setting its length to 0).  Calls that change them are
    ordered by the caller: threads that share a Pages take turns."""
    page_table: torch.Tensor
    free_pages: torch.Tensor
    n_free: torch.Tensor
    seq_lens: torch.Tensor
    page_size: int
    c: rbs_pages = field(init=False, repr=False)
    device: int = field(init=False, repr=False)
    state: tuple = field(init=False, repr=False)  # addresses of seq_lens and n_free

    def __post_init__(self):
        i32, table = torch.int32, self.page_table
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("page_table must be an [n_rows][max_pages] tensor")
        L._check_tensor("page_table", table, i32, tuple(table.shape))
        _one_dimensional("free_pages", self.free_pages, i32)
        L._check_tensor("n_free", self.n_free, i32, (1,))
        L._check_tensor("seq_lens", self.seq_lens, i32, (table.shape[0],))
        dev = L._on_gpu(("page_table", table), ("free_pages", self.free_pages), ("n_free", self.n_free),
                        ("seq_lens", self.seq_lens))
        object.__setattr__(self, "c", rbs_pages(table.shape[0], table.shape[1], self.free_pages.numel(),
                                                self.page_size, table.data_ptr(), self.free_pages.data_ptr()))
        object.__setattr__(self, "device", dev)
        object.__setattr__(self, "state", (self.seq_lens.data_ptr(), self.n_free.data_ptr()))

    @classmethod
    def allocate(cls, n_rows: int, max_pages: int, n_pages: int, page_size: int, device="cuda") -> "Pages":
        """Unused rows, every page free (page 0 on top of the stack)."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.zeros((n_rows, max_pages), **i32), torch.arange(n_pages - 1, -1, -1, **i32),
                   torch.full((1,), n_pages, **i32), torch.full((n_rows,), -1, **i32), page_size)

    @property
    def n_rows(self) -> int:
        return self.page_table.shape[0]


@dataclass(frozen=True, eq=False)
class PageStep:
    """Outputs of rbs_pages_extend (int32 device tensors)."""
    seq_lens: torch.Tensor   # [n_rows]
    n_free: torch.Tensor     # [1]
    cu_tokens: torch.Tensor  # [n_rows + 1]
    positions: torch.Tensor  # [max_tokens]
    slots: torch.Tensor      # [max_tokens]
    status: torch.Tensor     # [1]
    device: int = field(init=False, repr=False)
    max_tokens: int = field(init=False, repr=False)
    out: tuple = field(init=False, repr=False)  # the tensors' addresses

    def __post_init__(self):
        i32 = torch.int32
        _one_dimensional("step.seq_lens", self.seq_lens, i32)
        L._check_tensor("step.n_free", self.n_free, i32, (1,))
        L._check_tensor("step.cu_tokens", self.cu_tokens, i32, (self.seq_lens.numel() + 1,))
        _one_dimensional("step.positions", self.positions, i32)
        L._check_tensor("step.slots", self.slots, i32, (self.positions.numel(),))
        L._check_tensor("step.status", self.status, i32, (1,))
        object.__setattr__(self, "device", L._on_gpu(
            ("step.seq_lens", self.seq_lens), ("step.n_free", self.n_free), ("step.cu_tokens", self.cu_tokens),
            ("step.positions", self.positions), ("step.slots", self.slots), ("step.status", self.status)))
        object.__setattr__(self, "max_tokens", self.positions.numel())
        object.__setattr__(self, "out", tuple(t.data_ptr() for t in (
            self.seq_lens, self.n_free, self.cu_tokens, self.positions, self.slots, self.status)))

    @classmethod
    def allocate(cls, pages: Pages, max_tokens: int, in_place: bool = True) -> "PageStep":
        """in_place: the new lengths and n_free go into those of `pages`;
        otherwise into tensors of the step's own."""
        e = dict(dtype=torch.int32, device=pages.page_table.device)
        return cls(pages.seq_lens if in_place else torch.empty_like(pages.seq_lens),
                   pages.n_free if in_place else torch.empty_like(pages.n_free),
                   torch.empty(pages.n_rows + 1, **e), torch.empty(max_tokens, **e), torch.empty(max_tokens, **e),
                   torch.empty(1, **e))


def rbs_pages_extend(pages: Pages, new_tokens=None, max_tokens: int | None = None, step: PageStep | None = None,
                     stream=None) -> PageStep:
    """Pages, positions and slots for new_tokens[row] more tokens of every used
    row (None: one each).  step: the outputs; by default new ones for max_tokens
    tokens (the number of rows) with lengths and n_free updated in place."""
    if not isinstance(pages, Pages):
        raise ValueError("pages must be a Pages")
    if new_tokens is not None:
        L._check_tensor("new_tokens", new_tokens, torch.int32, (pages.page_table.shape[0],))
        if new_tokens.get_device() != pages.device:
            L._on_gpu(("page_table", pages.page_table), ("new_tokens", new_tokens))
    if step is None:
        step = L._made(pages.device, stream, PageStep.allocate, pages, pages.n_rows if max_tokens is None else max_tokens)
    else:
        if not isinstance(step, PageStep):
            raise ValueError("step must be a PageStep")
        if step.device != pages.device:
            raise ValueError(f"step is on cuda:{step.device}, pages on cuda:{pages.device}")
        if step.seq_lens.shape != pages.seq_lens.shape:
            raise ValueError(f"step is for {step.seq_lens.numel()} rows, pages has {pages.n_rows}")
        if max_tokens is not None and max_tokens != step.max_tokens:
            raise ValueError(f"max_tokens = {max_tokens} disagrees with the step's {step.max_tokens}")
    lens, n_free = pages.state
    L._check("rbs_pages_extend", _on(pages.device, stream, L.load().rbs_pages_extend, pages.c, lens,
                                     L._ptr(new_tokens), n_free, step.max_tokens, *step.out))
    return step


def rbs_pages_release(pages: Pages, released, status=None, stream=None) -> torch.Tensor:
    """The pages of the rows with released[row] != 0 (int32) back on the stack,
    their lengths -1; returns the status word."""
    if not isinstance(pages, Pages):
        raise ValueError("pages must be a Pages")
    L._check_tensor("released", released, torch.int32, (pages.n_rows,))
    if status is not None:
        L._check_tensor("status", status, torch.int32, (1,))
    L._on_gpu(("page_table", pages.page_table), ("released", released), ("status", status))
    if status is None:
        status = L._made(pages.device, stream, pages.n_free.new_empty, 1)
    L._check("rbs_pages_release", _on(pages.device, stream, L.load().rbs_pages_release, pages.c, released.data_ptr(),
                                      *pages.state, status.data_ptr()))
    return status


@dataclass(frozen=True, eq=False)
class Rope:
    """Norm and rotation of rbs_qk_norm_rope: inv_freq fp32 [rot_dim / 2] (None:
    no rotation), norm weights bf16 [d] (None: that tensor is not normed)."""
    inv_freq: torch.Tensor | None
    q_weight: torch.Tensor | None = None
    k_weight: torch.Tensor | None = None
    eps: float = 1e-6
    interleaved: bool = False
    factor: float = 1.0
    head_dim: int = 128
    c: rbs_rope = field(init=False, repr=False)
    device: int | None = field(init=False, repr=False)

    def __post_init__(self):
        if self.inv_freq is not None:
            _one_dimensional("inv_freq", self.inv_freq, torch.float32)
        for name in ("q_weight", "k_weight"):
            if getattr(self, name) is not None:
                L._check_tensor(name, getattr(self, name), torch.bfloat16, (self.head_dim,))
        rot = 0 if self.inv_freq is None else 2 * self.inv_freq.numel()
        dev = L._on_gpu(("inv_freq", self.inv_freq), ("q_weight", self.q_weight), ("k_weight", self.k_weight))
        object.__setattr__(self, "c", rbs_rope(L._ptr(self.q_weight), L._ptr(self.k_weight),
                                               L._ptr(self.inv_freq) if rot else None, rot, int(self.interleaved),
                                               float(self.eps), float(self.factor)))
        object.__setattr__(self, "device", dev)


def rope_frequencies(rot_dim: int = 128, base: float = 1.0e6, scaling: str | None = None, scale: float = 1.0,
                     original_tokens: int = 32768, fast: float = 32.0, slow: float = 1.0, device="cuda"):
    """(inv_freq, factor) of a Rope: base^(-2 j / rot_dim), j < rot_dim / 2, and 1.
    For contexts `scale` times longer than the original_tokens trained on:
      "linear"  every frequency divided by scale
      "parts"   by how many turns a pair makes over the original context: at
                least `fast` turns, kept; at most `slow`, divided by scale; in
                between, interpolated linearly over the pair's index; factor
                0.1 ln(scale) + 1 on queries and keys each (YaRN, Peng et al. 2023,
                Sec. 3.2 and 3.4, with whole indices as the ends of the interpolation)
    """
    if rot_dim < 2 or rot_dim % 2 != 0 or not base > 1 or not scale >= 1:
        raise ValueError("rot_dim must be even and positive, base past 1, scale at least 1")
    j = torch.arange(rot_dim // 2, dtype=torch.float64)
    f = base ** (-2 * j / rot_dim)
    factor = 1.0
    if scaling == "linear":
        f = f / scale
    elif scaling == "parts":
        if not fast > slow > 0:
            raise ValueError("fast and slow must be turns over the context with fast > slow > 0")

        def pair_of(turns):  # (real-valued) index of the pair that makes so many turns over the original context
            return rot_dim * math.log(original_tokens / (2 * math.pi * turns)) / (2 * math.log(base))

        low = max(math.floor(pair_of(fast)), 0)
        high = min(math.ceil(pair_of(slow)), rot_dim - 1)
        kept = 1 - ((j - low) / max(high - low, 1e-3)).clamp(0, 1)
        f = f * kept + f / scale * (1 - kept)
        factor = 0.1 * math.log(scale) + 1
    elif scaling is not None:
        raise ValueError(f"scaling must be None, 'linear' or 'parts', not {scaling!r}")
    return f.float().to(device), factor


def rbs_qk_norm_rope(shape: L.rbs_shape, rope: Rope, Q, K, positions, V=None, cache: PagedCache | None = None,
                     slots=None, Q_out=None, K_out=None, keep_k: bool = True, stream=None):
    """Queries and keys normed and rotated, keys and values put into the cache at
    `slots`; returns (Q_out, K_out).  Q_out and K_out may be Q and K.  By default
    they are new (K_out None with keep_k False, where only the cache needs it)."""
    if not isinstance(rope, Rope):
        raise ValueError("rope must be a Rope")
    hq, hkv, n, d = shape.n_q_heads, shape.n_kv_heads, shape.n_tokens, shape.head_dim
    q_sizes, k_sizes = (hq, n, d), (hkv, n, d)
    qs, ks = _rows("Q", Q, q_sizes), _rows("K", K, k_sizes)
    _int_row("positions", positions, n)
    if cache is not None:
        if not isinstance(cache, PagedCache):
            raise ValueError("cache must be a PagedCache")
        if V is None or slots is None:
            raise ValueError("a cache needs V and slots")
        vs = _rows("V", V, k_sizes)
        # (A stride over one head or one token is never used.)
        if vs != ks and ((vs[0] != ks[0] and hkv > 1) or (vs[1] != ks[1] and n > 1)):
            raise ValueError(f"V strides {vs} differ from K strides {ks}; the library takes one pair")
        _int_row("slots", slots, n)
    if Q_out is not None:
        _rows("Q_out", Q_out, q_sizes)
    if K_out is not None:
        _rows("K_out", K_out, k_sizes)
    dev = Q.get_device()
    if _elsewhere(dev, K, positions, Q_out, K_out) or (cache is not None and (
            cache.device != dev or _elsewhere(dev, V, slots))):
        L._on_gpu(("Q", Q), ("K", K), ("positions", positions), ("Q_out", Q_out), ("K_out", K_out),
                  *(() if cache is None else (("V", V), ("slots", slots), ("cache.K", cache.K))))
    if rope.device is not None and rope.device != dev:
        raise ValueError(f"rope is on cuda:{rope.device}, the other arguments on cuda:{dev}")
    if Q_out is None:
        # (Q's order of strides, without the gaps of a fused projection's view.)
        Q_out = L._made(dev, stream, torch.empty_like, Q)
    if K_out is None and keep_k:
        K_out = L._made(dev, stream, torch.empty_like, K)
    sh = _strided(shape, qs, ks)
    out = L.rbs_shape(n, hq, hkv, d, shape.block_size, *Q_out.stride()[:2],
                      *(ks if K_out is None else K_out.stride()[:2]))
    L._check("rbs_qk_norm_rope", _on(dev, stream, L.load().rbs_qk_norm_rope, sh, out, rope.c, Q.data_ptr(),
                                     K.data_ptr(), L._ptr(V), positions.data_ptr(), Q_out.data_ptr(), L._ptr(K_out),
                                     None if cache is None else cache.c, L._ptr(slots)))
    return Q_out, K_out


_decode_workspaces = threading.local()  # attributes of its own for every thread


def rbs_decode_workspace_bytes() -> int:
    return int(L.load().rbs_decode_workspace_bytes())


def _auto_workspace(device: int, handle: int) -> torch.Tensor:
    """The workspace of a (device, stream) and of this thread: a thread's calls on
    one stream are ordered, so they may share it.  Those of two threads are not: a
    call is two launches, and the other thread's may come between them.  While the
    stream is being captured, a new one, which belongs to the graph's memory:
    graphs that were captured on one stream may run side by side."""
    if handle != torch._C._cuda_getCurrentRawStream(device):
        # Made on the stream that uses it, whose order its memory's next use has to follow.
        with L._own(device, handle):
            return _workspace_of(device, handle)
    return _workspace_of(device, handle)


def _workspace_of(device: int, handle: int) -> torch.Tensor:
    capturing = torch.cuda.is_current_stream_capturing()
    held = _decode_workspaces.__dict__  # (freed with the thread; its memory's next use on the stream is ordered)
    ws = None if capturing else held.get((device, handle))
    if ws is None:
        ws = torch.empty(rbs_decode_workspace_bytes() // 4, dtype=torch.float32, device=torch.device("cuda", device))
        if not capturing:
            held[device, handle] = ws
    return ws


def rbs_paged_decode(shape: L.rbs_shape, Q, cache: PagedCache, page_table, seq_lens, softmax_scale: float = 0.0,
                     O=None, lse=None, stream=None, workspace=L.AUTO, cu_tokens=None):
    """Attention of one new token per row over the row's cached tokens; returns O
    (bf16, Q's sizes and strides).  Q: (head, row, dimension), a query for every
    row; or with cu_tokens, those of rbs_pages_extend's step, (head, token,
    dimension) as the step's tokens are packed: none of unused rows, and any behind
    the last one left alone."""
    hq, n, d = shape.n_q_heads, shape.n_tokens, shape.head_dim
    qs = _rows("Q", Q, (hq, n, d))
    if not isinstance(cache, PagedCache):
        raise ValueError("cache must be a PagedCache")
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an [n_rows][max_pages] tensor")
    rows = n if cu_tokens is None else page_table.shape[0]
    L._check_tensor("page_table", page_table, torch.int32, (rows, page_table.shape[1]))
    _int_row("seq_lens", seq_lens, rows)
    if cu_tokens is not None:
        _int_row("cu_tokens", cu_tokens, rows + 1)
    if O is not None:
        L._check_out(O, Q)
    if lse is not None:
        L._check_tensor("lse", lse, torch.float32, (hq, n))
    dev = Q.get_device()
    if cache.device != dev or _elsewhere(dev, page_table, seq_lens, O, lse, cu_tokens):
        L._on_gpu(("cache.K", cache.K), ("Q", Q), ("page_table", page_table), ("seq_lens", seq_lens), ("O", O),
                  ("lse", lse), ("cu_tokens", cu_tokens))
    if O is None:
        O = L._made(dev, stream, torch.empty_like, Q)
        if O.stride() != Q.stride():
            O = L._made(dev, stream, L._like_q, Q)
    if isinstance(workspace, str):
        if workspace != L.AUTO:
            raise ValueError(f"workspace must be AUTO or a tensor, not {workspace!r}")
    elif not isinstance(workspace, torch.Tensor) or workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError("workspace must be AUTO or a contiguous tensor on the inputs' GPU")
    elif workspace.numel() * workspace.element_size() < rbs_decode_workspace_bytes():
        raise ValueError("workspace is smaller than rbs_decode_workspace_bytes()")
    L._check("rbs_paged_decode", _on(dev, stream, _decode, _strided(shape, qs), cache, Q, page_table, seq_lens,
                                     softmax_scale, O, lse, workspace, cu_tokens, dev))
    return O


def _decode(shape, cache, Q, page_table, seq_lens, softmax_scale, O, lse, workspace, cu_tokens, dev, s):
    # (With the inputs' device current, which tells whether its stream is being captured.)
    ws = _auto_workspace(dev, s) if isinstance(workspace, str) else workspace
    rest = (page_table.data_ptr(), page_table.shape[1], seq_lens.data_ptr(), float(softmax_scale), O.data_ptr(),
            L._ptr(lse), ws.data_ptr(), s)
    if cu_tokens is None:
        return L.load().rbs_paged_decode(shape, cache.c, Q.data_ptr(), *rest)
    return L.load().rbs_paged_decode_packed(shape, cache.c, Q.data_ptr(), cu_tokens.data_ptr(), page_table.shape[0],
                                            *rest)
