"""Device-buffer plumbing around the decoder operators (PyTorch supplies memory and streams only): block tables of a paged cache, norm and
rotation of queries and keys into its 4-bit codes, attention over it, products in 8-bit floating point.

Every object enqueues on torch's current stream of its tensors' device.  An object that owns a workspace or results (BatchTables, CacheAttention,
Fp8Linear) serves one stream at a time, as ConvLayer does.  A call that needs more workspace than the object holds takes a new one; those that captured calls
use are kept as long as the object, which has to outlive the graph.  Arguments are checked (ValueError) and the calls made by the extension module _decoder; the
same calls under the C names are in binding.py."""
from __future__ import annotations

import ctypes
import os

import torch

from . import binding as B
from .layer import current_stream

B.lib()  # a missing librnswino.so is named as such
if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_decoder.so")):
    raise ImportError("paper_2007_12216_amd/_decoder.so is missing: build it with `python -m paper_2007_12216_amd.build` (or __graft_entry__.build())")
from . import _decoder  # noqa: E402


def _require_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("rnswino needs a GPU: there is no CPU execution path")


def _expect(t: torch.Tensor, name: str, dtype, shape, device=None) -> None:
    """A contiguous tensor of this dtype and shape on a GPU, on `device` if given."""
    if t.dtype is not dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or not t.is_cuda or t.device != (device or t.device):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device or 'the GPU'}, not {t.dtype} {tuple(t.shape)} on {t.device}")


class BatchTables:
    """Block tables and slot maps of a step (rnswino_block_tables): holds row_start, lens, slots, positions and needed for up to `n_tokens` packed rows."""

    def __init__(self, n_requests: int, n_tokens: int, page_size: int, device="cuda:0"):
        _require_gpu()
        self.n_requests, self.n_tokens, self.page_size, self.device = n_requests, n_tokens, page_size, torch.device(device)
        self.row_start = torch.empty(n_requests + 1, dtype=torch.int32, device=self.device)
        self.lens = torch.empty(n_requests, dtype=torch.int32, device=self.device)
        self.slots = torch.empty(n_tokens, dtype=torch.int64, device=self.device)
        self.positions = torch.empty(n_tokens, dtype=torch.int32, device=self.device)
        self.needed = torch.empty(1, dtype=torch.int32, device=self.device)

    def build(self, cached: torch.Tensor, fresh: torch.Tensor, free_pages: torch.Tensor, table: torch.Tensor) -> "BatchTables":
        """cached, fresh: int32 [n_requests]; free_pages: int32 [any]; table: int32 [n_requests][width], updated in place.  None of them may be one
        of the plan's own results: the next step's cached is a copy of lens."""
        _decoder.tables(cached, fresh, free_pages, table, self.row_start, self.lens, self.slots, self.positions, self.needed, self.page_size)
        return self


class Cache4:
    """A paged cache of keys and values in 4 bits (rnswino_cache4_t), new and zero or over given tensors (k, k_scale, v, v_scale)."""

    def __init__(self, pages: int, page_size: int, kv_heads: int, head_dim: int, device="cuda:0", tensors=None):
        _require_gpu()
        codes, scales = (pages, kv_heads, page_size, head_dim // 2), (pages, kv_heads, page_size, head_dim // 32)
        if tensors is None:
            tensors = tuple(torch.zeros(shape, dtype=torch.uint8, device=device) for shape in (codes, scales, codes, scales))
        self.k, self.k_scale, self.v, self.v_scale = tensors
        for t, name, shape in ((self.k, "k", codes), (self.k_scale, "k_scale", scales), (self.v, "v", codes), (self.v_scale, "v_scale", scales)):
            _expect(t, name, torch.uint8, shape, self.k.device if self.k.is_cuda else None)
        self.pages, self.page_size, self.kv_heads, self.head_dim, self.device = pages, page_size, kv_heads, head_dim, self.k.device
        self.desc = B.Cache4Desc(self.k.data_ptr(), self.k_scale.data_ptr(), self.v.data_ptr(), self.v_scale.data_ptr(), pages, page_size, kv_heads, head_dim)
        self.address = ctypes.addressof(self.desc)

    def read(self, slots: torch.Tensor, dtype=torch.bfloat16):
        """(keys, values) at `slots` (int64 [n]), each [n][kv_heads][head_dim], bfloat16 or float16."""
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError(f"dtype must be bfloat16 or float16, not {dtype}")
        return _decoder.read(self.address, slots, dtype is torch.float16, self.k)


class QKNormRope:
    """Norms of queries and keys per head and the position rotation in one pass, to memory (forward) or with the keys and values on into a Cache4 (append).

    angles: float32 [max_position][rotary], a row the cosines of its position's angles and then the sines.  wq, wk: [head_dim] of the rows' type, or None
    for no norm.  adjacent: rotate the pairs (2i, 2i + 1) instead of (i, i + rotary / 2)."""

    def __init__(self, q_heads: int, kv_heads: int, head_dim: int, angles: torch.Tensor, wq=None, wk=None, rotary: int | None = None, adjacent: bool = False, eps: float = 1e-6):
        _require_gpu()
        rotary = head_dim if rotary is None else rotary
        if rotary:
            _expect(angles, "angles", torch.float32, (angles.shape[0], rotary))
        for w, name in ((wq, "wq"), (wk, "wk")):
            if w is not None:
                _expect(w, name, w.dtype, (head_dim,))
        self.angles, self.wq, self.wk = angles, wq, wk
        self.desc = B.RopeDesc(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, rotary=rotary, adjacent=int(adjacent), max_position=angles.shape[0], eps=eps)
        self.address = ctypes.addressof(self.desc)

    def forward(self, qkv: torch.Tensor, positions: torch.Tensor):
        """qkv: rows of queries and keys, [n][(q_heads + kv_heads) * head_dim]; positions: int32 [n].  Returns (q, k), [n][heads][head_dim]."""
        return _decoder.rope(self.address, self.angles, self.wq, self.wk, qkv, positions)

    def append(self, qkv: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, cache: Cache4) -> torch.Tensor:
        """qkv: rows of queries, keys and values, [n][(q_heads + 2 kv_heads) * head_dim]; slots: int64 [n].  Keys and values go into `cache`; returns q."""
        return _decoder.append(self.address, self.angles, self.wq, self.wk, qkv, positions, slots, cache.address, cache.k)


class CacheAttention:
    """Attention of new tokens over a Cache4 (rnswino_cache4_attention); holds the workspace."""

    def __init__(self, cache: Cache4, q_heads: int, scale: float | None = None, window: int = 0):
        self.cache = cache
        self.desc = B.AttentionDesc(q_heads=q_heads, window=window, scale=cache.head_dim ** -0.5 if scale is None else scale)
        self.address, self.workspace, self.captured = ctypes.addressof(self.desc), None, []

    def forward(self, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, row_start: torch.Tensor, max_fresh: int = 0, max_len: int = 0,
                out: torch.Tensor | None = None) -> torch.Tensor:
        """q: [n][q_heads][head_dim], heads and dimensions contiguous; table: int32 [requests][width]; lens: int32 [requests]; row_start: int32 [requests + 1].
        max_fresh, max_len: bounds of a request's new tokens and length, 0 where not known.  max_fresh is a promise (the results of a request with more are right or NaN), max_len is for the
        choice of the launch only."""
        out, self.workspace = _decoder.attend(self.cache.address, self.address, q, table, lens, row_start, max_fresh, max_len, out, self.workspace, self.captured, self.cache.k)
        return out


class Fp8Linear:
    """y = x w^T in 8-bit floating point with a scale for each block of 128 (rnswino_fp8_linear); holds the workspace.

    codes: [outputs][128 * blocks] bytes (uint8 or float8_e4m3fn), zero behind `inputs`; scales: float32 [ceil(outputs / 128)][blocks]."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, inputs: int):
        _require_gpu()
        blocks = -(-inputs // 128)
        self.codes, self.scales, self.inputs, self.outputs = codes.view(torch.uint8), scales, inputs, codes.shape[0]
        _expect(self.codes, "codes", torch.uint8, (self.outputs, 128 * blocks))
        _expect(scales, "scales", torch.float32, (-(-self.outputs // 128), blocks), self.codes.device)
        self.workspace, self.captured = None, []

    @classmethod
    def from_weights(cls, w: torch.Tensor) -> "Fp8Linear":
        """Quantises w, bfloat16 or float16 [outputs][inputs]."""
        _require_gpu()
        types = {torch.bfloat16: B.TYPE_BF16, torch.float16: B.TYPE_F16}
        if w.dim() != 2 or w.dtype not in types or (w.shape[1] > 1 and w.stride(1) != 1) or not w.is_cuda:
            raise ValueError(f"w must be rows of contiguous bfloat16 or float16 on the GPU, not {w.dtype} {tuple(w.shape)} with strides {w.stride()} on {w.device}")
        outputs, inputs = w.shape
        blocks = -(-inputs // 128)
        codes = torch.empty((outputs, 128 * blocks), dtype=torch.uint8, device=w.device)
        scales = torch.empty((-(-outputs // 128), blocks), dtype=torch.float32, device=w.device)
        with torch.cuda.device(w.device):  # the library launches on the current device
            B.rnswino_fp8_quantize_weights(w, types[w.dtype], outputs, inputs, w.stride(0) if outputs > 1 else inputs, codes, scales, current_stream(w.device))
        return cls(codes, scales, inputs)

    def forward(self, x: torch.Tensor, y: torch.Tensor | None = None) -> torch.Tensor:
        """x: bfloat16 or float16 [n][inputs], rows contiguous.  Returns [n][outputs] of the same type."""
        y, self.workspace = _decoder.linear(self.codes, self.scales, self.inputs, x, y, self.workspace, self.captured)
        return y
