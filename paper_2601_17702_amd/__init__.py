"""Thin Python binding of libs3attn.so (C ABI in include/s3attn.h).

Argument marshalling only: every step of the path runs in the HIP kernels of the library.
PyTorch supplies device memory and the current stream.  There is no CPU fallback: if the
library is not built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libs3attn.so")
_lib = None

S3_BF16, S3_FP32 = 0, 1
MAX_K, MAX_FEAT = 128, 65536


class S3Error(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"s3attn error {code}: {msg}")
        self.code = code


# s3_kv_cache and s3_kv_batch of the header, packed into bytes (a call takes their address; a ctypes structure takes four times
# as long to fill)
_KV_CACHE, _KV_BATCH = struct.Struct("PPPiiiii4x"), struct.Struct("PPPqiiiii4x")
_KV8_CACHE, _KV_NORM = struct.Struct("PPPPiiii"), struct.Struct("PPqqf4x")         # s3_kv8_cache, s3_kv_norm


def lib():
    """Load the HIP library (built in-tree by paper_2601_17702_amd/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2601_17702_amd.build` "
                              "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, ci, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_int, C.c_size_t
        L.s3_last_error.restype = C.c_char_p
        L.s3_sae_encode_topk.argtypes = [vp, ci, ci, ci, vp, vp, ci, ci, ci, vp, vp, vp]
        L.s3_sae_encode_topk_workspace.argtypes = [ci, ci, ci, ci, ci, ci]
        L.s3_sae_encode_topk_workspace.restype = sz
        L.s3_sae_encode_topk_ws.argtypes = [vp, ci, ci, ci, vp, vp, ci, ci, ci, vp, vp, vp, sz, vp]
        L.s3_sae_encode_topk_ws.restype = ci
        L.s3_sae_encode_topk_stream.argtypes = [vp, ci, ci, ci, vp, vp, ci, ci, ci, vp, vp, vp, vp, sz, vp]
        L.s3_sae_encode_topk_stream_workspace.argtypes = [ci, ci]
        L.s3_sae_encode_topk_stream_workspace.restype = sz
        L.s3_index_create.argtypes = [ci, ci, ci, i64, C.POINTER(vp)]
        L.s3_index_destroy.argtypes = [vp]
        L.s3_index_destroy.restype = None
        L.s3_index_append.argtypes = [vp, vp, ci, vp, i32, vp]
        L.s3_index_finalize.argtypes = [vp, vp]
        L.s3_index_csr.argtypes = [vp, ci, C.POINTER(vp), C.POINTER(vp), C.POINTER(i64)]
        L.s3_index_export.argtypes = [vp, ci, vp, vp, vp]
        L.s3_index_export.restype = ci
        L.s3_index_reset.argtypes = [vp]
        L.s3_index_reset.restype = ci
        L.s3_index_tokens.argtypes = [vp]
        L.s3_index_tokens.restype = i64
        L.s3_index_build_workspace.argtypes = [ci, ci, ci]
        L.s3_index_build_workspace.restype = sz
        L.s3_index_build.argtypes = [vp, vp, ci, ci, ci, vp, vp, vp, sz, vp]
        L.s3_index_build_static.argtypes = [vp, vp, ci, ci, ci, vp, vp, vp]
        L.s3_index_build_static.restype = ci
        L.s3_coactivate_score_workspace.argtypes = [vp, i64]
        L.s3_coactivate_score_workspace.restype = sz
        L.s3_coactivate_score.argtypes = [vp, vp, vp, ci, i64, ci, ci, i32, ci, vp, vp, vp, vp, vp, sz, vp]
        L.s3_smoothing_kernel.argtypes = [ci, ci, vp]
        L.s3_smoothing_kernel.restype = ci
        L.s3_select_spans_workspace.argtypes = [i64]
        L.s3_select_spans_workspace.restype = sz
        L.s3_select_spans.argtypes = [vp, i64, vp, ci, ci, ci, C.c_float, ci, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.s3_select_spans.restype = ci
        L.s3_fuse_indices_workspace.argtypes = [i64]
        L.s3_fuse_indices_workspace.restype = sz
        L.s3_fuse_indices.argtypes = [i64, vp, vp, vp, ci, vp, i64, ci, ci, vp, vp, vp, vp, sz, vp]
        L.s3_fuse_indices.restype = ci
        L.s3_index_compact_bytes.argtypes = [vp]
        L.s3_index_compact_bytes.restype = sz
        L.s3_index_compact.argtypes = [vp, i32, vp, sz, C.POINTER(vp), vp]
        L.s3_index_compact.restype = ci
        L.s3_cindex_destroy.argtypes = [vp]
        L.s3_cindex_destroy.restype = None
        L.s3_cindex_info.argtypes = [vp, C.POINTER(ci), C.POINTER(i64)]
        L.s3_cindex_info.restype = ci
        L.s3_cindex_export.argtypes = [vp, ci, vp, vp, vp, vp]
        L.s3_cindex_export.restype = ci
        L.s3_coactivate_score_compact_workspace.argtypes = [vp, i64]
        L.s3_coactivate_score_compact_workspace.restype = sz
        L.s3_coactivate_score_compact.argtypes = [vp, vp, vp, ci, i64, ci, ci, i32, ci, vp, vp, vp, vp, vp, sz, vp]
        L.s3_coactivate_score_compact.restype = ci
        L.s3_sae_train_workspace.argtypes = [ci, ci, ci, ci]
        L.s3_sae_train_workspace.restype = sz
        cf = C.c_float
        L.s3_sae_train_step.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, vp, cf, cf, cf, cf, ci, vp, vp, vp, vp, sz, vp]
        L.s3_sae_train_step.restype = ci
        L.s3_rope_table.argtypes = [vp, i64, ci, C.c_double, vp]
        L.s3_rope_table.restype = ci
        L.s3_kv_append.argtypes = [vp, vp, vp, i64, i64, vp, i64, i64, vp, i64, ci, ci, vp, vp, ci, i64, i64, vp, vp]
        L.s3_kv_append.restype = ci
        L.s3_paged_attention_workspace.argtypes = [vp, vp, ci]
        L.s3_paged_attention_workspace.restype = sz
        L.s3_paged_attention.argtypes = [vp, vp, vp, ci, i64, i64, cf, ci, vp, vp, vp, sz, vp]
        L.s3_paged_attention.restype = ci
        L.s3_block_tiles.argtypes = [vp, ci]
        L.s3_block_tiles.restype = i64
        L.s3_block_select_workspace.argtypes = [vp, vp, ci, ci, ci]
        L.s3_block_select_workspace.restype = sz
        L.s3_block_select.argtypes = [vp, vp, vp, ci, i64, i64, ci, ci, ci, ci, vp, vp, sz, vp]
        L.s3_block_select.restype = ci
        L.s3_block_attention_workspace.argtypes = [vp, vp, ci, ci, ci]
        L.s3_block_attention_workspace.restype = sz
        L.s3_block_attention.argtypes = [vp, vp, vp, ci, i64, i64, vp, ci, ci, cf, vp, vp, vp, sz, vp]
        L.s3_block_attention.restype = ci
        for name in ("s3_kv_append_norm", "s3_kv8_append"):
            getattr(L, name).argtypes = [vp, vp, vp, i64, i64, vp, i64, i64, vp, i64, ci, ci, vp, vp, ci, i64, i64, vp, vp, vp]
        for name in ("s3_paged_attention_capped", "s3_kv8_attention"):
            getattr(L, name).argtypes = [vp, vp, vp, ci, i64, i64, cf, cf, ci, vp, vp, vp, sz, vp]
        for name in ("s3_block_attention_capped", "s3_kv8_block_attention"):
            getattr(L, name).argtypes = [vp, vp, vp, ci, i64, i64, vp, ci, ci, cf, cf, vp, vp, vp, sz, vp]
        for name in ("s3_kv_read", "s3_kv8_read"):
            getattr(L, name).argtypes = [vp, vp, vp, vp, vp, vp]
        L.s3_kv8_attention_workspace.argtypes = [vp, vp, ci]
        L.s3_kv8_attention_workspace.restype = sz
        L.s3_kv8_block_attention_workspace.argtypes = [vp, vp, ci, ci, ci]
        L.s3_kv8_block_attention_workspace.restype = sz
        for name in ("s3_sae_encode_topk", "s3_sae_encode_topk_stream", "s3_index_create", "s3_index_append", "s3_index_finalize",
                     "s3_index_csr", "s3_index_build", "s3_coactivate_score"):
            getattr(L, name).restype = ci
        _lib = L
    return _lib


def _check(rc: int):
    if rc != 0:
        raise S3Error(rc, lib().s3_last_error().decode())


_raw_stream = None


def _stream():
    """The current stream's handle.  torch.cuda.current_stream() builds a Stream object around it, 3.2 us a call; the two
    calls it makes itself take 0.2."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        if not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        _raw_stream = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
    stream, device = _raw_stream
    return stream(device())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return S3_BF16
    if t.dtype == torch.float32:
        return S3_FP32
    raise TypeError(f"x must be bfloat16 or float32, got {t.dtype}")


def sae_encode_topk(x, w_enc, b_enc, k: int, ids=None, vals=None):
    """x [n_heads, T, d_head], w_enc [n_heads, n_feat, d_head] (same dtype), b_enc [n_heads, n_feat] fp32,
    all on the GPU and contiguous.  Returns (ids int32 [n_heads, T, k], vals fp32 [n_heads, T, k])."""
    import torch
    assert x.is_cuda and x.is_contiguous() and w_enc.is_contiguous() and b_enc.is_contiguous()
    assert x.dim() == 3 and w_enc.dim() == 3 and b_enc.dim() == 2
    n_heads, T, d = x.shape
    n_feat = w_enc.shape[1]
    assert w_enc.shape == (n_heads, n_feat, d) and b_enc.shape == (n_heads, n_feat)
    assert w_enc.dtype == x.dtype and b_enc.dtype == torch.float32
    if ids is None:
        ids = torch.empty((n_heads, T, k), dtype=torch.int32, device=x.device)
    if vals is None:
        vals = torch.empty((n_heads, T, k), dtype=torch.float32, device=x.device)
    assert ids.is_contiguous() and vals.is_contiguous() and ids.dtype == torch.int32 and vals.dtype == torch.float32
    assert ids.numel() == n_heads * T * k and vals.numel() == n_heads * T * k
    dt = _dtype_code(x)
    need = int(lib().s3_sae_encode_topk_workspace(dt, T, d, n_feat, k, n_heads))
    ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None     # the caching allocator's, stream-ordered
    _check(lib().s3_sae_encode_topk_ws(_ptr(x), dt, T, d, _ptr(w_enc), _ptr(b_enc), n_feat, k, n_heads,
                                       _ptr(ids), _ptr(vals), _ptr(ws), need, _stream()))
    return ids, vals


def new_tau_hint(n_heads: int, device="cuda"):
    """Carried thresholds of a stream before its first chunk: [n_heads, 2] fp32 filled with -inf."""
    import torch
    return torch.full((n_heads, 2), float("-inf"), dtype=torch.float32, device=device)


def sae_encode_topk_stream_workspace(n_heads: int, T: int) -> int:
    return int(lib().s3_sae_encode_topk_stream_workspace(n_heads, T))


def sae_encode_topk_stream(x, w_enc, b_enc, k: int, tau_hint, ws=None, ids=None, vals=None):
    """sae_encode_topk for the chunks of one stream: tau_hint [n_heads, 2] fp32 (new_tau_hint) is read and updated;
    the results are the same as sae_encode_topk's whatever it holds."""
    import torch
    assert x.is_cuda and x.is_contiguous() and w_enc.is_contiguous() and b_enc.is_contiguous()
    assert x.dim() == 3 and w_enc.dim() == 3 and b_enc.dim() == 2
    n_heads, T, d = x.shape
    n_feat = w_enc.shape[1]
    assert w_enc.shape == (n_heads, n_feat, d) and b_enc.shape == (n_heads, n_feat)
    assert w_enc.dtype == x.dtype and b_enc.dtype == torch.float32
    assert tau_hint.is_cuda and tau_hint.is_contiguous() and tau_hint.dtype == torch.float32
    assert tau_hint.numel() == 2 * n_heads
    need = sae_encode_topk_stream_workspace(n_heads, T)
    if ws is None:
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=x.device)
    assert ws.numel() >= need
    if ids is None:
        ids = torch.empty((n_heads, T, k), dtype=torch.int32, device=x.device)
    if vals is None:
        vals = torch.empty((n_heads, T, k), dtype=torch.float32, device=x.device)
    assert ids.is_contiguous() and vals.is_contiguous() and ids.dtype == torch.int32 and vals.dtype == torch.float32
    assert ids.numel() == n_heads * T * k and vals.numel() == n_heads * T * k
    _check(lib().s3_sae_encode_topk_stream(_ptr(x), _dtype_code(x), T, d, _ptr(w_enc), _ptr(b_enc), n_feat, k, n_heads,
                                           _ptr(ids), _ptr(vals), _ptr(tau_hint), _ptr(ws), ws.numel(), _stream()))
    return ids, vals


class Index:
    """n_heads inverted indexes (feature -> positions) living on the GPU (s3_index_* calls)."""

    def __init__(self, n_heads: int, n_feat: int, k: int, max_tokens: int):
        h = C.c_void_p()
        _check(lib().s3_index_create(n_heads, n_feat, k, max_tokens, C.byref(h)))
        self._h = h
        self.n_heads, self.n_feat, self.k, self.max_tokens = n_heads, n_feat, k, max_tokens

    def append(self, ids, positions=None, base_pos: int = 0):
        import torch
        assert ids.is_cuda and ids.is_contiguous() and ids.dtype == torch.int32 and ids.dim() == 3
        assert ids.shape[0] == self.n_heads and ids.shape[2] == self.k
        if positions is not None:
            assert positions.is_cuda and positions.dtype == torch.int32 and positions.numel() == ids.shape[1]
        _check(lib().s3_index_append(self._h, _ptr(ids), ids.shape[1], _ptr(positions), base_pos, _stream()))

    def finalize(self):
        _check(lib().s3_index_finalize(self._h, _stream()))

    def reset(self):
        _check(lib().s3_index_reset(self._h))

    @property
    def tokens(self) -> int:
        return int(lib().s3_index_tokens(self._h))

    def csr(self, head: int):
        """Copies of one head's (offsets [n_feat + 1], positions [P]) as torch int32 tensors."""
        import torch
        off, pos, n = C.c_void_p(), C.c_void_p(), C.c_int64()
        _check(lib().s3_index_csr(self._h, head, C.byref(off), C.byref(pos), C.byref(n)))
        o = torch.empty(self.n_feat + 1, dtype=torch.int32, device="cuda")
        p = torch.empty(n.value, dtype=torch.int32, device="cuda")
        _check(lib().s3_index_export(self._h, head, _ptr(o), _ptr(p) if n.value else None, _stream()))
        return o, p

    def csr_offsets(self, head: int):
        """Copy of one head's offsets [n_feat + 1] only."""
        import torch
        o = torch.empty(self.n_feat + 1, dtype=torch.int32, device="cuda")
        _check(lib().s3_index_export(self._h, head, _ptr(o), None, _stream()))
        return o

    def score_workspace(self, n_positions: int) -> int:
        return int(lib().s3_coactivate_score_workspace(self._h, n_positions))

    def coactivate_score(self, qids, qvals, n_positions: int, span_len: int, top_b: int, max_freq: int = 0,
                         nms: bool = True, want_scores: bool = False, ws=None):
        """Returns (span_start int32 [top_b], span_score fp32 [top_b], n_found int32 [1], scores fp32 [L] | None)."""
        import torch
        assert qids.is_cuda and qids.is_contiguous() and qvals.is_contiguous()
        assert qids.dtype == torch.int32 and qvals.dtype == torch.float32 and qids.dim() == 3
        assert qids.shape[0] == self.n_heads and qids.shape[2] == self.k and qvals.shape == qids.shape
        dev = qids.device
        if ws is None:
            ws = torch.empty(self.score_workspace(n_positions), dtype=torch.uint8, device=dev)
        starts = torch.empty(top_b, dtype=torch.int32, device=dev)
        scores = torch.empty(top_b, dtype=torch.float32, device=dev)
        found = torch.empty(1, dtype=torch.int32, device=dev)
        S = torch.empty(n_positions, dtype=torch.float32, device=dev) if want_scores else None
        _check(lib().s3_coactivate_score(self._h, _ptr(qids), _ptr(qvals), qids.shape[1], n_positions, span_len,
                                         top_b, max_freq, int(bool(nms)), _ptr(S), _ptr(starts), _ptr(scores),
                                         _ptr(found), _ptr(ws), ws.numel(), _stream()))
        return starts, scores, found, S

    def compact(self, prune_freq: int = 0):
        """s3_index_compact: the compact form of this (finalized) index in a buffer of its own."""
        return CompactIndex(self, prune_freq)

    def destroy(self):
        if getattr(self, "_h", None) and lib is not None:    # module globals are gone at interpreter shutdown
            lib().s3_index_destroy(self._h)
            self._h = None

    def __del__(self):
        self.destroy()


class CompactIndex:
    """Compact form of a finalized Index (s3_index_compact): 16-bit block-relative postings in block-major order, a
    segment table, optional stop-feature pruning.  Owns its buffer; independent of the Index it was built from."""

    def __init__(self, index: "Index", prune_freq: int = 0):
        import torch
        need = int(lib().s3_index_compact_bytes(index._h))
        self.buf = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        h = C.c_void_p()
        _check(lib().s3_index_compact(index._h, prune_freq, _ptr(self.buf), self.buf.numel(), C.byref(h), _stream()))
        self._h = h
        self.n_heads, self.n_feat, self.k = index.n_heads, index.n_feat, index.k
        nb, mp = C.c_int(), C.c_int64()
        _check(lib().s3_cindex_info(self._h, C.byref(nb), C.byref(mp)))
        self.n_blocks, self.max_postings = nb.value, mp.value
        self.nbytes = need

    def arrays(self, head: int):
        """Copies of one head's (cstart int32 [n_blocks * n_feat + 1], delta int16-view-of-uint16 [kept], cfreq [n_feat])."""
        import torch
        cs = torch.empty(self.n_blocks * self.n_feat + 1, dtype=torch.int32, device="cuda")
        de = torch.empty(max(self.max_postings, 1), dtype=torch.int16, device="cuda")
        cf = torch.empty(self.n_feat, dtype=torch.int32, device="cuda")
        _check(lib().s3_cindex_export(self._h, head, _ptr(cs), _ptr(de), _ptr(cf), _stream()))
        torch.cuda.synchronize()
        return cs, de[: int(cs[-1].item())], cf

    def score_workspace(self, n_positions: int) -> int:
        return int(lib().s3_coactivate_score_compact_workspace(self._h, n_positions))

    def coactivate_score(self, qids, qvals, n_positions: int, span_len: int, top_b: int, max_freq: int = 0,
                         nms: bool = True, want_scores: bool = False, ws=None):
        """As Index.coactivate_score, reading the compact index."""
        import torch
        assert qids.is_cuda and qids.is_contiguous() and qvals.is_contiguous()
        assert qids.dtype == torch.int32 and qvals.dtype == torch.float32 and qids.dim() == 3
        assert qids.shape[0] == self.n_heads and qids.shape[2] == self.k and qvals.shape == qids.shape
        dev = qids.device
        if ws is None:
            ws = torch.empty(self.score_workspace(n_positions), dtype=torch.uint8, device=dev)
        starts = torch.empty(top_b, dtype=torch.int32, device=dev)
        scores = torch.empty(top_b, dtype=torch.float32, device=dev)
        found = torch.empty(1, dtype=torch.int32, device=dev)
        S = torch.empty(n_positions, dtype=torch.float32, device=dev) if want_scores else None
        _check(lib().s3_coactivate_score_compact(self._h, _ptr(qids), _ptr(qvals), qids.shape[1], n_positions, span_len,
                                                 top_b, max_freq, int(bool(nms)), _ptr(S), _ptr(starts), _ptr(scores),
                                                 _ptr(found), _ptr(ws), ws.numel(), _stream()))
        return starts, scores, found, S

    def destroy(self):
        if getattr(self, "_h", None) and lib is not None:
            lib().s3_cindex_destroy(self._h)
            self._h = None

    def __del__(self):
        self.destroy()


def index_build(ids, n_feat: int, positions=None):
    """One-shot CSR of a single index: ids [T, k] int32 -> (offsets [n_feat + 1], positions [T * k])."""
    import torch
    assert ids.is_cuda and ids.is_contiguous() and ids.dtype == torch.int32 and ids.dim() == 2
    T, k = ids.shape
    need = int(lib().s3_index_build_workspace(T, k, n_feat))
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device=ids.device)
    off = torch.empty(n_feat + 1, dtype=torch.int32, device=ids.device)
    pos = torch.empty(T * k, dtype=torch.int32, device=ids.device)
    _check(lib().s3_index_build(_ptr(ids), _ptr(positions), T, k, n_feat, _ptr(off), _ptr(pos), _ptr(ws),
                                ws.numel(), _stream()))
    return off, pos


STATIC_SCRATCH_BYTES = 16 << 20


def index_build_static(ids, n_feat: int, off, pos, positions=None):
    """s3_index_build_static: one-shot CSR into the caller's off [n_feat + 1] / pos [T * k]; allocates nothing."""
    import torch
    assert ids.is_cuda and ids.is_contiguous() and ids.dtype == torch.int32 and ids.dim() == 2
    T, k = ids.shape
    assert off.is_cuda and off.dtype == torch.int32 and off.numel() >= n_feat + 1 and off.is_contiguous()
    assert pos.is_cuda and pos.dtype == torch.int32 and pos.numel() >= T * k and pos.is_contiguous()
    _check(lib().s3_index_build_static(_ptr(ids), _ptr(positions), T, k, n_feat, _ptr(off), _ptr(pos), _stream()))
    return off, pos


KERNEL_BOX, KERNEL_TRIANGULAR, KERNEL_GAUSSIAN = 0, 1, 2


def smoothing_kernel(kind: int, K: int):
    """Weights of a smoothing kernel (s3_smoothing_kernel, computed by the library on the host) as a float32 GPU tensor."""
    import torch
    host = (C.c_float * K)()
    _check(lib().s3_smoothing_kernel(kind, K, host))
    return torch.tensor(list(host), dtype=torch.float32).cuda()


def select_spans(scores, kernel, n_centers: int, nms_radius: int, rel_threshold: float, max_half_len: int,
                 want_density: bool = False):
    """s3_select_spans: scores [L] fp32, kernel [K] fp32 (GPU).  Returns (center, center_density, span_lo, span_hi,
    n_found, density | None)."""
    import torch
    assert scores.is_cuda and scores.is_contiguous() and scores.dtype == torch.float32 and scores.dim() == 1
    assert kernel.is_cuda and kernel.is_contiguous() and kernel.dtype == torch.float32 and kernel.dim() == 1
    L, dev = scores.numel(), scores.device
    ws = torch.empty(max(int(lib().s3_select_spans_workspace(L)), 1), dtype=torch.uint8, device=dev)
    center = torch.empty(n_centers, dtype=torch.int32, device=dev)
    dens_c = torch.empty(n_centers, dtype=torch.float32, device=dev)
    lo = torch.empty(n_centers, dtype=torch.int32, device=dev)
    hi = torch.empty(n_centers, dtype=torch.int32, device=dev)
    found = torch.empty(1, dtype=torch.int32, device=dev)
    D = torch.empty(L, dtype=torch.float32, device=dev) if want_density else None
    _check(lib().s3_select_spans(_ptr(scores), L, _ptr(kernel), kernel.numel(), n_centers, nms_radius, rel_threshold,
                                 max_half_len, _ptr(D), _ptr(center), _ptr(dens_c), _ptr(lo), _ptr(hi), _ptr(found),
                                 _ptr(ws), ws.numel(), _stream()))
    return center, dens_c, lo, hi, found, D


def fuse_indices(n_positions: int, span_lo, span_hi, n_spans, extra=None, lead: int = 0, tail: int = 0):
    """s3_fuse_indices: returns (mask uint8 [L], idx int32 [L], n_out int32 [1]); n_spans is a GPU int32 [1] or None."""
    import torch
    dev = span_lo.device
    ws = torch.empty(max(int(lib().s3_fuse_indices_workspace(n_positions)), 1), dtype=torch.uint8, device=dev)
    mask = torch.empty(n_positions, dtype=torch.uint8, device=dev)
    idx = torch.empty(n_positions, dtype=torch.int32, device=dev)
    n_out = torch.empty(1, dtype=torch.int32, device=dev)
    assert span_lo.dtype == torch.int32 and span_hi.dtype == torch.int32 and span_lo.numel() == span_hi.numel()
    if extra is not None:
        assert extra.is_cuda and extra.dtype == torch.int32 and extra.is_contiguous()
    _check(lib().s3_fuse_indices(n_positions, _ptr(span_lo), _ptr(span_hi), _ptr(n_spans), span_lo.numel(), _ptr(extra),
                                 0 if extra is None else extra.numel(), lead, tail, _ptr(mask), _ptr(idx), _ptr(n_out),
                                 _ptr(ws), ws.numel(), _stream()))
    return mask, idx, n_out


class SaeTrainer:
    """Parameters, Adam moments and workspace of one Top-K SAE on the GPU; step(x) is one s3_sae_train_step.
    w_enc, w_dec [n_feat, d] / b_enc [n_feat] / b_dec [d]: float32 GPU tensors, updated in place."""

    def __init__(self, w_enc, b_enc, w_dec, b_dec, k: int, batch: int, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8):
        import torch
        for t in (w_enc, b_enc, w_dec, b_dec):
            assert t.is_cuda and t.is_contiguous() and t.dtype == torch.float32
        self.n_feat, self.d = w_enc.shape
        assert w_dec.shape == w_enc.shape and b_enc.shape == (self.n_feat,) and b_dec.shape == (self.d,)
        self.w_enc, self.b_enc, self.w_dec, self.b_dec = w_enc, b_enc, w_dec, b_dec
        self.k, self.batch, self.hyper, self.steps = k, batch, (lr, beta1, beta2, eps), 0
        self.P = 2 * self.n_feat * self.d + self.n_feat + self.d
        self.m = torch.zeros(self.P, dtype=torch.float32, device=w_enc.device)
        self.v = torch.zeros_like(self.m)
        need = int(lib().s3_sae_train_workspace(batch, self.d, self.n_feat, k))
        if need == 0:
            raise S3Error(1, f"s3_sae_train_workspace: shape not supported (batch {batch}, d {self.d}, n_feat {self.n_feat}, k {k})")
        self.ws = torch.empty(need, dtype=torch.uint8, device=w_enc.device)
        self.loss = torch.empty(1, dtype=torch.float32, device=w_enc.device)

    def step(self, x, want_ids=False, want_grads=False):
        """x [batch, d] float32 on the GPU.  Returns (loss tensor [1], ids or None, grads [P] or None)."""
        import torch
        assert x.is_cuda and x.is_contiguous() and x.dtype == torch.float32 and x.shape == (self.batch, self.d)
        ids = torch.empty((self.batch, self.k), dtype=torch.int32, device=x.device) if want_ids else None
        grads = torch.empty(self.P, dtype=torch.float32, device=x.device) if want_grads else None
        self.steps += 1
        lr, b1, b2, eps = self.hyper
        _check(lib().s3_sae_train_step(_ptr(x), self.batch, self.d, self.n_feat, self.k, _ptr(self.w_enc), _ptr(self.b_enc),
                                       _ptr(self.w_dec), _ptr(self.b_dec), _ptr(self.m), _ptr(self.v), lr, b1, b2, eps,
                                       self.steps, _ptr(self.loss), _ptr(ids), _ptr(grads), _ptr(self.ws), self.ws.numel(),
                                       _stream()))
        return self.loss, ids, grads


def _torch():
    """torch, imported on the first use of the cache and not with the package."""
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


_torch_module = None


def rope_table(n_pos: int, rot_dim: int, theta: float = 10000.0, device="cuda"):
    """s3_rope_table: cos | sin of positions 0 .. n_pos - 1, [n_pos, rot_dim] fp32."""
    import torch
    t = torch.empty((n_pos, rot_dim), dtype=torch.float32, device=device)
    _check(lib().s3_rope_table(_ptr(t), n_pos, rot_dim, theta, _stream()))
    return t


class KVCache:
    """Keys and values of many sequences in pages (s3_kv_cache), and the calls around them.  With E elements in 16 bytes:
    k [n_pages, n_kv_heads, d_head / E, page_size, E], v [n_pages, n_kv_heads, page_size / E, d_head, E] in bfloat16 or float32,
    sig [n_pages, n_kv_heads, d_head] bfloat16 (signatures, for select) or None.  The tensors are allocated here unless given.

    Arguments that the calls share: kv_len [n_seq] int32, the sequences' lengths with the new tokens counted; block_table
    [n_seq, max_pages] int32, page numbers; q_start [n_seq + 1] int32, rows of the new tokens (None: one per sequence); max_new and
    max_kv, bounds of the new tokens and of kv_len that the host knows (they share out the work; give max_new with q_start, without it
    a batch of single tokens is planned as if chunks were among them, with their launch and workspace).  Arrays of rows are [n_tokens, heads, d_head],
    the last axis contiguous, the others of any stride that is a multiple of 16 bytes.  ws: scratch of a call, uint8 of the size that the library's
    ..._workspace names for this very call (a smaller batch may take more: s3_paged_attention in the header says which size is enough for all); None: allocated here."""

    _eight = False            # whether the cache is one of 8 bits

    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, d_head: int, dtype=None, signatures: bool = False,
                 device="cuda", k=None, v=None, sig=None):
        import torch
        dtype = dtype or torch.bfloat16
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError(f"dtype must be bfloat16 or float32, got {dtype}")
        e = 16 // dtype.itemsize
        shapes = {"k": (n_pages, n_kv_heads, d_head // e, page_size, e), "v": (n_pages, n_kv_heads, page_size // e, d_head, e),
                  "sig": (n_pages, n_kv_heads, d_head)}

        def array(name, t, dt):
            if t is None:
                return torch.empty(shapes[name], dtype=dt, device=device)
            assert t.is_cuda and t.is_contiguous() and t.dtype == dt and tuple(t.shape) == shapes[name], name
            return t
        self.k, self.v = array("k", k, dtype), array("v", v, dtype)
        self.sig = array("sig", sig, torch.bfloat16) if signatures or sig is not None else None
        lib()
        self.scale = d_head ** -0.5
        self.dtype, self.page_size, self.n_kv_heads, self.d_head, self.n_pages = dtype, page_size, n_kv_heads, d_head, n_pages
        self._c = self._c16 = _KV_CACHE.pack(_ptr(self.k), _ptr(self.v), _ptr(self.sig) or 0, _dtype_code(self.k), n_pages, page_size, n_kv_heads, d_head)

    # These run before every launch: as few attribute reads as the checks allow.
    def _batch(self, n_tokens, kv_len, block_table, q_start, max_new, max_kv):
        i32 = kv_len.dtype
        n_seq, = kv_len.shape
        rows, width = block_table.shape
        stride, inner = block_table.stride()
        assert i32 is _torch().int32 and block_table.dtype is i32 and kv_len.is_cuda and block_table.is_cuda
        assert rows == n_seq and (inner == 1 or width <= 1) and (stride >= width or rows <= 1) and kv_len.is_contiguous()
        qs = 0
        if q_start is not None:
            assert q_start.dtype is i32 and q_start.is_cuda and q_start.shape == (n_seq + 1,) and q_start.is_contiguous()
            qs = q_start.data_ptr()
        else:
            assert n_tokens == n_seq
            max_new = 1
        return _KV_BATCH.pack(qs, kv_len.data_ptr(), block_table.data_ptr(), stride if rows > 1 else width, n_seq, n_tokens, width,
                              n_tokens if max_new is None else max_new, width * self.page_size if max_kv is None else max_kv)

    def _rows(self, x, tokens, heads=None):
        T, n, d = x.shape
        ts, hs, inner = x.stride()
        assert x.dtype is self.dtype and x.is_cuda and d == self.d_head and inner == 1 and T == tokens and (heads is None or n == heads)
        return x.data_ptr(), ts, hs, n

    def _weights(self, w, heads):
        """A norm's weights, [d_head] for all heads or [heads, d_head]: address, and from head to head."""
        if w is None:
            return 0, 0
        d = self.d_head
        each = w.dim() == 2
        assert w.is_cuda and w.dtype is _torch().float32 and w.is_contiguous() and w.shape == ((heads, d) if each else (d,))
        return w.data_ptr(), d if each else 0

    def append(self, k, v, kv_len, block_table, q_start=None, rope=None, interleaved: bool = False, positions=None, q=None, q_out=None,
               max_new=None, q_norm=None, k_norm=None, eps: float = 1e-6):
        """s3_kv_append: k, v [n_tokens, n_kv_heads, d_head] into their pages, keys (and q) rotated by rope (rope_table) first.  With q_norm
        or k_norm (fp32 weights, [d_head] or [heads, d_head]) s3_kv_append_norm: rows over the root of their mean square plus eps, before the
        rotation.  Returns the rotated q, or None without q."""
        T = k.shape[0]
        kp, kt, kh, heads = self._rows(k, T, self.n_kv_heads)
        vp, vt, vh, _ = self._rows(v, T, heads)
        b = self._batch(T, kv_len, block_table, q_start, max_new, None)
        rp = n_pos = rot = n_q = qp = qt = qh = op = 0
        if rope is not None:
            n_pos, rot = rope.shape
            assert rope.is_cuda and rope.is_contiguous() and rope.dtype is _torch().float32
            rp = rope.data_ptr()
        if positions is not None:
            assert positions.is_cuda and positions.is_contiguous() and positions.dtype is kv_len.dtype and positions.shape == (T,)
        if q is not None:
            qp, qt, qh, n_q = self._rows(q, T)
            if q_out is None:
                q_out = _torch().empty_like(q, memory_format=_torch().contiguous_format)
            else:
                assert q_out.shape == q.shape and q_out.dtype is q.dtype and q_out.is_contiguous() and q_out.is_cuda
            op = q_out.data_ptr()
        norm = None
        if q_norm is not None or k_norm is not None:
            assert q_norm is None or q is not None
            (qw, qs), (kw, ks) = self._weights(q_norm, n_q), self._weights(k_norm, heads)
            norm = _KV_NORM.pack(qw, kw, qs, ks, eps)
        args = self._c, b, kp, kt, kh, vp, vt, vh, rp, n_pos, rot, interleaved, _ptr(positions), qp, n_q, qt, qh, op
        if self._eight:
            rc = _lib.s3_kv8_append(*args, norm, _stream())
        else:
            rc = _lib.s3_kv_append(*args, _stream()) if norm is None else _lib.s3_kv_append_norm(*args, norm, _stream())
        if rc:
            _check(rc)
        return q_out

    def read(self, kv_len, block_table, n_rows: int, q_start=None, positions=None, k_out=None, v_out=None):
        """s3_kv_read: tokens back as rows.  Rows q_start[s] .. q_start[s + 1] - 1 (None: row s) are those of sequence s at `positions`
        [n_rows] int32, or without them its last ones, as append would store them.  Returns (k, v) [n_rows, n_kv_heads, d_head]."""
        torch = _torch()
        b = self._batch(n_rows, kv_len, block_table, q_start, None, None)
        if positions is not None:
            assert positions.is_cuda and positions.is_contiguous() and positions.dtype is torch.int32 and positions.shape == (n_rows,)
        shape = (n_rows, self.n_kv_heads, self.d_head)
        for x in (k_out, v_out):
            assert x is None or (x.is_cuda and x.is_contiguous() and x.dtype is self.dtype and x.shape == shape)
        k = self.k.new_empty(shape, dtype=self.dtype) if k_out is None else k_out
        v = torch.empty_like(k) if v_out is None else v_out
        rc = (_lib.s3_kv8_read if self._eight else _lib.s3_kv_read)(self._c, b, _ptr(positions), k.data_ptr(), v.data_ptr(), _stream())
        if rc:
            _check(rc)
        return k, v

    @staticmethod
    def _scratch(q, need, ws):
        if ws is None:
            return q.new_empty(need, dtype=_torch().uint8) if need else None
        assert ws.is_cuda and ws.is_contiguous()
        return ws

    def _out(self, q, out, want_lse, need, ws):
        torch = _torch()
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        else:
            assert out.shape == q.shape and out.dtype is q.dtype and out.is_contiguous() and out.is_cuda
        lse = q.new_empty(q.shape[:2], dtype=torch.float32) if want_lse else None
        return out, lse, self._scratch(q, need, ws)

    def attention(self, q, kv_len, block_table, q_start=None, scale=None, window: int = 0, max_new=None, max_kv=None, out=None,
                  want_lse: bool = False, ws=None, softcap: float = 0.0):
        """s3_paged_attention: q [n_tokens, n_q_heads, d_head] over all that the sequences hold (append first); with softcap
        s3_paged_attention_capped: scores softcap * tanh(score / softcap).  Returns (out, lse fp32 [n_tokens, n_q_heads] | None)."""
        T, n_q, _ = q.shape
        b = self._batch(T, kv_len, block_table, q_start, max_new, max_kv)
        qp, qt, qh, _ = self._rows(q, T)
        c, L = self._c, _lib
        need = (L.s3_kv8_attention_workspace if self._eight else L.s3_paged_attention_workspace)(c, b, n_q)
        out, lse, ws = self._out(q, out, want_lse, need, ws)
        if scale is None:
            scale = self.scale
        op, lp, wp, size = out.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel()
        if self._eight:
            rc = L.s3_kv8_attention(c, b, qp, n_q, qt, qh, scale, softcap, window, op, lp, wp, size, _stream())
        elif softcap:
            rc = L.s3_paged_attention_capped(c, b, qp, n_q, qt, qh, scale, softcap, window, op, lp, wp, size, _stream())
        else:
            rc = L.s3_paged_attention(c, b, qp, n_q, qt, qh, scale, window, op, lp, wp, size, _stream())
        if rc:
            _check(rc)
        return out, lse

    def select(self, q, kv_len, block_table, top_b: int, q_start=None, q_block: int = 1, lead: int = 1, tail: int = 1, max_new=None,
               max_kv=None, ws=None):
        """s3_block_select: per tile of q_block queries and key/value head the top_b blocks (pages) whose signatures score
        highest, the first `lead` and the last `tail` among them.  Returns sel int32 [tiles, n_kv_heads, top_b], ascending, -1 filled."""
        torch = _torch()
        T, n_q, _ = q.shape
        b = self._batch(T, kv_len, block_table, q_start, max_new, max_kv)
        qp, qt, qh, _ = self._rows(q, T)
        sel = q.new_empty((_lib.s3_block_tiles(b, q_block), self.n_kv_heads, top_b), dtype=torch.int32)
        need = _lib.s3_block_select_workspace(self._c16, b, n_q, q_block, top_b)
        ws = self._scratch(q, need, ws)
        rc = _lib.s3_block_select(self._c16, b, qp, n_q, qt, qh, q_block, top_b, lead, tail, sel.data_ptr(), _ptr(ws),
                                  0 if ws is None else ws.numel(), _stream())
        if rc:
            _check(rc)
        return sel

    def block_attention(self, q, kv_len, block_table, sel, q_start=None, q_block: int = 1, scale=None, max_new=None, max_kv=None,
                        out=None, want_lse: bool = False, ws=None, softcap: float = 0.0):
        """s3_block_attention (softcap: s3_block_attention_capped): as attention, over the blocks that sel [tiles, n_kv_heads, top_b] lists (select, or blocks of
        evidence spans).  Returns (out, lse | None)."""
        T, n_q, _ = q.shape
        b = self._batch(T, kv_len, block_table, q_start, max_new, max_kv)
        qp, qt, qh, _ = self._rows(q, T)
        tiles, heads, top_b = sel.shape
        assert sel.is_cuda and sel.is_contiguous() and sel.dtype is kv_len.dtype and heads == self.n_kv_heads
        assert tiles >= _lib.s3_block_tiles(b, q_block)
        c, L = self._c, _lib
        need = (L.s3_kv8_block_attention_workspace if self._eight else L.s3_block_attention_workspace)(c, b, n_q, q_block, top_b)
        out, lse, ws = self._out(q, out, want_lse, need, ws)
        if scale is None:
            scale = self.scale
        sp, op, lp, wp, size = sel.data_ptr(), out.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel()
        if self._eight:
            rc = L.s3_kv8_block_attention(c, b, qp, n_q, qt, qh, sp, q_block, top_b, scale, softcap, op, lp, wp, size, _stream())
        elif softcap:
            rc = L.s3_block_attention_capped(c, b, qp, n_q, qt, qh, sp, q_block, top_b, scale, softcap, op, lp, wp, size, _stream())
        else:
            rc = L.s3_block_attention(c, b, qp, n_q, qt, qh, sp, q_block, top_b, scale, op, lp, wp, size, _stream())
        if rc:
            _check(rc)
        return out, lse


class KVCache8(KVCache):
    """The same in 8 bits (s3_kv8_cache): half of a bf16 cache's memory, and of its traffic.  k [n_pages, n_kv_heads, d_head / 16, page_size, 16] and
    v [n_pages, n_kv_heads, page_size / 16, d_head, 16] in float8_e4m3fn, scale [n_pages, n_kv_heads, 2, page_size] uint8: element times
    2^(code - 127) is what it stands for.  Every call of KVCache is here, with the same arguments; rows are bfloat16.  The argument `scale` takes those codes, which the cache
    keeps as .codes; .scale is what attention multiplies scores by, as in KVCache."""

    _eight = True

    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, d_head: int, signatures: bool = False, device="cuda", k=None, v=None,
                 scale=None, sig=None):
        import torch
        f8 = torch.float8_e4m3fn

        def array(name, t, dt, shape):
            if t is None:
                return torch.empty(shape, dtype=dt, device=device)
            assert t.is_cuda and t.is_contiguous() and t.dtype == dt and tuple(t.shape) == shape, name
            return t
        self.k = array("k", k, f8, (n_pages, n_kv_heads, d_head // 16, page_size, 16))
        self.v = array("v", v, f8, (n_pages, n_kv_heads, page_size // 16, d_head, 16))
        self.codes = array("scale", scale, torch.uint8, (n_pages, n_kv_heads, 2, page_size))
        self.sig = array("sig", sig, torch.bfloat16, (n_pages, n_kv_heads, d_head)) if signatures or sig is not None else None
        lib()
        self.scale = d_head ** -0.5
        self.dtype, self.page_size, self.n_kv_heads, self.d_head, self.n_pages = torch.bfloat16, page_size, n_kv_heads, d_head, n_pages
        sizes = (n_pages, page_size, n_kv_heads, d_head)
        self._c = _KV8_CACHE.pack(_ptr(self.k), _ptr(self.v), _ptr(self.codes), _ptr(self.sig) or 0, *sizes)
        self._c16 = _KV_CACHE.pack(_ptr(self.k), _ptr(self.v), _ptr(self.sig) or 0, S3_BF16, *sizes)      # for the choice, which reads sig only
