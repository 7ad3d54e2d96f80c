"""Python binding of librest.so, the CUDA (sm_100a) hot path of one REST decoding step.

Argument marshalling only: every step runs in the library's kernels.  torch is used to own
device memory and to supply the current CUDA stream.  There is no CPU fallback: importing
works without the library, but every call raises if librest.so is missing or cannot load.

The entry points mirror include/rest.h.  One decoding step:
    rest_datastore_create / Datastore   Sec. 3.2, datastore = token stream + suffix array
    rest_draft                          Algorithms 1 and 2, breadth-first tree + mask
    rest_tree_attention                 Sec. 3.2, draft verification (tree attention)
    rest_accept                         Sec. 3.2, draft acceptance
    rest_kv_commit                      accepted K/V rows moved to the front
Serving, with a KV cache in pages:
    rest_paged_attention                tree attention or one-token steps over pages, windows
    rest_accept_sampled                 Sec. 4.1, acceptance against the target's probabilities
    rest_paged_kv_write / _commit       a step's new rows; the accepted ones moved to the front
    rest_pages_fork / _copy / _reserve / _release   contexts that share, get and give back pages
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "librest.so")

REST_OK = 0
REST_SAMPLE_STRIDED = 0
REST_SAMPLE_FIRST_K = 1
REST_SEARCH_AUTO = 0
REST_SEARCH_SINGLE = 1
REST_SEARCH_BATCHED = 2
REST_BF16 = 0
REST_FP16 = 1
REST_FP32 = 2
REST_CTX_OK = 0
REST_CTX_NO_PAGES = 4
REST_CTX_BAD_PAGES = 5
REST_DS_VALIDATE = 1
REST_DS_INDEX = 2

EXPORTS = (
    "rest_datastore_aux_bytes", "rest_datastore_create", "rest_datastore_create_shard",
    "rest_datastore_destroy", "rest_draft_workspace_bytes", "rest_draft",
    "rest_retrieve", "rest_gather_rows", "rest_draft_from_runs_workspace_bytes", "rest_draft_from_runs",
    "rest_tree_attention_workspace_bytes", "rest_tree_attention",
    "rest_tree_attention_static_scratch",
    "rest_device_error_flags", "rest_kv_commit", "rest_probe_dependent_reads",
    "rest_suffix_array_workspace_bytes", "rest_suffix_array_min_workspace_bytes",
    "rest_suffix_array_build", "rest_suffix_array_build_in_groups", "rest_suffix_array_build_full",
    "rest_suffix_array_append_workspace_bytes", "rest_suffix_array_append", "rest_tree_attention_plan",
    "rest_paged_attention_workspace_bytes", "rest_paged_attention", "rest_accept_sampled_workspace_bytes",
    "rest_accept_sampled",
    "rest_paged_kv_write", "rest_paged_kv_commit", "rest_pages_fork", "rest_pages_copy",
    "rest_pages_reserve", "rest_pages_release",
    "rest_accept", "rest_status_string", "rest_last_cuda_error", "rest_launch_count",
)


class RestError(RuntimeError):
    pass


class _Params(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_max", "n_min", "K", "m", "N", "sample_mode",
                                              "search_path")]


_lib = None


def library_path() -> str:
    return _SO


def lib():
    """Loads librest.so; raises RestError when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_SO):
        raise RestError(f"{_SO} is missing: build it with `python -m paper_2311_08252_b200.build` "
                        "(there is no CPU fallback)")
    L = ctypes.CDLL(_SO)
    vp, i32, i64, u32, u64, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64,
                                  ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t)
    L.rest_datastore_aux_bytes.restype = sz
    L.rest_datastore_aux_bytes.argtypes = [u64, i32, u32]
    L.rest_datastore_create.restype = i32
    L.rest_datastore_create.argtypes = [vp, u64, vp, i32, u32, u32, vp, sz, vp,
                                        ctypes.POINTER(vp)]
    L.rest_datastore_create_shard.restype = i32
    L.rest_datastore_create_shard.argtypes = [vp, u64, vp, u64, i32, u32, u32, vp, sz, vp,
                                              ctypes.POINTER(vp)]
    L.rest_retrieve.restype = i32
    L.rest_retrieve.argtypes = [vp, ctypes.POINTER(_Params), vp, i64, vp, i32, vp, vp, vp, vp]
    L.rest_gather_rows.restype = i32
    L.rest_gather_rows.argtypes = [vp, ctypes.POINTER(_Params), vp, vp, vp, i32, i32, vp, vp, vp, vp]
    L.rest_draft_from_runs_workspace_bytes.restype = sz
    L.rest_draft_from_runs_workspace_bytes.argtypes = [i32, i32, i32]
    L.rest_draft_from_runs.restype = i32
    L.rest_draft_from_runs.argtypes = [ctypes.POINTER(_Params), vp, vp, vp, i32, i32, vp, i32] + [vp] * 8 + \
        [vp, sz, vp]
    L.rest_datastore_destroy.restype = None
    L.rest_datastore_destroy.argtypes = [vp]
    L.rest_draft_workspace_bytes.restype = sz
    L.rest_draft_workspace_bytes.argtypes = [ctypes.POINTER(_Params), i32]
    L.rest_draft.restype = i32
    L.rest_draft.argtypes = [vp, ctypes.POINTER(_Params), vp, i64, vp, i32] + [vp] * 10 + [vp, sz, vp]
    L.rest_tree_attention_workspace_bytes.restype = sz
    L.rest_tree_attention_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    L.rest_tree_attention.restype = i32
    L.rest_tree_attention.argtypes = [vp, vp, vp, ctypes.POINTER(i64), vp, vp, i32, i32, i32, i32,
                                      i32, i32, ctypes.c_float, vp, vp, vp, sz, vp]
    L.rest_tree_attention_static_scratch.restype = i32
    L.rest_tree_attention_static_scratch.argtypes = [vp, vp, vp, ctypes.POINTER(i64), vp, vp, i32,
                                                     i32, i32, i32, i32, i32, ctypes.c_float, vp,
                                                     vp, vp]
    L.rest_accept.restype = i32
    L.rest_accept.argtypes = [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp]
    L.rest_kv_commit.restype = i32
    L.rest_kv_commit.argtypes = [vp, vp, ctypes.POINTER(i64), vp, vp, vp, i32, i32, i32, i32, i32, vp, vp]
    L.rest_paged_attention_workspace_bytes.restype = sz
    L.rest_paged_attention_workspace_bytes.argtypes = [i32] * 5
    L.rest_paged_attention.restype = i32
    L.rest_paged_attention.argtypes = [vp, vp, vp, ctypes.POINTER(i64), i32, i32, i32, vp, i64, i32, vp, vp, vp, i32,
                                       i32, i32, i32, i32, i32, i32, ctypes.c_float, vp, vp, vp, sz, vp]
    L.rest_accept_sampled.restype = i32
    L.rest_accept_sampled.argtypes = [vp, i32, i64, i64, i32] + [vp] * 6 + [i32, i32, i32] + [vp] * 4 + [sz, vp]
    L.rest_accept_sampled_workspace_bytes.restype = sz
    L.rest_accept_sampled_workspace_bytes.argtypes = [i32, i32]
    pool = [vp, vp, ctypes.POINTER(i64), i32, i32]           # K, V, strides, pages, rows per page
    table = [vp, i64, i32]                                   # block table, row stride, columns
    L.rest_paged_kv_write.restype = i32
    L.rest_paged_kv_write.argtypes = pool + table + [vp, vp, vp, ctypes.POINTER(i64), vp, i32, i32, i32, i32, vp]
    L.rest_paged_kv_commit.restype = i32
    L.rest_paged_kv_commit.argtypes = pool + table + [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp]
    L.rest_pages_copy.restype = i32
    L.rest_pages_copy.argtypes = pool + [i32, i32, vp, vp, i32, vp]
    L.rest_pages_fork.restype = i32
    L.rest_pages_fork.argtypes = [vp, i32] + table + [vp, vp, i32, i32, vp, vp, i32, vp, vp, vp, vp]
    L.rest_pages_reserve.restype = i32
    L.rest_pages_reserve.argtypes = [vp, i32] + table + [vp, vp, i32, i32, vp, vp]
    L.rest_pages_release.restype = i32
    L.rest_pages_release.argtypes = [vp, i32] + table + [vp, vp, i32, i32, i32, i32, vp]
    L.rest_suffix_array_workspace_bytes.restype = sz
    L.rest_suffix_array_workspace_bytes.argtypes = [u64]
    L.rest_suffix_array_min_workspace_bytes.restype = sz
    L.rest_suffix_array_min_workspace_bytes.argtypes = [u64, u64]
    L.rest_suffix_array_build.restype = i32
    L.rest_suffix_array_build.argtypes = [vp, u64, i32, vp, vp, sz, vp]
    L.rest_suffix_array_append_workspace_bytes.restype = sz
    L.rest_suffix_array_append_workspace_bytes.argtypes = [u64]
    L.rest_suffix_array_append.restype = i32
    L.rest_suffix_array_append.argtypes = [vp, u64, u64, vp, i32, vp, vp, sz, vp]
    L.rest_suffix_array_build_full.restype = i32
    L.rest_suffix_array_build_full.argtypes = [vp, u64, i32, vp, vp, sz, vp]
    L.rest_suffix_array_build_in_groups.restype = i32
    L.rest_suffix_array_build_in_groups.argtypes = [vp, u64, i32, vp, u64, vp, sz, vp]
    L.rest_tree_attention_plan.restype = i32
    L.rest_tree_attention_plan.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
    L.rest_probe_dependent_reads.restype = i32
    L.rest_probe_dependent_reads.argtypes = [vp, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_uint32, vp, vp]
    L.rest_device_error_flags.restype = i32
    L.rest_device_error_flags.argtypes = [ctypes.POINTER(u32)]
    L.rest_status_string.restype = ctypes.c_char_p
    L.rest_status_string.argtypes = [i32]
    L.rest_last_cuda_error.restype = ctypes.c_char_p
    L.rest_launch_count.restype = u64
    _lib = L
    return L


def _check(rc: int, what: str):
    if rc != REST_OK:
        L = lib()
        msg = L.rest_status_string(rc).decode()
        if rc == 4:
            msg += ": " + L.rest_last_cuda_error().decode()
        raise RestError(f"{what} failed: {msg} (status {rc})")


def _stream(stream=None) -> int:
    import torch
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _dev_i32(t, name):
    import torch
    if not (t.is_cuda and t.dtype == torch.int32 and t.is_contiguous()):
        raise RestError(f"{name} must be a contiguous int32 CUDA tensor")
    return t


def device_error_flags() -> int:
    """Reads and clears the device-side error bits (0 = no kernel ever gave up on a wait)."""
    v = ctypes.c_uint32(0)
    _check(lib().rest_device_error_flags(ctypes.byref(v)), "rest_device_error_flags")
    return int(v.value)


def launch_count() -> int:
    return int(lib().rest_launch_count())


class Datastore:
    """Handle over device-resident tokens int32[n] and suffix array int32[n] / int64[n].
    The tensors are borrowed: this object keeps references so they outlive the handle.
    index=True also builds the bucket index (token and token-pair ranges of the suffix array)
    that lets rest_draft start its searches inside a small range; results do not depend on it."""

    def __init__(self, tokens, sa, vocab: int, validate: bool = False, stream=None,
                 index: bool = True):
        import torch
        if not (tokens.is_cuda and tokens.dtype == torch.int32 and tokens.is_contiguous()):
            raise RestError("tokens must be a contiguous int32 CUDA tensor")
        if not (sa.is_cuda and sa.dtype in (torch.int32, torch.int64) and sa.is_contiguous()
                and 0 < sa.numel() <= tokens.numel()):
            raise RestError("sa must be a contiguous int32/int64 CUDA tensor, at most as long as tokens")
        self.tokens, self.sa, self.vocab = tokens, sa, int(vocab)
        self.n_tokens = tokens.numel()
        self.sa_bytes = sa.element_size()
        L = lib()
        aux, aux_bytes = None, 0
        flags = (REST_DS_VALIDATE if validate else 0) | (REST_DS_INDEX if index else 0)
        if flags:
            aux_bytes = L.rest_datastore_aux_bytes(self.n_tokens, self.sa_bytes, self.vocab)
            aux = torch.empty(aux_bytes, dtype=torch.uint8, device=tokens.device)
        h = ctypes.c_void_p()
        # a suffix array shorter than the token stream lists the positions of a shard's own range
        rc = L.rest_datastore_create_shard(tokens.data_ptr(), self.n_tokens, sa.data_ptr(), sa.numel(),
                                           self.sa_bytes, self.vocab, flags, _ptr(aux), aux_bytes,
                                           _stream(stream), ctypes.byref(h))
        _check(rc, "rest_datastore_create")
        self._h = h
        self._aux = aux if index else None      # the handle reads the index for its whole life

    def close(self):
        if getattr(self, "_h", None):
            lib().rest_datastore_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rest_datastore_create(tokens, sa, vocab, validate=False, stream=None, index=True) -> Datastore:
    return Datastore(tokens, sa, vocab, validate, stream, index)


@dataclass
class DraftOutput:
    tokens: "object"
    parents: "object"
    depth: "object"
    pos_ids: "object"
    mask: "object"
    n_nodes: "object"
    match_n: "object"
    match_range: "object"
    node_count: "object"
    status: "object"


def alloc_draft_output(B: int, N: int, device) -> DraftOutput:
    import torch
    i32 = dict(dtype=torch.int32, device=device)
    Wm = (N + 31) // 32
    return DraftOutput(
        torch.empty((B, N), **i32), torch.empty((B, N), **i32), torch.empty((B, N), **i32),
        torch.empty((B, N), **i32), torch.empty((B, N, Wm), **i32), torch.empty(B, **i32),
        torch.empty(B, **i32), torch.empty((B, 2), dtype=torch.int64, device=device),
        torch.empty((B, N), **i32), torch.empty(B, **i32))


def draft_workspace_bytes(B: int, n_max=16, n_min=2, K=5000, m=10, N=64,
                          sample_mode=REST_SAMPLE_STRIDED, search=REST_SEARCH_AUTO) -> int:
    """Scratch bytes rest_draft can use for a call of B contexts on the current device (0 when
    a scratch would not make the call faster)."""
    prm = _Params(n_max, n_min, K, m, N, sample_mode, search)
    return int(lib().rest_draft_workspace_bytes(ctypes.byref(prm), B))


def rest_draft(ds: Datastore, ctx, ctx_len, n_max=16, n_min=2, K=5000, m=10, N=64,
               sample_mode=REST_SAMPLE_STRIDED, out: DraftOutput | None = None, stream=None,
               search=REST_SEARCH_AUTO, workspace=None) -> DraftOutput:
    """Draft trees for contexts ctx int32[B, Lc] (row b holds ctx_len[b] tokens).  The mask
    tensor is int32 storage of the uint32 words.  `search` (REST_SEARCH_*) picks the
    single-context or the batched path; the results do not depend on it.  `workspace`: a uint8
    CUDA tensor of rest_draft_workspace_bytes() bytes, None to allocate one when the library
    asks for it, False to pass none (the batched path then runs as a single launch)."""
    L = lib()
    _dev_i32(ctx_len, "ctx_len")
    import torch
    if not (ctx.is_cuda and ctx.dtype == torch.int32 and ctx.dim() == 2 and ctx.stride(1) == 1):
        raise RestError("ctx must be an int32 CUDA tensor [B, Lc] with contiguous rows")
    B = ctx.shape[0]
    if out is None:
        out = alloc_draft_output(B, N, ctx.device)
    prm = _Params(n_max, n_min, K, m, N, sample_mode, search)
    ws_ptr, ws_bytes = 0, 0
    if workspace is None:
        need = L.rest_draft_workspace_bytes(ctypes.byref(prm), B)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=ctx.device)
    if workspace is not None and workspace is not False:
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = L.rest_draft(ds._h, ctypes.byref(prm), ctx.data_ptr(), ctx.stride(0), ctx_len.data_ptr(), B,
                      out.tokens.data_ptr(), out.parents.data_ptr(), out.depth.data_ptr(),
                      out.pos_ids.data_ptr(), out.mask.data_ptr(), out.n_nodes.data_ptr(),
                      out.match_n.data_ptr(), out.match_range.data_ptr(), _ptr(out.node_count),
                      out.status.data_ptr(), ws_ptr, ws_bytes, _stream(stream))
    _check(rc, "rest_draft")
    return out


def rest_retrieve(ds: Datastore, ctx, ctx_len, n_max=16, n_min=2, stream=None):
    """Algorithm 1 alone: returns (match_n int32[B], match_range int64[B,2], status int32[B])."""
    import torch
    L = lib()
    _dev_i32(ctx_len, "ctx_len")
    if not (ctx.is_cuda and ctx.dtype == torch.int32 and ctx.dim() == 2 and ctx.stride(1) == 1):
        raise RestError("ctx must be an int32 CUDA tensor [B, Lc] with contiguous rows")
    B = ctx.shape[0]
    match_n = torch.empty(B, dtype=torch.int32, device=ctx.device)
    match_range = torch.empty((B, 2), dtype=torch.int64, device=ctx.device)
    status = torch.empty(B, dtype=torch.int32, device=ctx.device)
    prm = _Params(n_max, n_min, 1, 1, 1, 0, 0)
    _check(L.rest_retrieve(ds._h, ctypes.byref(prm), ctx.data_ptr(), ctx.stride(0), ctx_len.data_ptr(), B,
                           match_n.data_ptr(), match_range.data_ptr(), status.data_ptr(), _stream(stream)),
           "rest_retrieve")
    return match_n, match_range, status


def rest_gather_rows(ds: Datastore, match_n, match_range, take, Kr: int, m=10,
                     sample_mode=REST_SAMPLE_STRIDED, status=None, stream=None):
    """The take[b] sampled candidate rows of every context's matched range: returns
    (rows int32[B,Kr,m], row_len int32[B,Kr], status int32[B])."""
    import torch
    L = lib()
    for t, nm in ((match_n, "match_n"), (take, "take")):
        _dev_i32(t, nm)
    B = match_n.shape[0]
    rows = torch.empty((B, Kr, m), dtype=torch.int32, device=match_n.device)
    row_len = torch.empty((B, Kr), dtype=torch.int32, device=match_n.device)
    if status is None:
        status = torch.zeros(B, dtype=torch.int32, device=match_n.device)
    prm = _Params(16, 2, Kr, m, 1, sample_mode, 0)
    _check(L.rest_gather_rows(ds._h, ctypes.byref(prm), match_n.data_ptr(), match_range.data_ptr(),
                              take.data_ptr(), B, Kr, rows.data_ptr(), row_len.data_ptr(),
                              status.data_ptr(), _stream(stream)), "rest_gather_rows")
    return rows, row_len, status


def rest_draft_from_runs(rows, row_len, run_rows, ctx_len, m=None, N=64, out: DraftOutput | None = None,
                         stream=None) -> DraftOutput:
    """Trees from candidate rows handed in as sorted runs: rows int32[B,R,Kr,m], row_len
    int32[B,R,Kr], run_rows int32[B,R].  match_n / match_range of the result are not written."""
    import torch
    L = lib()
    for t, nm in ((rows, "rows"), (row_len, "row_len"), (run_rows, "run_rows"), (ctx_len, "ctx_len")):
        _dev_i32(t, nm)
    B, R, Kr, mm = rows.shape
    m = mm if m is None else m
    if m != mm or row_len.shape != (B, R, Kr) or run_rows.shape != (B, R):
        raise RestError("rows [B,R,Kr,m], row_len [B,R,Kr] and run_rows [B,R] do not fit together")
    if out is None:
        out = alloc_draft_output(B, N, rows.device)
    ws_bytes = L.rest_draft_from_runs_workspace_bytes(B, R, Kr)
    ws = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=rows.device)
    prm = _Params(16, 2, R * Kr, m, N, 0, 0)
    _check(L.rest_draft_from_runs(ctypes.byref(prm), rows.data_ptr(), row_len.data_ptr(), run_rows.data_ptr(),
                                  R, Kr, ctx_len.data_ptr(), B, out.tokens.data_ptr(), out.parents.data_ptr(),
                                  out.depth.data_ptr(), out.pos_ids.data_ptr(), out.mask.data_ptr(),
                                  out.n_nodes.data_ptr(), _ptr(out.node_count), out.status.data_ptr(),
                                  ws.data_ptr(), ws_bytes, _stream(stream)), "rest_draft_from_runs")
    return out


def tree_attention_workspace_bytes(B, H, N, D, max_kv) -> int:
    return int(lib().rest_tree_attention_workspace_bytes(B, H, N, D, max_kv))


def rest_tree_attention(q, k, v, kv_len, mask, scale, max_kv=None, out=None, lse=None,
                        workspace=None, stream=None):
    """q bf16 [B,N,H,D]; k, v bf16 [B,H_kv,Lcap,D] (tree rows at kv_len[b]..kv_len[b]+N-1);
    kv_len int32[B]; mask int32/uint32 words [B,N,ceil(N/32)].  Returns out bf16 [B,N,H,D]."""
    import torch
    L = lib()
    B, N, H, D = q.shape
    H_kv, Lcap = k.shape[1], k.shape[2]
    for t, nm in ((q, "q"), (k, "k"), (v, "v")):
        if not (t.is_cuda and t.dtype == torch.bfloat16 and t.stride(-1) == 1):
            raise RestError(f"{nm} must be a bf16 CUDA tensor with a contiguous last dimension")
    if k.stride() != v.stride() or k.shape != v.shape:
        raise RestError("k and v must have the same shape and strides")
    _dev_i32(kv_len, "kv_len")
    if not (mask.is_cuda and mask.is_contiguous() and mask.element_size() == 4):
        raise RestError("mask must be a contiguous 32-bit CUDA tensor")
    if out is None:
        out = torch.empty((B, N, H, D), dtype=torch.bfloat16, device=q.device)
    max_kv = Lcap if max_kv is None else int(max_kv)
    need = L.rest_tree_attention_workspace_bytes(B, H, N, D, max_kv)
    if need and (workspace is None or workspace.numel() * workspace.element_size() < need):
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    strides = (ctypes.c_int64 * 9)(q.stride(0), q.stride(1), q.stride(2),
                                   k.stride(0), k.stride(1), k.stride(2),
                                   out.stride(0), out.stride(1), out.stride(2))
    rc = L.rest_tree_attention(q.data_ptr(), k.data_ptr(), v.data_ptr(), strides, kv_len.data_ptr(),
                               mask.data_ptr(), B, H, H_kv, N, D, max_kv, float(scale),
                               out.data_ptr(), _ptr(lse), _ptr(workspace),
                               0 if workspace is None else workspace.numel() * workspace.element_size(),
                               _stream(stream))
    _check(rc, "rest_tree_attention")
    return out


def rest_tree_attention_static_scratch(q, k, v, kv_len, mask, scale, out, max_kv=None, lse=None,
                                       stream=None):
    """rest_tree_attention without a workspace argument, for callers that must not allocate:
    the split partials go to a fixed 768 KiB array inside the library.  `out` (bf16 [B,N,H,D])
    is supplied by the caller, so this wrapper allocates nothing on the device either.
    Raises RestError (workspace too small) when the shape needs more than the fixed array.
    Calls share that array: do not let two of them overlap on the GPU."""
    L = lib()
    B, N, H, D = q.shape
    H_kv, Lcap = k.shape[1], k.shape[2]
    max_kv = Lcap if max_kv is None else int(max_kv)
    strides = (ctypes.c_int64 * 9)(q.stride(0), q.stride(1), q.stride(2),
                                   k.stride(0), k.stride(1), k.stride(2),
                                   out.stride(0), out.stride(1), out.stride(2))
    rc = L.rest_tree_attention_static_scratch(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), strides, kv_len.data_ptr(), mask.data_ptr(),
        B, H, H_kv, N, D, max_kv, float(scale), out.data_ptr(), _ptr(lse), _stream(stream))
    _check(rc, "rest_tree_attention_static_scratch")
    return out


def rest_accept(tokens, parents, n_nodes, verifier_tokens, max_depth, out=None, stream=None):
    """Returns (accept_len int32[B], accept_nodes int32[B,max_depth], out_tokens int32[B,max_depth+1])."""
    import torch
    L = lib()
    for t, nm in ((tokens, "tokens"), (parents, "parents"), (n_nodes, "n_nodes"),
                  (verifier_tokens, "verifier_tokens")):
        _dev_i32(t, nm)
    B, N = tokens.shape
    if verifier_tokens.shape != (B, N + 1):
        raise RestError("verifier_tokens must be [B, N+1]")
    if out is None:
        i32 = dict(dtype=torch.int32, device=tokens.device)
        out = (torch.empty(B, **i32), torch.empty((B, max_depth), **i32),
               torch.empty((B, max_depth + 1), **i32))
    rc = L.rest_accept(tokens.data_ptr(), parents.data_ptr(), n_nodes.data_ptr(),
                       verifier_tokens.data_ptr(), B, N, max_depth, out[0].data_ptr(),
                       out[1].data_ptr(), out[2].data_ptr(), _stream(stream))
    _check(rc, "rest_accept")
    return out


def rest_kv_commit(k, v, kv_len, accept_nodes, accept_len, N, new_kv_len=None, stream=None):
    """Moves the K/V rows of the accepted draft nodes (tree slots kv_len[b] + node) to the
    contiguous slots kv_len[b] .. kv_len[b] + accept_len[b] - 1 of k, v bf16 [B,H_kv,Lcap,D], in
    place.  new_kv_len (optional int32[B]) receives kv_len + accept_len."""
    import torch
    L = lib()
    for t, nm in ((k, "k"), (v, "v")):
        if not (t.is_cuda and t.dtype == torch.bfloat16 and t.stride(-1) == 1):
            raise RestError(f"{nm} must be a bf16 CUDA tensor with a contiguous last dimension")
    if k.stride() != v.stride() or k.shape != v.shape:
        raise RestError("k and v must have the same shape and strides")
    for t, nm in ((kv_len, "kv_len"), (accept_nodes, "accept_nodes"), (accept_len, "accept_len")):
        _dev_i32(t, nm)
    B, H_kv, _, D = k.shape
    max_depth = accept_nodes.shape[1]
    strides = (ctypes.c_int64 * 3)(k.stride(0), k.stride(1), k.stride(2))
    rc = L.rest_kv_commit(k.data_ptr(), v.data_ptr(), strides, kv_len.data_ptr(), _ptr(accept_nodes),
                          accept_len.data_ptr(), B, H_kv, N, D, max_depth, _ptr(new_kv_len),
                          _stream(stream))
    _check(rc, "rest_kv_commit")
    return new_kv_len


# ------------------------------------------------------------------------------ cache in pages
# These calls are made many times per decoding step, so their checks go through few, cheap tensor
# queries: get_device() says both that a tensor is on a GPU (-1: it is not) and on which.
_I64x3 = ctypes.c_int64 * 3
_I64x9 = ctypes.c_int64 * 9


def _call(fn, what, index, stream, *args):
    """fn(*args, stream) on GPU `index`, whatever the current device is; raises on an error status."""
    import torch
    if index < 0:
        raise RestError(f"{what}: the tensors must be on a CUDA device")
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            return _call(fn, what, index, stream, *args)
    if stream is None:
        raw = torch._C._cuda_getCurrentRawStream(index)
    else:
        _same_device(stream, index)
        raw = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    rc = fn(*args, raw)
    if rc:
        _check(rc, what)


def _same_device(stream, index):
    """Refuses a torch stream of another GPU than `index` (a handle does not say whose it is)."""
    own = getattr(stream, "device_index", index)
    if own != index:
        raise RestError(f"stream belongs to GPU {own}, the tensors are on GPU {index}")


def _scratch_bytes(fn, index, *args):
    """fn(*args) with GPU `index` as the current device, which the scratch sizes go by."""
    import torch
    if index < 0 or torch.cuda.current_device() == index:
        return fn(*args)
    with torch.cuda.device(index):
        return fn(*args)


def _as_current(stream, t):
    """`stream` (a torch stream or a handle) as the current one: what a call allocates and clears belongs to it."""
    import torch
    if t.get_device() < 0:
        raise RestError("the tensors must be on a CUDA device")
    _same_device(stream, t.get_device())
    if isinstance(stream, torch.cuda.Stream):
        return torch.cuda.stream(stream)
    handle = int(getattr(stream, "cuda_stream", stream))
    handle = 0 if handle == 1 else handle                # cudaStreamLegacy: torch knows the default stream as 0 only
    return torch.cuda.stream(torch.cuda.ExternalStream(handle, device=t.device))


def _window(window, sinks):
    """Refuses what 32 bits would wrap round into another window."""
    if not (0 <= window <= 0x7FFFFFFF and 0 <= sinks <= 0x7FFFFFFF):
        raise RestError("window and sinks must lie in [0, 2^31)")
    return window, sinks


def _vec(t, name, index, n=None, dtype=None):
    """Pointer of a contiguous vector (int32 unless told otherwise) of n elements on GPU `index`."""
    import torch
    dtype = torch.int32 if dtype is None else dtype
    if t.dtype is not dtype or t.get_device() != index or not t.is_contiguous() or t.dim() != 1 or (
            n is not None and t.numel() != n):
        raise RestError(f"{name} must be a contiguous {str(dtype).split('.')[-1]} vector"
                        + ("" if n is None else f" of {n} elements") + " on the same CUDA device as the others")
    return t.data_ptr()


def _array(t, name, index, shape, dtype):
    """Pointer of a contiguous tensor of that shape and type on GPU `index`."""
    if t.dtype is not dtype or t.get_device() != index or not t.is_contiguous() or t.shape != shape:
        raise RestError(f"{name} must be a contiguous {str(dtype).split('.')[-1]} tensor {list(shape)} on the same "
                        "CUDA device as the others")
    return t.data_ptr()


def _pool(k_pages, v_pages):
    """Device, shape, and (pointers, strides, pages, rows per page) of a pool [P, H_kv, page, D]."""
    import torch
    index, shape, strides, dtype = k_pages.get_device(), k_pages.shape, k_pages.stride(), k_pages.dtype
    if len(shape) != 4 or strides[3] != 1 or not (dtype is torch.bfloat16 or dtype is torch.float16):
        raise RestError("k_pages must be a bf16 or fp16 tensor [P, H_kv, page, D] with a contiguous last dimension")
    if v_pages.stride() != strides or v_pages.shape != shape or v_pages.dtype is not dtype or v_pages.get_device() != index:
        raise RestError("k_pages and v_pages must have the same shape, strides, type and device")
    return index, shape, (k_pages.data_ptr(), v_pages.data_ptr(), _I64x3(*strides[:3]), shape[0], shape[2])


def _table(table, index, B=None):
    """Pointer, row stride and columns of a block table."""
    import torch
    shape = table.shape
    if table.dtype is not torch.int32 or table.get_device() != index or len(shape) != 2 or table.stride(1) != 1 or (
            B is not None and shape[0] != B):
        raise RestError("block_table must be an int32 tensor [B, columns] with contiguous rows on the same CUDA device "
                        "as the others")
    stride = table.stride(0)
    # a single row may come with any stride; the library wants rows that do not overlap
    return table.data_ptr(), stride if shape[0] > 1 else max(stride, shape[1]), shape[1]


def paged_attention_workspace_bytes(B, H, H_kv, N, D) -> int:
    """Scratch bytes of rest_paged_attention on the current device."""
    return int(lib().rest_paged_attention_workspace_bytes(B, H, H_kv, N, D))


def rest_paged_attention(q, k_pages, v_pages, block_table, kv_len, mask, scale, window=0, sinks=0, n_nodes=None,
                         out=None, lse=None, workspace=None, stream=None):
    """Attention of q [B,N,H,D] (bf16 or fp16; D 64 or 128; N = 1: one ordinary token) over a cache
    in pages k_pages, v_pages [P,H_kv,page,D], and over the new rows kv_len[b] + i themselves.
    mask: int32 or uint32 words [B,N,ceil(N/32)] as rest_draft writes them, None: node i sees nodes 0..i.
    window > 0: a node sees the last `window` positions up to its own and the first `sinks` ones.
    n_nodes int32[B]: later rows do not exist (their out / lse rows stay as they were).
    lse: optional float32 [B,H,N].  workspace: a uint8 tensor of paged_attention_workspace_bytes(),
    not shared by calls that may overlap; None: one is allocated.  out overlaps no input.  Returns
    out [B,N,H,D]."""
    import torch
    if stream is not None:
        with _as_current(stream, q):
            return rest_paged_attention(q, k_pages, v_pages, block_table, kv_len, mask, scale, window, sinks, n_nodes,
                                        out, lse, workspace)
    L = _lib or lib()
    index, (P, H_kv, page, Dk), pool = _pool(k_pages, v_pages)
    dtype, shape, qs = q.dtype, q.shape, q.stride()
    if len(shape) != 4 or qs[3] != 1 or dtype is not k_pages.dtype or shape[3] != Dk or q.get_device() != index:
        raise RestError("q must be [B,N,H,D] with a contiguous last dimension, of the pages' type, head size and device")
    B, N, H, D = shape
    window, sinks = _window(window, sinks)
    table = _table(block_table, index, B)
    mask_ptr = lse_ptr = nodes_ptr = ws_ptr = ws_bytes = 0
    if mask is not None:
        if (mask.dtype is not torch.int32 and mask.dtype is not torch.uint32) or mask.get_device() != index or (
                not mask.is_contiguous() or mask.shape != (B, N, (N + 31) // 32)):
            raise RestError("mask must be a contiguous int32 or uint32 tensor [B,N,ceil(N/32)] on the same CUDA device")
        mask_ptr = mask.data_ptr()
    if n_nodes is not None:
        nodes_ptr = _vec(n_nodes, "n_nodes", index, B)
    if lse is not None:
        lse_ptr = _array(lse, "lse", index, (B, H, N), torch.float32)
    if out is None:
        out = (torch.empty if n_nodes is None else torch.zeros)(shape, dtype=dtype, device=q.device)
    elif out.dtype is not dtype or out.shape != shape or out.stride(3) != 1 or out.get_device() != index:
        raise RestError("out must be a tensor like q with a contiguous last dimension")
    if workspace is None:
        need = _scratch_bytes(L.rest_paged_attention_workspace_bytes, index, B, H, H_kv, N, D)
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise RestError("workspace must be a contiguous tensor on the same CUDA device")
    if workspace is not None:
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    strides = _I64x9(*qs[:3], *pool[2], *out.stride()[:3])
    _call(L.rest_paged_attention, "rest_paged_attention", index, stream, q.data_ptr(), pool[0], pool[1], strides,
          REST_BF16 if dtype is torch.bfloat16 else REST_FP16, P, page, *table, _vec(kv_len, "kv_len", index, B),
          nodes_ptr, mask_ptr, B, H, H_kv, N, D, window, sinks, scale, out.data_ptr(), lse_ptr, ws_ptr, ws_bytes)
    return out


def rest_accept_sampled(logits, tokens, parents, n_nodes, uniforms, temperature, top_p, max_depth, out=None,
                        stream=None, workspace=None):
    """Acceptance of draft trees against the verifier's probabilities: logits [B,N+1,V] (bf16, fp16
    or fp32; slot 0 after the prefix, slot i+1 after node i), uniforms float32 [B,N+1] in [0, 1),
    temperature and top_p float32 [B].  workspace: a uint8 tensor of
    rest_accept_sampled_workspace_bytes() bytes, not shared by calls that may overlap; None: one is
    allocated when the library asks for it; False: none (each context walks row by row).  Returns
    (accept_len, accept_nodes, out_tokens) like rest_accept."""
    import torch
    if stream is not None:
        with _as_current(stream, tokens):
            return rest_accept_sampled(logits, tokens, parents, n_nodes, uniforms, temperature, top_p, max_depth, out,
                                       workspace=workspace)
    L = _lib or lib()
    index, (B, N), i32, f32 = tokens.get_device(), tokens.shape, torch.int32, torch.float32
    dtype, shape, ls = logits.dtype, logits.shape, logits.stride()
    kind = {torch.bfloat16: REST_BF16, torch.float16: REST_FP16, f32: REST_FP32}.get(dtype)
    if kind is None or len(shape) != 3 or shape[0] != B or shape[1] != N + 1 or ls[2] != 1 or logits.get_device() != index:
        raise RestError("logits must be a bf16, fp16 or fp32 tensor [B,N+1,V] with contiguous rows on the same CUDA device")
    if out is None:
        out = (torch.empty(B, dtype=i32, device=tokens.device), torch.empty((B, max_depth), dtype=i32, device=tokens.device),
               torch.empty((B, max_depth + 1), dtype=i32, device=tokens.device))
    ws_ptr = ws_bytes = 0
    if workspace is None:
        need = _scratch_bytes(L.rest_accept_sampled_workspace_bytes, index, B, N)
        workspace = torch.empty(need, dtype=torch.uint8, device=tokens.device) if need else False
    if workspace is not False:
        if workspace.get_device() != index or not workspace.is_contiguous():
            raise RestError("workspace must be a contiguous tensor on the same CUDA device")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _call(L.rest_accept_sampled, "rest_accept_sampled", index, stream, logits.data_ptr(), kind, ls[0], ls[1], shape[2],
          _array(tokens, "tokens", index, (B, N), i32), _array(parents, "parents", index, (B, N), i32),
          _vec(n_nodes, "n_nodes", index, B), _array(uniforms, "uniforms", index, (B, N + 1), f32),
          _vec(temperature, "temperature", index, B, f32), _vec(top_p, "top_p", index, B, f32), B, N, max_depth,
          _vec(out[0], "accept_len", index, B), _array(out[1], "accept_nodes", index, (B, max_depth), i32),
          _array(out[2], "out_tokens", index, (B, max_depth + 1), i32), ws_ptr, ws_bytes)
    return out


def rest_paged_kv_write(k_pages, v_pages, block_table, kv_len, k_new, v_new, n_nodes=None, stream=None):
    """Writes new K/V rows k_new, v_new [B,N,H_kv,D] as rows kv_len[b] + i of the contexts' pages
    (k_pages, v_pages [P,H_kv,page,D] with any 16-byte strides); with n_nodes int32[B] only rows
    i < n_nodes[b].  Rows whose page does not exist are left out."""
    index, (P, H_kv, page, D), pool = _pool(k_pages, v_pages)
    shape, ns = k_new.shape, k_new.stride()
    if len(shape) != 4 or shape[2] != H_kv or shape[3] != D or ns[3] != 1 or k_new.dtype is not k_pages.dtype or (
            k_new.get_device() != index):
        raise RestError("k_new must be [B,N,H_kv,D] of the pages' heads, type and device, with a contiguous last dimension")
    if v_new.shape != shape or v_new.stride() != ns or v_new.dtype is not k_new.dtype or v_new.get_device() != index:
        raise RestError("k_new and v_new must have the same shape, strides, type and device")
    B, N = shape[0], shape[1]
    _call((_lib or lib()).rest_paged_kv_write, "rest_paged_kv_write", index, stream, *pool, *_table(block_table, index, B),
          _vec(kv_len, "kv_len", index, B), k_new.data_ptr(), v_new.data_ptr(), _I64x3(*ns[:3]),
          0 if n_nodes is None else _vec(n_nodes, "n_nodes", index, B), B, H_kv, N, D)


def rest_paged_kv_commit(k_pages, v_pages, block_table, kv_len, accept_nodes, accept_len, N, new_kv_len=None,
                         stream=None):
    """rest_kv_commit over pages: row kv_len[b] + accept_nodes[b][i] moves to row kv_len[b] + i.
    new_kv_len (optional int32[B], may be kv_len itself) receives kv_len + accept_len."""
    import torch
    index, (P, H_kv, page, D), pool = _pool(k_pages, v_pages)
    B, max_depth = accept_nodes.shape
    _call((_lib or lib()).rest_paged_kv_commit, "rest_paged_kv_commit", index, stream, *pool,
          *_table(block_table, index, B), _vec(kv_len, "kv_len", index, B),
          _array(accept_nodes, "accept_nodes", index, (B, max_depth), torch.int32),
          _vec(accept_len, "accept_len", index, B), B, H_kv, N, D, max_depth,
          0 if new_kv_len is None else _vec(new_kv_len, "new_kv_len", index, B))
    return new_kv_len


def rest_pages_fork(refs, block_table, n_pages, kv_len, parents, children, page, copy_src=None, copy_dst=None,
                    status=None, stream=None):
    """Makes context children[f] a copy of parents[f]: whole pages are shared, a partly filled last
    page is replaced by a page of the child's own.  Returns (copy_src, copy_dst, status) int32[F]:
    the pages to copy with rest_pages_copy in every layer (-1: none), and REST_CTX_* codes."""
    import torch
    if stream is not None:
        with _as_current(stream, refs):
            return rest_pages_fork(refs, block_table, n_pages, kv_len, parents, children, page, copy_src, copy_dst, status)
    F, B, index = parents.numel(), block_table.shape[0], refs.get_device()
    out = tuple(torch.empty(F, dtype=torch.int32, device=refs.device) if t is None else t
                for t in (copy_src, copy_dst, status))
    _call((_lib or lib()).rest_pages_fork, "rest_pages_fork", index, stream, _vec(refs, "refs", index), refs.numel(),
          *_table(block_table, index), _vec(n_pages, "n_pages", index, B), _vec(kv_len, "kv_len", index, B), B, page,
          _vec(parents, "parents", index, F), _vec(children, "children", index, F), F, _vec(out[0], "copy_src", index, F),
          _vec(out[1], "copy_dst", index, F), _vec(out[2], "status", index, F))
    return out


def rest_pages_copy(k_pages, v_pages, src, dst, stream=None):
    """Page dst[i] of K and V becomes a copy of page src[i] (entries outside the pool: left out)."""
    index, shape, pool = _pool(k_pages, v_pages)
    n = src.numel()
    _call((_lib or lib()).rest_pages_copy, "rest_pages_copy", index, stream, *pool, shape[1], shape[3],
          _vec(src, "src", index), _vec(dst, "dst", index, n), n)


def rest_pages_reserve(refs, block_table, n_pages, need_len, page, status=None, stream=None):
    """Gives every context pages until its table holds need_len[b] rows, all or none, in the contexts'
    order: from the first that the pool is too small for, every one that needs a page is refused.
    Returns status int32[B] (REST_CTX_*)."""
    import torch
    if stream is not None:
        with _as_current(stream, refs):
            return rest_pages_reserve(refs, block_table, n_pages, need_len, page, status)
    B, index = block_table.shape[0], refs.get_device()
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=refs.device)
    _call((_lib or lib()).rest_pages_reserve, "rest_pages_reserve", index, stream, _vec(refs, "refs", index),
          refs.numel(), *_table(block_table, index), _vec(n_pages, "n_pages", index, B),
          _vec(need_len, "need_len", index, B), B, page, _vec(status, "status", index, B))
    return status


def rest_pages_release(refs, block_table, n_pages, keep_len, page, window=0, sinks=0, stream=None):
    """Gives back the pages beyond each context's first keep_len[b] rows and, with a window, those
    no later token sees.  keep_len[b] < 0 leaves a context as it is."""
    B, index = block_table.shape[0], refs.get_device()
    _call((_lib or lib()).rest_pages_release, "rest_pages_release", index, stream, _vec(refs, "refs", index),
          refs.numel(), *_table(block_table, index), _vec(n_pages, "n_pages", index, B),
          _vec(keep_len, "keep_len", index, B), B, page, *_window(window, sinks))


def dependent_read_latency_ns(table_bytes: int = 1 << 30, steps: int = 4096, device=None, seed: int = 1) -> float:
    """Nanoseconds per dependent DRAM read on this GPU: builds a random single-cycle table of
    table_bytes (much larger than L2) with torch, then one device thread chases it
    (rest_probe_dependent_reads).  A measurement aid for the draft path's latency floor."""
    import torch
    L = lib()
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    n = table_bytes // 4
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    perm = torch.randperm(n, generator=g, device=device)
    nxt = torch.empty(n, dtype=torch.int32, device=device)
    nxt[perm] = torch.roll(perm, -1).to(torch.int32)       # values < 2^31 for n <= 2^31
    del perm
    out = torch.zeros(2, dtype=torch.int64, device=device)
    best = None
    for rep in range(3):                                   # different stretches of the cycle
        start = int(nxt[rep * 7919 % n].item())
        torch.cuda.synchronize(device)
        _check(L.rest_probe_dependent_reads(nxt.data_ptr(), n, start, steps, out.data_ptr(), _stream(None)),
               "rest_probe_dependent_reads")
        torch.cuda.synchronize(device)
        ns = float(out[0].item()) / steps
        best = ns if best is None else min(best, ns)
    return best


def rest_suffix_array_build(tokens, sa_bytes: int = 4, stream=None, max_group: int | None = None,
                            full: bool = False):
    """Suffix array of the int32 CUDA tensor `tokens`, built on the device and ordered on the
    first 32 tokens of each suffix (ties by position).  Returns an int32 or int64 CUDA tensor.
    max_group: sort the stream in groups of first-token buckets of at most that many positions
    (the method for streams beyond 2^31 - 1 tokens), whatever its size.  full=True: the true
    suffix array (whole suffixes compared) instead of the order on 32 tokens."""
    import torch
    L = lib()
    _dev_i32(tokens, "tokens")
    n = tokens.numel()
    sa = torch.empty(n, dtype=torch.int32 if sa_bytes == 4 else torch.int64, device=tokens.device)
    if max_group is None:
        ws_bytes = L.rest_suffix_array_workspace_bytes(n)
    else:
        ws_bytes = L.rest_suffix_array_min_workspace_bytes(n, int(max_group))
    if ws_bytes == 0:
        raise RestError("rest_suffix_array_build: between 1 and 2^40 tokens are supported")
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=tokens.device)
    if full:
        rc = L.rest_suffix_array_build_full(tokens.data_ptr(), n, sa_bytes, sa.data_ptr(), ws.data_ptr(),
                                            ws_bytes, _stream(stream))
    elif max_group is None:
        rc = L.rest_suffix_array_build(tokens.data_ptr(), n, sa_bytes, sa.data_ptr(), ws.data_ptr(),
                                       ws_bytes, _stream(stream))
    else:
        rc = L.rest_suffix_array_build_in_groups(tokens.data_ptr(), n, sa_bytes, sa.data_ptr(), int(max_group),
                                                 ws.data_ptr(), ws_bytes, _stream(stream))
    _check(rc, "rest_suffix_array_build")
    # set-up call: wait here, so that the scratch can be released whatever stream was used
    torch.cuda.synchronize(tokens.device)
    return sa


def rest_suffix_array_append(tokens, sa_old, stream=None):
    """Suffix array of `tokens` (int32 CUDA tensor: the old stream followed by the appended
    tokens) from the array `sa_old` of its first sa_old.numel() tokens."""
    import torch
    L = lib()
    _dev_i32(tokens, "tokens")
    n, n_old = tokens.numel(), sa_old.numel()
    if not (sa_old.is_cuda and sa_old.dtype in (torch.int32, torch.int64) and sa_old.is_contiguous()) or n_old >= n:
        raise RestError("sa_old must be a contiguous int32/int64 CUDA tensor shorter than tokens")
    sa = torch.empty(n, dtype=sa_old.dtype, device=tokens.device)
    ws_bytes = L.rest_suffix_array_append_workspace_bytes(n - n_old)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=tokens.device)
    _check(L.rest_suffix_array_append(tokens.data_ptr(), n_old, n - n_old, _ptr(sa_old) if n_old else 0,
                                      sa_old.element_size(), sa.data_ptr(), ws.data_ptr(), ws_bytes,
                                      _stream(stream)), "rest_suffix_array_append")
    torch.cuda.synchronize(tokens.device)
    return sa


def tree_attention_plan(B, H, N, D, max_kv) -> dict:
    """Key ranges per (context, head), blocks per cluster, clusters per (context, head), and how
    many clusters of that size the current device runs at once."""
    out = (ctypes.c_int32 * 4)()
    _check(lib().rest_tree_attention_plan(B, H, N, D, max_kv, out), "rest_tree_attention_plan")
    return {"splits": out[0], "cluster": out[1], "clusters_per_unit": out[2], "capacity": out[3]}
