"""ctypes binding of libsparsp.so: argument marshalling only.

Every function here has the name of the C entry point it forwards to (include/sparsp.h).  Tensors
are torch CUDA tensors used purely as device buffers; the current torch CUDA stream is passed down.
There is no fallback: if the library is missing or fails to load, importing a function works but the
first call raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsparsp.so")

SPARSP_OK = 0
SPARSP_ERR_INVALID_ARG = -1
SPARSP_ERR_UNSUPPORTED = -2
SPARSP_ERR_CAPACITY = -3
SPARSP_ERR_CUDA = -4
SPARSP_ERR_TIMEOUT = -5
SPARSP_PLAN_ONLY = 1
SPARSP_INCLUDE_LOCAL = 2

EXPORTS = [
    "sparsp_geometry", "sparsp_resolve_topk", "sparsp_placement_contiguous", "sparsp_placement_periodic",
    "sparsp_workspace_bytes", "sparsp_block_mask", "sparsp_demand_pack", "sparsp_sparse_attn_fwd",
    "sparsp_status", "sparsp_last_error", "sparsp_launch_count", "sparsp_demand_plan_noalloc",
    "sparsp_hop_mask", "sparsp_attn_merge", "sparsp_sparse_attn_fwd_packed", "sparsp_block_mask_cdf",
    "sparsp_placement_permutation", "sparsp_permute_tokens", "sparsp_sharing_histogram", "sparsp_exchange_plan",
    "sparsp_hop_chunk_mask", "sparsp_selftest_wait_timeout", "sparsp_attn_merge_rows", "sparsp_pack_segment",
    "sparsp_xchg_flag_bytes", "sparsp_xchg_export", "sparsp_xchg_connect", "sparsp_xchg_fence", "sparsp_xchg_acquire",
    "sparsp_xchg_publish", "sparsp_xchg_fetch", "sparsp_xchg_release", "sparsp_xchg_stats", "sparsp_xchg_destroy",
    "sparsp_rotary_frequencies", "sparsp_rotary_table_bytes", "sparsp_rotary_table", "sparsp_rotary_apply",
    "sparsp_layer_norm_fwd", "sparsp_layer_norm_workspace_bytes", "sparsp_layer_norm_bwd",
    "sparsp_gated_ffn_workspace_bytes", "sparsp_gated_ffn_fwd", "sparsp_gated_ffn_bwd",
    "sparsp_gated_norm_fwd", "sparsp_gated_norm_workspace_bytes", "sparsp_gated_norm_bwd",
    "sparsp_grad_table_bytes", "sparsp_grad_table", "sparsp_grad_workspace_bytes", "sparsp_grad_squares", "sparsp_grad_clip",
    "sparsp_fp4_scales_bytes", "sparsp_fp4_quantize", "sparsp_fp4_product_workspace_bytes", "sparsp_fp4_product",
]
SPARSP_XCHG_HOST_MEMORY = 1
SPARSP_BF16, SPARSP_FP16, SPARSP_FP32 = 0, 1, 2
DTYPES = {torch.bfloat16: SPARSP_BF16, torch.float16: SPARSP_FP16, torch.float32: SPARSP_FP32}
PAIRINGS = {"interleaved": 0, "half": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}
ACTIVATIONS = {"silu": 0, "gelu_tanh": 1, "gelu": 2}
NORMS = {"none": 0, "layer": 1, "rms": 2}
FP4_FORMATS = {"mxfp4": 0, "nvfp4": 1}

# Argument types of the calls that a layer makes (s: shape, r / n / m / e / t / q / g: description of rotary
# positions, a norm, a feed-forward, a residual step, a list of gradients, a 4-bit operand or a product of two, p: pointer, i / l: 32 / 64-bit integer, f / d: 32 / 64-bit float), so that ctypes
# converts plain values itself: a ctypes object per argument costs more than the call.
_SIGNATURES = {
    "sparsp_block_mask": "sppippppppp",
    "sparsp_block_mask_cdf": "sppffpppppp",
    "sparsp_demand_pack": "sppiipppppppplppp",
    "sparsp_demand_plan_noalloc": "sppiipppppp",
    "sparsp_sparse_attn_fwd": "sppppfpppp",
    "sparsp_sparse_attn_fwd_packed": "spppppiipppplpfpppp",
    "sparsp_hop_mask": "sppiiipp",
    "sparsp_hop_chunk_mask": "sppiiiiipp",
    "sparsp_attn_merge": "sppppppp",
    "sparsp_attn_merge_rows": "spppppppiiiip",
    "sparsp_pack_segment": "sppiiippppplpp",
    "sparsp_rotary_frequencies": "ididdddpp",
    "sparsp_rotary_table_bytes": "rp",
    "sparsp_rotary_table": "rpdpp",
    "sparsp_rotary_apply": "srppliiippppipp",
    "sparsp_layer_norm_fwd": "nppppppp",
    "sparsp_layer_norm_workspace_bytes": "np",
    "sparsp_layer_norm_bwd": "npppppppppp",
    "sparsp_gated_ffn_workspace_bytes": "mip",
    "sparsp_gated_ffn_fwd": "mpppppppp",
    "sparsp_gated_ffn_bwd": "mppppppppppp",
    "sparsp_gated_norm_fwd": "e" + 12 * "p",
    "sparsp_gated_norm_workspace_bytes": "ep",
    "sparsp_gated_norm_bwd": "e" + 19 * "p",
    "sparsp_grad_workspace_bytes": "p",
    "sparsp_grad_table_bytes": "tp",
    "sparsp_grad_table": "tp",
    "sparsp_grad_squares": "tpipp",
    "sparsp_grad_clip": "tpdppp",
    "sparsp_fp4_scales_bytes": "qp",
    "sparsp_fp4_quantize": "qppppp",
    "sparsp_fp4_product_workspace_bytes": "gp",
    "sparsp_fp4_product": "gpppppppp",
}


class SparspError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"sparsp error {code}: {text}")
        self.code = code


class sparsp_shape(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("grid_t", ctypes.c_int32), ("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("n_text", ctypes.c_int32), ("block", ctypes.c_int32),
                ("stride_batch", ctypes.c_int64), ("stride_head", ctypes.c_int64),
                ("stride_token", ctypes.c_int64)]


class sparsp_rotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "pairing", "rot_begin", "pairs_t", "pairs_h", "pairs_w", "len_t",
                                              "len_h", "len_w")]


class sparsp_norm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("rows_per_group", ctypes.c_int64), ("stride_x", ctypes.c_int64),
                ("stride_y", ctypes.c_int64), ("dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("weight_dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class sparsp_ffn(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("stride_x", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_w", ctypes.c_int64), ("dim", ctypes.c_int32), ("hidden", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("activation", ctypes.c_int32)]


class sparsp_gated_norm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("rows_per_group", ctypes.c_int64), ("stride_x", ctypes.c_int64),
                ("stride_y", ctypes.c_int64), ("stride_n", ctypes.c_int64), ("dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("norm_y", ctypes.c_int32),
                ("norm_r", ctypes.c_int32), ("eps", ctypes.c_float)]


class sparsp_grad_list(ctypes.Structure):
    stream = None  # that make_grad_list's table was made on
    _fields_ = [("count", ctypes.c_int32), ("dtype", ctypes.c_int32), ("grads", ctypes.c_void_p),
                ("outs", ctypes.c_void_p), ("sizes", ctypes.c_void_p), ("chunks", ctypes.c_int32),
                ("ctas", ctypes.c_int32), ("in_place", ctypes.c_int32)]


class sparsp_fp4(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("stride_x", ctypes.c_int64), ("cols", ctypes.c_int32),
                ("format", ctypes.c_int32), ("exponent", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class sparsp_fp4_gemm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("stride_c", ctypes.c_int64), ("cols", ctypes.c_int32),
                ("depth", ctypes.c_int32), ("format", ctypes.c_int32), ("exponent", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            # not built yet (e.g. a fresh checkout): compile it in-tree with nvcc; if that is impossible
            # the call fails loudly -- there is no CPU fallback
            try:
                from . import build as _build
                _build.build()
            except Exception as exc:  # noqa: BLE001
                raise RuntimeError(f"{LIB_PATH} is missing and could not be built with nvcc ({exc}); "
                                   "there is no CPU fallback") from exc
        L = ctypes.CDLL(LIB_PATH)
        L.sparsp_last_error.restype = ctypes.c_char_p
        L.sparsp_launch_count.restype = ctypes.c_int64
        L.sparsp_resolve_topk.restype = ctypes.c_int32
        for name in EXPORTS:
            getattr(L, name)  # AttributeError if a declared symbol is not exported
        kinds = {"s": ctypes.POINTER(sparsp_shape), "r": ctypes.POINTER(sparsp_rotary),
                 "n": ctypes.POINTER(sparsp_norm), "m": ctypes.POINTER(sparsp_ffn),
                 "e": ctypes.POINTER(sparsp_gated_norm), "t": ctypes.POINTER(sparsp_grad_list), "q": ctypes.POINTER(sparsp_fp4), "g": ctypes.POINTER(sparsp_fp4_gemm), "p": ctypes.c_void_p,
                 "i": ctypes.c_int32, "l": ctypes.c_int64, "f": ctypes.c_float, "d": ctypes.c_double}
        for name, args in _SIGNATURES.items():
            getattr(L, name).argtypes = [kinds[a] for a in args]
        _lib = L
    return _lib


def _check(rc: int):
    if rc != SPARSP_OK:
        raise SparspError(rc, lib().sparsp_last_error().decode())


def _ptr(t):
    if t is None:
        return ctypes.c_void_p(0)
    return ctypes.c_void_p(t.data_ptr())


def _data(t):
    """Data pointer of a tensor as a plain value, None for None."""
    return None if t is None else t.data_ptr()


def _stream_handle():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream():
    # the handle itself: torch.cuda.current_stream() builds a Stream object around it, 3 us per call
    return ctypes.c_void_p(_stream_handle())


@dataclass
class Geometry:
    n_tokens: int
    n_blocks: int
    n_words: int
    n_video_blocks: int


def make_shape(heads: int, head_dim: int, grid, n_text: int, block: int, batch: int = 1,
               layout: str = "HND") -> sparsp_shape:
    """Shape for dense tensors laid out [B][H][N][d] ("HND") or [B][N][H][d] ("NHD")."""
    N = grid[0] * grid[1] * grid[2] + n_text
    if layout == "HND":
        sh, st = N * head_dim, head_dim
    elif layout == "NHD":
        sh, st = head_dim, heads * head_dim
    else:
        raise ValueError(layout)
    return sparsp_shape(batch, heads, head_dim, grid[0], grid[1], grid[2], n_text, block,
                        heads * N * head_dim, sh, st)


def sparsp_geometry(shape: sparsp_shape) -> Geometry:
    n, nb, wd, nv = ctypes.c_int64(), ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    _check(lib().sparsp_geometry(ctypes.byref(shape), ctypes.byref(n), ctypes.byref(nb), ctypes.byref(wd),
                                 ctypes.byref(nv)))
    return Geometry(n.value, nb.value, wd.value, nv.value)


def sparsp_resolve_topk(pct: int, n_video_blocks: int) -> int:
    return int(lib().sparsp_resolve_topk(ctypes.c_int32(pct), ctypes.c_int32(n_video_blocks)))


def _placement(fn, shape, n_ranks):
    g = sparsp_geometry(shape)
    out = torch.empty(g.n_blocks, dtype=torch.int32)
    _check(fn(ctypes.byref(shape), ctypes.c_int32(n_ranks), ctypes.c_void_p(out.data_ptr())))
    return out


def sparsp_placement_contiguous(shape: sparsp_shape, n_ranks: int) -> torch.Tensor:
    return _placement(lib().sparsp_placement_contiguous, shape, n_ranks)


def sparsp_placement_periodic(shape: sparsp_shape, n_ranks: int) -> torch.Tensor:
    return _placement(lib().sparsp_placement_periodic, shape, n_ranks)


def sparsp_placement_permutation(shape: sparsp_shape, n_ranks: int, rank_of_block: torch.Tensor):
    """-> (block_of_slot int32 [NB], token_offset_of_slot int64 [NB+1], first_slot_of_rank int32 [P+1]), host."""
    g = sparsp_geometry(shape)
    rank = rank_of_block.to(torch.int32).cpu().contiguous()
    bos = torch.empty(g.n_blocks, dtype=torch.int32)
    off = torch.empty(g.n_blocks + 1, dtype=torch.int64)
    first = torch.empty(n_ranks + 1, dtype=torch.int32)
    _check(lib().sparsp_placement_permutation(ctypes.byref(shape), ctypes.c_int32(n_ranks),
                                              ctypes.c_void_p(rank.data_ptr()), ctypes.c_void_p(bos.data_ptr()),
                                              ctypes.c_void_p(off.data_ptr()), ctypes.c_void_p(first.data_ptr())))
    return bos, off, first


class sparsp_transfer(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("consumer", ctypes.c_int32), ("producer", ctypes.c_int32),
                ("round", ctypes.c_int32), ("order", ctypes.c_int32), ("head_begin", ctypes.c_int32),
                ("head_end", ctypes.c_int32), ("reserved", ctypes.c_int32), ("entry_begin", ctypes.c_int64),
                ("n_entries", ctypes.c_int64), ("byte_offset", ctypes.c_int64), ("n_bytes", ctypes.c_int64)]


def sparsp_exchange_plan(shape: sparsp_shape, n_ranks: int, cnt: torch.Tensor, seg_offset: torch.Tensor,
                         steady_chunks: int = 1, tail_chunks: int = 1):
    """-> list of sparsp_transfer (host).  cnt / seg_offset: sparsp_demand_pack's outputs (any device)."""
    c = cnt.to(torch.int32).cpu().contiguous()
    o = seg_offset.to(torch.int64).cpu().contiguous()
    n = ctypes.c_int64(0)
    args = (ctypes.byref(shape), ctypes.c_int32(n_ranks), ctypes.c_void_p(c.data_ptr()),
            ctypes.c_void_p(o.data_ptr()), ctypes.c_int32(steady_chunks), ctypes.c_int32(tail_chunks))
    rc = lib().sparsp_exchange_plan(*args, None, ctypes.c_int64(0), ctypes.byref(n))
    if rc not in (SPARSP_OK, SPARSP_ERR_CAPACITY):
        _check(rc)
    buf = (sparsp_transfer * max(n.value, 1))()
    _check(lib().sparsp_exchange_plan(*args, buf, ctypes.c_int64(n.value), ctypes.byref(n)))
    return list(buf[:n.value])


def sparsp_permute_tokens(shape, X, Y, block_of_slot, token_offset_of_slot, inverse):
    _check(lib().sparsp_permute_tokens(ctypes.byref(shape), _ptr(X), _ptr(Y), _ptr(block_of_slot),
                                       _ptr(token_offset_of_slot), ctypes.c_int32(1 if inverse else 0), _stream()))


def sparsp_sharing_histogram(shape, mask, rank_of_block, n_ranks, hist):
    _check(lib().sparsp_sharing_histogram(ctypes.byref(shape), _ptr(mask), _ptr(rank_of_block),
                                          ctypes.c_int32(n_ranks), _ptr(hist), _stream()))


def sparsp_workspace_bytes(shape: sparsp_shape, n_ranks: int) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_workspace_bytes(ctypes.byref(shape), ctypes.c_int32(n_ranks), ctypes.byref(out)))
    return out.value


def make_workspace(shape: sparsp_shape, n_ranks: int, device="cuda") -> torch.Tensor:
    """Allocates a workspace (torch owns the memory) with its header zero-filled."""
    ws = torch.empty(sparsp_workspace_bytes(shape, n_ranks), dtype=torch.uint8, device=device)
    ws[:256].zero_()
    return ws


def sparsp_block_mask(shape, Q, K, topk_video, mask, kv_list, kv_count, pooled_q, pooled_k, workspace):
    _check(lib().sparsp_block_mask(shape, _data(Q), _data(K), topk_video, _data(mask), _data(kv_list),
                                   _data(kv_count), _data(pooled_q), _data(pooled_k), _data(workspace),
                                   _stream_handle()))


def sparsp_block_mask_cdf(shape, Q, K, tau, score_scale, mask, kv_count, pooled_q, pooled_k, workspace):
    _check(lib().sparsp_block_mask_cdf(shape, _data(Q), _data(K), tau, score_scale, _data(mask), _data(kv_count),
                                       _data(pooled_q), _data(pooled_k), _data(workspace), _stream_handle()))


def sparsp_demand_pack(shape, mask, rank_of_block, n_ranks, flags, K, V, union_mask, cnt, seg_offset,
                       seg_total, volume_bytes, packed, packed_capacity_bytes, dst_base_bytes, workspace):
    _check(lib().sparsp_demand_pack(shape, _data(mask), _data(rank_of_block), n_ranks, flags, _data(K), _data(V),
                                    _data(union_mask), _data(cnt), _data(seg_offset), _data(seg_total),
                                    _data(volume_bytes), _data(packed), packed_capacity_bytes, _data(dst_base_bytes),
                                    _data(workspace), _stream_handle()))


def sparsp_demand_plan_noalloc(shape, mask, rank_of_block, n_ranks, flags, union_mask, cnt, seg_offset, seg_total,
                               volume_bytes):
    """Planning half of sparsp_demand_pack for callers that cannot allocate device memory: no workspace
    argument, the scratch is a small array inside the library.  Outputs as for SPARSP_PLAN_ONLY."""
    _check(lib().sparsp_demand_plan_noalloc(shape, _data(mask), _data(rank_of_block), n_ranks, flags,
                                            _data(union_mask), _data(cnt), _data(seg_offset), _data(seg_total),
                                            _data(volume_bytes), _stream_handle()))


def sparsp_sparse_attn_fwd(shape, Q, K, V, mask, softmax_scale, O, lse, workspace):
    _check(lib().sparsp_sparse_attn_fwd(shape, _data(Q), _data(K), _data(V), _data(mask), softmax_scale, _data(O),
                                        _data(lse), _data(workspace), _stream_handle()))


def sparsp_sparse_attn_fwd_packed(shape, Q, K, V, mask, rank_of_block, n_ranks, consumer, union_mask, seg_offset,
                                  seg_total, packed, packed_capacity_bytes, dst_base_bytes, softmax_scale, O, lse,
                                  workspace):
    _check(lib().sparsp_sparse_attn_fwd_packed(shape, _data(Q), _data(K), _data(V), _data(mask), _data(rank_of_block),
                                               n_ranks, consumer, _data(union_mask), _data(seg_offset),
                                               _data(seg_total), _data(packed), packed_capacity_bytes,
                                               _data(dst_base_bytes), softmax_scale, _data(O), _data(lse),
                                               _data(workspace), _stream_handle()))


def sparsp_hop_mask(shape, mask, rank_of_block, n_ranks, consumer, producer, hop_mask):
    _check(lib().sparsp_hop_mask(shape, _data(mask), _data(rank_of_block), n_ranks, consumer, producer,
                                 _data(hop_mask), _stream_handle()))


def sparsp_hop_chunk_mask(shape, mask, rank_of_block, n_ranks, consumer, producer, head_begin, head_end, hop_mask):
    _check(lib().sparsp_hop_chunk_mask(shape, _data(mask), _data(rank_of_block), n_ranks, consumer, producer,
                                       head_begin, head_end, _data(hop_mask), _stream_handle()))


def sparsp_attn_merge(shape, O_a, lse_a, O_b, lse_b, O, lse):
    _check(lib().sparsp_attn_merge(shape, _data(O_a), _data(lse_a), _data(O_b), _data(lse_b), _data(O), _data(lse),
                                   _stream_handle()))


def sparsp_attn_merge_rows(shape, O_a, lse_a, O_b, lse_b, O, lse, rank_of_block, n_ranks, consumer, head_begin,
                           head_end):
    _check(lib().sparsp_attn_merge_rows(shape, _data(O_a), _data(lse_a), _data(O_b), _data(lse_b), _data(O),
                                        _data(lse), _data(rank_of_block), n_ranks, consumer, head_begin, head_end,
                                        _stream_handle()))


def _addr(x):
    """Raw address: an int, a torch tensor (its data pointer) or None."""
    if x is None:
        return ctypes.c_void_p(0)
    if isinstance(x, int):
        return ctypes.c_void_p(x)
    return ctypes.c_void_p(x.data_ptr())


def _stream_of(stream):
    """cudaStream_t of a torch stream (None: the current stream; 0: no stream, host-memory endpoints)."""
    if stream is None:
        return _stream()
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def sparsp_pack_segment(shape, union_mask, rank_of_block, n_ranks, consumer, producer, cnt, seg_offset, K, V, dst,
                        dst_capacity_bytes, workspace):
    """dst: a tensor or a raw device address (a slot of the producer's window)."""
    _check(lib().sparsp_pack_segment(shape, _data(union_mask), _data(rank_of_block), n_ranks, consumer, producer,
                                     _data(cnt), _data(seg_offset), _data(K), _data(V), _addr(dst),
                                     dst_capacity_bytes, _data(workspace), _stream_handle()))


def sparsp_xchg_flag_bytes(n_ranks: int, window: int) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_xchg_flag_bytes(ctypes.c_int32(n_ranks), ctypes.c_int32(window), ctypes.byref(out)))
    return out.value


def sparsp_xchg_export(n_ranks, rank, window, slot_bytes, slots, flag_page, wait_limit_us, flags=0):
    """-> endpoint handle.  slots / flag_page: tensors or raw addresses."""
    h = ctypes.c_void_p()
    _check(lib().sparsp_xchg_export(ctypes.c_int32(n_ranks), ctypes.c_int32(rank), ctypes.c_int32(window),
                                    ctypes.c_int64(slot_bytes), _addr(slots), _addr(flag_page),
                                    ctypes.c_int64(wait_limit_us), ctypes.c_int32(flags), ctypes.byref(h)))
    return h


def sparsp_xchg_connect(x, peer, peer_slots):
    _check(lib().sparsp_xchg_connect(x, ctypes.c_int32(peer), _addr(peer_slots)))


def sparsp_xchg_fence(x):
    _check(lib().sparsp_xchg_fence(x))


def sparsp_xchg_acquire(x, use):
    """-> (slot index, slot address)"""
    slot, ptr = ctypes.c_int32(), ctypes.c_void_p()
    _check(lib().sparsp_xchg_acquire(x, ctypes.c_int64(use), ctypes.byref(slot), ctypes.byref(ptr)))
    return slot.value, ptr.value


def sparsp_xchg_publish(x, use, stream=None):
    _check(lib().sparsp_xchg_publish(x, ctypes.c_int64(use), _stream_of(stream)))


def sparsp_xchg_fetch(x, producer, use, src_offset, dst, n_bytes, copy_stream=None):
    _check(lib().sparsp_xchg_fetch(x, ctypes.c_int32(producer), ctypes.c_int64(use), ctypes.c_int64(src_offset),
                                   _addr(dst), ctypes.c_int64(n_bytes), _stream_of(copy_stream)))


def sparsp_xchg_release(x, producer, use, copy_stream=None):
    _check(lib().sparsp_xchg_release(x, ctypes.c_int32(producer), ctypes.c_int64(use), _stream_of(copy_stream)))


def sparsp_xchg_stats(x) -> dict:
    out = (ctypes.c_int64 * 8)()
    _check(lib().sparsp_xchg_stats(x, out))
    names = ("publications", "fetches", "releases", "acquires_that_waited", "bytes_fetched", "us_waiting_for_release",
             "us_waiting_for_publish", "timeouts")
    return dict(zip(names, [int(v) for v in out]))


def sparsp_xchg_destroy(x):
    _check(lib().sparsp_xchg_destroy(x))


# ---- token-wise operators of a layer ----
def _dtype(dtype) -> int:
    if dtype not in DTYPES:
        raise ValueError(f"unsupported dtype {dtype}")
    return DTYPES[dtype]


def make_rotary(pairs, lengths, pairing: str = "interleaved", rot_begin: int = 0,
                dtype=torch.bfloat16) -> sparsp_rotary:
    """pairs, lengths: channel pairs and positions of the t, h and w coordinates."""
    return sparsp_rotary(_dtype(dtype), PAIRINGS[pairing], rot_begin, *pairs, *lengths)


def sparsp_rotary_frequencies(n_pairs: int, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                              original_length: float = 4096.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """-> (float64 [n_pairs] on the host, amplitude)"""
    out = torch.empty(max(n_pairs, 0), dtype=torch.float64)
    amplitude = ctypes.c_double()
    _check(lib().sparsp_rotary_frequencies(n_pairs, theta, SCALINGS[scaling], factor, original_length, beta_fast,
                                           beta_slow, out.data_ptr() or None, ctypes.addressof(amplitude)))
    return out, amplitude.value


def sparsp_rotary_table_bytes(rotary: sparsp_rotary) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_rotary_table_bytes(rotary, ctypes.addressof(out)))
    return out.value


def sparsp_rotary_table(rotary, inv_freq, amplitude, table):
    _check(lib().sparsp_rotary_table(rotary, _data(inv_freq), amplitude, _data(table), _stream_handle()))


def make_rotary_table(rotary: sparsp_rotary, inv_freq: torch.Tensor, amplitude: float = 1.0,
                      device="cuda") -> torch.Tensor:
    """Allocates and fills the table; inv_freq: frequencies of all pairs in their order (any device)."""
    table = torch.empty(sparsp_rotary_table_bytes(rotary) // 4, dtype=torch.float32, device=device)
    freq = inv_freq.to(device=device, dtype=torch.float64).contiguous()
    if freq.numel() != rotary.pairs_t + rotary.pairs_h + rotary.pairs_w:
        raise ValueError(f"{freq.numel()} frequencies for {rotary.pairs_t + rotary.pairs_h + rotary.pairs_w} pairs")
    sparsp_rotary_table(rotary, freq, amplitude, table)
    return table


def make_status_workspace(device="cuda") -> torch.Tensor:
    """A workspace of the status words alone."""
    return torch.zeros(256, dtype=torch.uint8, device=device)


def _positions_stride(shape: sparsp_shape, positions) -> int:
    """Elements from one batch item's positions to the next's, 0 where all have the same."""
    if not isinstance(positions, torch.Tensor):
        return 0
    N, dims = shape.grid_t * shape.grid_h * shape.grid_w + shape.n_text, positions.shape
    if positions.dtype is not torch.int32:
        raise ValueError(f"positions have to be int32, not {positions.dtype}")
    if dims != (N, 3) and dims != (shape.batch, N, 3) and dims != (1, N, 3):
        raise ValueError(f"positions {tuple(dims)} for {shape.batch} x {N} tokens")
    one = len(dims) == 2 or dims[0] == 1
    if positions.is_contiguous():  # (asked first: the rest costs a call of one token half a microsecond)
        return 0 if one else 3 * N
    if positions.stride(-1) != 1 or (N > 1 and positions.stride(-2) != 3):
        raise ValueError("a token's positions and the tokens have to follow one another in memory")
    return 0 if one else positions.stride(0)


def sparsp_rotary_apply(shape, rotary, table, positions, origin, Q, K, Q_out, K_out, inverse, workspace):
    """positions: int32 [N][3] or [1][N][3] (for every batch item) or [B][N][3], or None; origin: first (t, h, w) without
    them."""
    _check(lib().sparsp_rotary_apply(shape, rotary, _data(table), _data(positions), _positions_stride(shape, positions),
                                     *origin, _data(Q), _data(K), _data(Q_out), _data(K_out), 1 if inverse else 0,
                                     _data(workspace), _stream_handle()))


def make_norm(rows: int, dim: int, rows_per_group: int = 0, eps: float = 1e-5, dtype=torch.bfloat16, weight_dtype=None,
              stride_x: int = 0, stride_y: int = 0) -> sparsp_norm:
    """Strides of 0: contiguous rows.  weight_dtype None: dtype."""
    return sparsp_norm(rows, rows_per_group, stride_x or dim, stride_y or dim, dim, _dtype(dtype),
                       _dtype(dtype if weight_dtype is None else weight_dtype), eps)


def sparsp_layer_norm_fwd(norm, X, weight, bias, Y, mean, rstd):
    _check(lib().sparsp_layer_norm_fwd(norm, _data(X), _data(weight), _data(bias), _data(Y), _data(mean), _data(rstd),
                                       _stream_handle()))


def sparsp_layer_norm_workspace_bytes(norm: sparsp_norm) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_layer_norm_workspace_bytes(norm, ctypes.addressof(out)))
    return out.value


def make_norm_workspace(norm: sparsp_norm, device="cuda") -> torch.Tensor:
    ws = torch.empty(sparsp_layer_norm_workspace_bytes(norm), dtype=torch.uint8, device=device)
    ws[:256].zero_()
    return ws


def sparsp_layer_norm_bwd(norm, dY, X, weight, mean, rstd, dX, dweight, dbias, workspace):
    _check(lib().sparsp_layer_norm_bwd(norm, _data(dY), _data(X), _data(weight), _data(mean), _data(rstd), _data(dX),
                                       _data(dweight), _data(dbias), _data(workspace), _stream_handle()))


def make_ffn(tokens: int, dim: int, hidden: int, activation: str = "silu", dtype=torch.bfloat16, stride_x: int = 0,
             stride_h: int = 0, stride_w: int = 0) -> sparsp_ffn:
    """Strides of 0: contiguous rows."""
    return sparsp_ffn(tokens, stride_x or dim, stride_h or hidden, stride_w or dim, dim, hidden, _dtype(dtype),
                      ACTIVATIONS[activation])


def sparsp_gated_ffn_workspace_bytes(ffn: sparsp_ffn, backward: bool) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_gated_ffn_workspace_bytes(ffn, 1 if backward else 0, ctypes.addressof(out)))
    return out.value


def make_ffn_workspace(ffn: sparsp_ffn, backward: bool = True, device="cuda") -> torch.Tensor:
    ws = torch.empty(sparsp_gated_ffn_workspace_bytes(ffn, backward), dtype=torch.uint8, device=device)
    ws[:256].zero_()
    return ws


def sparsp_gated_ffn_fwd(ffn, X, Wgate, Wup, H, gate, up, workspace):
    _check(lib().sparsp_gated_ffn_fwd(ffn, _data(X), _data(Wgate), _data(Wup), _data(H), _data(gate), _data(up),
                                      _data(workspace), _stream_handle()))


def sparsp_gated_ffn_bwd(ffn, dH, X, Wgate, Wup, gate, up, dX, dWgate, dWup, workspace):
    _check(lib().sparsp_gated_ffn_bwd(ffn, _data(dH), _data(X), _data(Wgate), _data(Wup), _data(gate), _data(up),
                                      _data(dX), _data(dWgate), _data(dWup), _data(workspace), _stream_handle()))


# ---- the residual step between two blocks ----
def make_gated_norm(rows: int, dim: int, rows_per_group: int = 0, norm_y: str = "none", norm_r: str = "layer",
                    eps: float = 1e-5, dtype=torch.bfloat16, weight_dtype=None, stride_x: int = 0, stride_y: int = 0,
                    stride_n: int = 0) -> sparsp_gated_norm:
    """Strides of 0: contiguous rows.  weight_dtype None: dtype."""
    return sparsp_gated_norm(rows, rows_per_group, stride_x or dim, stride_y or dim, stride_n or dim, dim, _dtype(dtype),
                             _dtype(dtype if weight_dtype is None else weight_dtype), NORMS[norm_y], NORMS[norm_r], eps)


def sparsp_gated_norm_fwd(step, X, Y, gate, weight_y, bias_y, weight_r, bias_r, R, N, stats_y, stats_r):
    _check(lib().sparsp_gated_norm_fwd(step, _data(X), _data(Y), _data(gate), _data(weight_y), _data(bias_y),
                                       _data(weight_r), _data(bias_r), _data(R), _data(N), _data(stats_y),
                                       _data(stats_r), _stream_handle()))


def sparsp_gated_norm_workspace_bytes(step: sparsp_gated_norm) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_gated_norm_workspace_bytes(step, ctypes.addressof(out)))
    return out.value


def make_gated_norm_workspace(step: sparsp_gated_norm, device="cuda") -> torch.Tensor:
    ws = torch.empty(sparsp_gated_norm_workspace_bytes(step), dtype=torch.uint8, device=device)
    ws[:256].zero_()
    return ws


def sparsp_gated_norm_bwd(step, dN, dR, R, Y, gate, weight_y, bias_y, weight_r, stats_y, stats_r, dX, dY, dgate, dweight_y,
                          dbias_y, dweight_r, dbias_r, workspace):
    _check(lib().sparsp_gated_norm_bwd(step, _data(dN), _data(dR), _data(R), _data(Y), _data(gate), _data(weight_y),
                                       _data(bias_y), _data(weight_r), _data(stats_y), _data(stats_r), _data(dX),
                                       _data(dY), _data(dgate), _data(dweight_y), _data(dbias_y), _data(dweight_r),
                                       _data(dbias_r), _data(workspace), _stream_handle()))


# ---- the norm of a list of gradients, and clipping ----
def sparsp_grad_table_bytes(grad_list: sparsp_grad_list) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_grad_table_bytes(grad_list, ctypes.addressof(out)))
    return out.value


def sparsp_grad_table(grad_list: sparsp_grad_list, table: torch.Tensor):
    """table: uint8 on the host"""
    _check(lib().sparsp_grad_table(grad_list, _data(table)))


def make_grad_list(grads, outs=None) -> sparsp_grad_list:
    """grads: contiguous tensors of one type on one device; outs: where the clipped ones go, None = in place.  The list keeps
    them and its table alive; it is made once, outside of a graph's capture, and serves as long as they stay where they are:
    once for gradients that are kept and zeroed, each time for those that are made anew (about 0.6 us a tensor on the host).
    It may be dropped while calls on any stream still run; what a captured graph replays needs it for as long as the graph."""
    grads, outs = list(grads), None if outs is None else list(outs)
    if outs is not None and len(outs) != len(grads):
        raise ValueError(f"{len(outs)} outputs for {len(grads)} gradients")
    n = len(grads)
    dtype, device = (grads[0].dtype, grads[0].device) if n else (torch.bfloat16, torch.device("cuda"))
    sizes = [t.numel() for t in grads]
    for tensors in (grads, outs or []):
        for i, t in enumerate(tensors):
            if t.dtype is not dtype or t.device != device or not t.is_contiguous() or t.numel() != sizes[i]:
                raise ValueError(f"gradient {i}: contiguous tensors of one type and device, an output as large as its gradient")
    room = ctypes.c_void_p * max(n, 1)
    addresses = room(*[t.data_ptr() for t in grads])
    to = None if outs is None else room(*[t.data_ptr() for t in outs])
    sizes = (ctypes.c_int64 * max(n, 1))(*sizes)
    out = sparsp_grad_list(n, _dtype(dtype), ctypes.addressof(addresses), None if to is None else ctypes.addressof(to),
                           ctypes.addressof(sizes), 0, 0, 0)
    table = torch.zeros(sparsp_grad_table_bytes(out), dtype=torch.uint8)
    sparsp_grad_table(out, table)
    out.table = table.to(device)
    if out.table.is_cuda:
        out.stream = torch._C._cuda_getCurrentRawStream(out.table.device.index)
    out.kept = (grads, outs, addresses, to, sizes)
    return out


def sparsp_grad_workspace_bytes() -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_grad_workspace_bytes(ctypes.addressof(out)))
    return out.value


def make_grad_workspace(device="cuda") -> torch.Tensor:
    return torch.zeros(sparsp_grad_workspace_bytes(), dtype=torch.uint8, device=device)


def grad_square_sum(workspace) -> torch.Tensor:
    """The sum of squares in the workspace, float64 [1]: what ranks that share a norm add up."""
    return workspace[256:264].view(torch.float64)


def _grad_table_on(grad_list, stream):
    """The list's table for a call on `stream`: its memory is not given out again before what that stream has now is done."""
    if grad_list.stream is not None and stream != grad_list.stream:
        grad_list.table.record_stream(torch.cuda.current_stream())
    return _data(grad_list.table)


def sparsp_grad_squares(grad_list, workspace, accumulate=False):
    stream = _stream_handle()
    _check(lib().sparsp_grad_squares(grad_list, _grad_table_on(grad_list, stream), 1 if accumulate else 0, _data(workspace),
                                     stream))


def sparsp_grad_clip(grad_list, max_norm, norm, workspace):
    stream = _stream_handle()
    _check(lib().sparsp_grad_clip(grad_list, _grad_table_on(grad_list, stream), max_norm, _data(norm), _data(workspace),
                                  stream))


# ---- 4-bit operands and their product ----
def make_fp4(rows: int, cols: int, format: str = "mxfp4", exponent: int = 0, dtype=torch.bfloat16,
             stride_x: int = 0) -> sparsp_fp4:
    """stride_x 0: contiguous rows."""
    return sparsp_fp4(rows, stride_x or cols, cols, FP4_FORMATS[format], exponent, _dtype(dtype))


def sparsp_fp4_scales_bytes(fp4: sparsp_fp4) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_fp4_scales_bytes(fp4, ctypes.addressof(out)))
    return out.value


def make_fp4_operand(fp4: sparsp_fp4, device="cuda"):
    """-> (codes uint8 [rows][cols / 2], scales uint8), to be filled by sparsp_fp4_quantize"""
    return (torch.empty(fp4.rows, fp4.cols // 2, dtype=torch.uint8, device=device),
            torch.empty(sparsp_fp4_scales_bytes(fp4), dtype=torch.uint8, device=device))


def sparsp_fp4_quantize(fp4, X, codes, scales, values):
    _check(lib().sparsp_fp4_quantize(fp4, _data(X), _data(codes), _data(scales), _data(values), _stream_handle()))


def make_fp4_product(rows: int, cols: int, depth: int, format: str = "mxfp4", exponent: int = 0, dtype=torch.bfloat16,
                     stride_c: int = 0) -> sparsp_fp4_gemm:
    """exponent: the sum of both operands' exponents; stride_c 0: contiguous rows."""
    return sparsp_fp4_gemm(rows, stride_c or cols, cols, depth, FP4_FORMATS[format], exponent, _dtype(dtype))


def sparsp_fp4_product_workspace_bytes(product: sparsp_fp4_gemm) -> int:
    out = ctypes.c_int64()
    _check(lib().sparsp_fp4_product_workspace_bytes(product, ctypes.addressof(out)))
    return out.value


def make_fp4_product_workspace(product: sparsp_fp4_gemm, device="cuda") -> torch.Tensor:
    ws = torch.empty(sparsp_fp4_product_workspace_bytes(product), dtype=torch.uint8, device=device)
    ws[:256].zero_()
    return ws


def sparsp_fp4_product(product, A, A_scales, B, B_scales, bias, C, workspace):
    _check(lib().sparsp_fp4_product(product, _data(A), _data(A_scales), _data(B), _data(B_scales), _data(bias), _data(C),
                                    _data(workspace), _stream_handle()))


def sparsp_status(workspace) -> int:
    code = ctypes.c_int32()
    _check(lib().sparsp_status(_ptr(workspace), _stream(), ctypes.byref(code)))
    return code.value


def sparsp_selftest_wait_timeout(workspace, limit_cycles: int):
    _check(lib().sparsp_selftest_wait_timeout(_ptr(workspace), ctypes.c_int64(limit_cycles), _stream()))


def sparsp_last_error() -> str:
    return lib().sparsp_last_error().decode()


def sparsp_launch_count() -> int:
    return int(lib().sparsp_launch_count())


# ---------------------------------------------------------------------------------------------
# allocation helpers (device buffers for the outputs; no arithmetic)
# ---------------------------------------------------------------------------------------------
def alloc_mask_outputs(shape: sparsp_shape, topk_video: int, device="cuda", with_list=True, with_pooled=False):
    g = sparsp_geometry(shape)
    B, H, d = shape.batch, shape.heads, shape.head_dim
    kept = topk_video + (g.n_blocks - g.n_video_blocks)
    out = dict(mask=torch.empty(B, H, g.n_blocks, g.n_words, dtype=torch.int32, device=device))
    out["kv_list"] = torch.full((B, H, g.n_blocks, kept), -1, dtype=torch.int32, device=device) if with_list else None
    out["kv_count"] = torch.empty(B, H, g.n_blocks, dtype=torch.int32, device=device) if with_list else None
    out["pooled_q"] = torch.empty(B, H, g.n_blocks, d, dtype=torch.float32, device=device) if with_pooled else None
    out["pooled_k"] = torch.empty(B, H, g.n_blocks, d, dtype=torch.float32, device=device) if with_pooled else None
    return out


def alloc_demand_outputs(shape: sparsp_shape, n_ranks: int, device="cuda"):
    g = sparsp_geometry(shape)
    B, H, P = shape.batch, shape.heads, n_ranks
    return dict(union_mask=torch.empty(B, P, H, g.n_words, dtype=torch.int32, device=device),
                cnt=torch.empty(B, P, P, H, dtype=torch.int32, device=device),
                seg_offset=torch.empty(B, P, P, H, dtype=torch.int64, device=device),
                seg_total=torch.empty(B, P, dtype=torch.int64, device=device),
                volume_bytes=torch.empty(B, P, dtype=torch.int64, device=device))
