"""MI355X (gfx950) implementation of MUSTAFAR's decode hot path (arxiv 2505.22913).

Thin ctypes binding of ``libmustafar.so``; every step of the path runs in the
library's HIP kernels. Function names mirror the C ABI in ``include/mustafar.h``;
this module only turns torch tensors into device pointers, passes the current
HIP stream and raises ``MustafarError`` on a non-zero status. torch is used for
device memory and streams only.

The library is loaded on first use; if it has not been built the call raises
(there is no CPU fallback). Build it with
``python -m paper_2505_22913_amd.build_lib`` or ``__graft_entry__.build()``.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmustafar.so")
TILE = 64
PAD = 8

OK, EINVAL, ECAPACITY, EWORKSPACE, ELAUNCH, EUNSUPPORTED, ESCRATCH = 0, -1, -2, -3, -4, -5, -6
STATIC_SCRATCH_BYTES = 32 << 20   # the static buffer of mustafar_sparse_decode_attn_static
STREAM_POISONED = 0xFFFFFFFF   # stream_len of a stream whose bulk compression gave up
LOOKBACK_POLLS = 1 << 20

_lib = None


class MustafarError(RuntimeError):
    def __init__(self, fn: str, status: int):
        super().__init__(f"{fn} failed: {status} ({strerror(status)})")
        self.status = status


class ccache_t(ctypes.Structure):
    """Mirror of ``mustafar_ccache_t``."""
    _fields_ = [("bitmaps", ctypes.c_void_p), ("offsets", ctypes.c_void_p),
                ("values", ctypes.c_void_p), ("stream_len", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("n_keep", ctypes.c_int32), ("cap_tokens", ctypes.c_int32),
                ("n_tokens", ctypes.c_int32), ("val_stride", ctypes.c_int64),
                ("group_keep", ctypes.c_int32)]


class window_t(ctypes.Structure):
    """Mirror of ``mustafar_window_t``."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("len", ctypes.c_void_p),
                ("head", ctypes.c_void_p), ("n_comp", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("W", ctypes.c_int32), ("max_len", ctypes.c_int32)]


class prune_opts_t(ctypes.Structure):
    """Mirror of ``mustafar_prune_opts_t``."""
    _fields_ = [("mode", ctypes.c_int32), ("head_keep", ctypes.c_void_p),
                ("weights", ctypes.c_void_p)]


class pages_t(ctypes.Structure):
    """Mirror of ``mustafar_pages_t``."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("state", ctypes.c_void_p), ("free_pages", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("type", ctypes.c_int32),
                ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("token_stride", ctypes.c_int64)]


class pages8_t(ctypes.Structure):
    """Mirror of ``mustafar_pages8_t``."""
    _fields_ = [("pages", pages_t), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("type", ctypes.c_int32), ("block_tokens", ctypes.c_int32)]


class rotation_t(ctypes.Structure):
    """Mirror of ``mustafar_rotation_t``."""
    _fields_ = [("rates", ctypes.c_void_p), ("rot", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("magnitude", ctypes.c_float)]


PRUNE_MAGNITUDE, PRUNE_2_4, PRUNE_OUTPUT_AWARE = 0, 1, 2
PRUNE_CHANNEL, PRUNE_CHANNEL_OUTPUT_AWARE = 3, 4
ATTN_SPARSE, ATTN_DENSE = 0, 1
FP16, BF16, E4M3, INT8 = 0, 1, 2, 3
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "base": 2, "turns": 3}
PLAN_PAGES, PLAN_TABLE, PLAN_SLOTS, PLAN_STATE = 1, 2, 4, 8   # status bits of mustafar_paged_plan
GROUP = 32  # tokens per group of per-channel value pruning

_SIGS = {
    "mustafar_keep_count": (ctypes.c_int, [ctypes.c_int, ctypes.c_float]),
    "mustafar_token_max_elems": (ctypes.c_int64, [ctypes.c_int, ctypes.c_int]),
    "mustafar_stream_capacity": (ctypes.c_int64, [ctypes.c_int, ctypes.c_int, ctypes.c_int]),
    "mustafar_ccache_init": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                            ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                            ctypes.c_float, ctypes.c_int, ctypes.c_int64]),
    "mustafar_grouped_stream_capacity": (ctypes.c_int64, [ctypes.c_int, ctypes.c_int, ctypes.c_int]),
    "mustafar_ccache_init_grouped": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                    ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                                    ctypes.c_float, ctypes.c_int, ctypes.c_int64]),
    "mustafar_compress_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int] * 3),
    "mustafar_prune_compress": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                               ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t,
                                               ctypes.c_void_p]),
    "mustafar_prune_compress_bounded": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                       ctypes.c_int, ctypes.c_uint32, ctypes.c_void_p,
                                                       ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_append_kv": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.POINTER(ccache_t),
                                          ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "mustafar_append": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                       ctypes.c_void_p]),
    "mustafar_attn_default_splits": (ctypes.c_int, [ctypes.c_int] * 5),
    "mustafar_sparse_attn_splits": (ctypes.c_int, [ctypes.POINTER(ccache_t)] * 2 + [ctypes.c_int] * 2
                                    + [ctypes.c_size_t]),
    "mustafar_attn_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int] * 6),
    "mustafar_sparse_decode_attn": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                                   ctypes.POINTER(ccache_t),
                                                   ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                   ctypes.c_void_p, ctypes.c_int, ctypes.c_float,
                                                   ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                                   ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_sparse_decode_attn_static": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                                          ctypes.POINTER(ccache_t),
                                                          ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                          ctypes.c_void_p, ctypes.c_int, ctypes.c_float,
                                                          ctypes.c_void_p, ctypes.c_int,
                                                          ctypes.c_void_p]),
    "mustafar_dense_decode_attn": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                                  ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p,
                                                  ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                                  ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                                  ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_window_init": (ctypes.c_int, [ctypes.POINTER(window_t)] + [ctypes.c_void_p] * 5
                             + [ctypes.c_int] * 5),
    "mustafar_window_prefill": (ctypes.c_int, [ctypes.POINTER(window_t), ctypes.POINTER(ccache_t),
                                               ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                               ctypes.c_void_p, ctypes.c_int,
                                               ctypes.POINTER(ctypes.c_int32), ctypes.c_void_p,
                                               ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_window_step": (ctypes.c_int, [ctypes.POINTER(window_t), ctypes.POINTER(ccache_t),
                                            ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                            ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "mustafar_window_step_weighted": (ctypes.c_int, [ctypes.POINTER(window_t), ctypes.POINTER(ccache_t),
                                                     ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                     ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                     ctypes.c_void_p]),
    "mustafar_window_key_weights": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                                   ctypes.POINTER(window_t), ctypes.c_void_p,
                                                   ctypes.c_void_p, ctypes.c_void_p]),
    "mustafar_window_decode_attn": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                                   ctypes.POINTER(ccache_t),
                                                   ctypes.POINTER(ccache_t),
                                                   ctypes.POINTER(window_t), ctypes.c_float,
                                                   ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p,
                                                   ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_window_decode_attn_scores": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                                          ctypes.POINTER(ccache_t),
                                                          ctypes.POINTER(ccache_t),
                                                          ctypes.POINTER(window_t), ctypes.c_void_p,
                                                          ctypes.c_void_p,
                                                          ctypes.c_float, ctypes.c_void_p, ctypes.c_int,
                                                          ctypes.c_void_p, ctypes.c_size_t,
                                                          ctypes.c_void_p]),
    "mustafar_window_step_grouped": (ctypes.c_int, [ctypes.POINTER(window_t), ctypes.POINTER(ccache_t),
                                                    ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                    ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                                    ctypes.c_void_p]),
    "mustafar_prune_compress_ex": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                                  ctypes.c_int, ctypes.POINTER(prune_opts_t),
                                                  ctypes.c_void_p, ctypes.c_size_t,
                                                  ctypes.c_void_p]),
    "mustafar_append_ex": (ctypes.c_int, [ctypes.POINTER(ccache_t), ctypes.c_void_p,
                                          ctypes.POINTER(prune_opts_t), ctypes.c_void_p]),
    "mustafar_query_lookahead": (ctypes.c_int, [ctypes.c_void_p] + [ctypes.c_int] * 6
                                 + [ctypes.c_void_p, ctypes.c_void_p]),
    "mustafar_paged_init": (ctypes.c_int, [ctypes.POINTER(pages_t)] + [ctypes.c_void_p] * 5
                            + [ctypes.c_int] * 7 + [ctypes.c_int64] * 3),
    "mustafar_paged_plan": (ctypes.c_int, [ctypes.POINTER(pages_t)] + [ctypes.c_void_p] * 5
                            + [ctypes.c_int] + [ctypes.c_void_p] * 2),
    "mustafar_paged_write": (ctypes.c_int, [ctypes.POINTER(pages_t), ctypes.c_void_p, ctypes.c_int64,
                                            ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                            ctypes.c_int, ctypes.c_void_p]),
    "mustafar_paged_gather": (ctypes.c_int, [ctypes.POINTER(pages_t)] + [ctypes.c_void_p] * 3
                              + [ctypes.c_int, ctypes.c_void_p]),
    "mustafar_paged_attn_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(pages_t)] + [ctypes.c_int] * 5),
    "mustafar_paged_attn": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                           ctypes.POINTER(pages_t), ctypes.c_void_p, ctypes.c_int,
                                           ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_int64,
                                           ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                           ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_paged8_init": (ctypes.c_int, [ctypes.POINTER(pages8_t)] + [ctypes.c_void_p] * 7 + [ctypes.c_int] * 9
                             + [ctypes.c_int64] * 3),
    "mustafar_paged8_write": (ctypes.c_int, [ctypes.POINTER(pages8_t), ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p,
                                             ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]),
    "mustafar_paged8_gather": (ctypes.c_int, [ctypes.POINTER(pages8_t)] + [ctypes.c_void_p] * 3
                               + [ctypes.c_int, ctypes.c_void_p]),
    "mustafar_paged8_attn_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(pages8_t)] + [ctypes.c_int] * 5),
    "mustafar_paged8_attn": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                            ctypes.POINTER(pages8_t), ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
                                            ctypes.c_float, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                            ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]),
    "mustafar_rope_rates": (ctypes.c_int, [ctypes.POINTER(ctypes.c_double), ctypes.c_int, ctypes.c_double, ctypes.c_int]
                            + [ctypes.c_double] * 4),
    "mustafar_rope": (ctypes.c_int, [ctypes.POINTER(rotation_t)] + [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int] * 2
                      + [ctypes.c_int] * 3 + [ctypes.c_void_p, ctypes.POINTER(pages_t), ctypes.c_void_p, ctypes.c_int]
                      + [ctypes.c_void_p, ctypes.c_int64] * 2 + [ctypes.c_void_p]),
    "mustafar_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "mustafar_stream_read_sink_bytes": (ctypes.c_size_t, []),
    "mustafar_stream_read": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                            ctypes.c_void_p]),
    "mustafar_attn_set_route": (ctypes.c_int, [ctypes.c_int]),
    "mustafar_attn_route": (ctypes.c_int, []),
    "mustafar_stream_mix": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int,
                                           ctypes.c_void_p, ctypes.c_void_p]),
    "mustafar_stream_chunks": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_void_p,
                                              ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p]),
}


def lib() -> ctypes.CDLL:
    """The loaded library; raises if libmustafar.so has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2505_22913_amd.build_lib` (no CPU fallback)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def strerror(status: int) -> str:
    try:
        return lib().mustafar_strerror(int(status)).decode()
    except Exception:  # noqa: BLE001 - the message is best effort
        return "unknown"


def _check(fn: str, status: int) -> None:
    if status != OK:
        raise MustafarError(fn, status)


def _dptr(t) -> int | None:
    """Device pointer of a CUDA (HIP) tensor; None for None."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("libmustafar takes device tensors only")
    return t.data_ptr()


def _stream(stream) -> int | None:
    """Raw handle of `stream`, or of torch's current stream on the current device
    (looked up without building a Stream object: 0.2 us a call against 2.7, where a
    whole decode call costs the host 7 to 12)."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # not public: another torch may lack it
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


# ---- host-only helpers --------------------------------------------------------------------
def mustafar_keep_count(d: int, sparsity: float) -> int:
    k = lib().mustafar_keep_count(int(d), float(sparsity))
    _check("mustafar_keep_count", min(k, 0))
    return k


def mustafar_token_max_elems(d: int, n_keep: int) -> int:
    return lib().mustafar_token_max_elems(int(d), int(n_keep))


def mustafar_stream_capacity(d: int, n_keep: int, cap_tokens: int) -> int:
    return lib().mustafar_stream_capacity(int(d), int(n_keep), int(cap_tokens))


def mustafar_compress_workspace_bytes(B: int, H: int, n_new: int) -> int:
    return lib().mustafar_compress_workspace_bytes(int(B), int(H), int(n_new))


def mustafar_attn_default_splits(B: int, Hq: int, Hkv: int, n_tokens: int,
                                 kind: int = ATTN_SPARSE) -> int:
    return lib().mustafar_attn_default_splits(int(B), int(Hq), int(Hkv), int(n_tokens), int(kind))


def mustafar_attn_workspace_bytes(B: int, Hq: int, Hkv: int, d: int, n_tokens: int,
                                  n_splits: int = 0) -> int:
    return lib().mustafar_attn_workspace_bytes(int(B), int(Hq), int(Hkv), int(d), int(n_tokens),
                                               int(n_splits))


# ---- the compressed cache -----------------------------------------------------------------
class CompressedCache:
    """A compressed K or V cache: device buffers (torch) plus the C descriptor.

    bitmaps u64 [B][H][cap][d/64], offsets u32 [B][H][cap][d/64],
    values fp16 bits [B][H][val_stride], stream_len u32 [B][H].

    The capacity is rounded up to a multiple of ``align`` tokens (64 by default),
    so that every stream's bitmaps and offsets start on a 256-byte boundary: the
    attention kernels read them in 32-token blocks, and a block that straddles
    an extra 128-byte line costs 5% more traffic.
    """

    def __init__(self, B: int, H: int, d: int, sparsity: float, cap_tokens: int, device="cuda",
                 grouped: bool = False, align: int = 64):
        import torch
        T = d // TILE
        cap_tokens = (int(cap_tokens) + align - 1) // align * align
        if grouped:   # per-channel pruning in groups of 32 tokens
            stride = lib().mustafar_grouped_stream_capacity(d, mustafar_keep_count(GROUP, sparsity),
                                                            cap_tokens)
        else:
            stride = mustafar_stream_capacity(d, mustafar_keep_count(d, sparsity), cap_tokens)
        stride = max(PAD, (stride + PAD - 1) // PAD * PAD)
        self.bitmaps = torch.zeros((B, H, cap_tokens, T), dtype=torch.int64, device=device)
        self.offsets = torch.zeros((B, H, cap_tokens, T), dtype=torch.int32, device=device)
        self.values = torch.zeros((B, H, stride), dtype=torch.int16, device=device)
        self.stream_len = torch.zeros((B, H), dtype=torch.int32, device=device)
        self.desc = ccache_t()
        init = "mustafar_ccache_init_grouped" if grouped else "mustafar_ccache_init"
        _check(init, getattr(lib(), init)(
            ctypes.byref(self.desc), self.bitmaps.data_ptr(), self.offsets.data_ptr(),
            self.values.data_ptr(), self.stream_len.data_ptr(), B, H, d, float(sparsity),
            cap_tokens, stride))

    @property
    def n_tokens(self) -> int:
        return self.desc.n_tokens

    @property
    def n_keep(self) -> int:
        return self.desc.n_keep

    @property
    def group_keep(self) -> int:
        return self.desc.group_keep

    @property
    def shape(self):
        return self.desc.B, self.desc.H, self.desc.d


def mustafar_prune_compress(cache: CompressedCache, x, ws=None, stream=None) -> None:
    """Append x [B][H][n_new][d] (fp16, device) to the cache, pruned and compressed."""
    import torch
    n_new = int(x.shape[2])
    need = mustafar_compress_workspace_bytes(cache.desc.B, cache.desc.H, n_new)
    if ws is None:
        ws = torch.empty(max(need, 4), dtype=torch.uint8, device=x.device)
    _check("mustafar_prune_compress", lib().mustafar_prune_compress(
        ctypes.byref(cache.desc), _dptr(x), n_new, _dptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def mustafar_prune_compress_bounded(cache: CompressedCache, x, max_polls: int, ws=None,
                                    stream=None) -> None:
    """mustafar_prune_compress with the caller's bound on a chunk's look-back polls."""
    import torch
    n_new = int(x.shape[2])
    need = mustafar_compress_workspace_bytes(cache.desc.B, cache.desc.H, n_new)
    if ws is None:
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    _check("mustafar_prune_compress_bounded", lib().mustafar_prune_compress_bounded(
        ctypes.byref(cache.desc), _dptr(x), n_new, int(max_polls), _dptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def compress_status(ws) -> int:
    """The status word a bulk compression left at the start of its workspace: 0 if
    every stream was compressed, nonzero if a stream was poisoned (synchronises)."""
    return int(ws[:4].view(dtype=__import__("torch").int32).item())


def mustafar_append_kv(Kc: CompressedCache, Vc: CompressedCache, k_new, v_new, stream=None) -> None:
    """Append one decode step's key and value per stream, [B][H][d] fp16 each, in one launch."""
    _check("mustafar_append_kv", lib().mustafar_append_kv(ctypes.byref(Kc.desc), ctypes.byref(Vc.desc),
                                                          _dptr(k_new), _dptr(v_new), _stream(stream)))


def mustafar_append(cache: CompressedCache, x_new, stream=None) -> None:
    """Append one token per stream, x_new [B][H][d] (fp16, device)."""
    _check("mustafar_append", lib().mustafar_append(ctypes.byref(cache.desc), _dptr(x_new),
                                                    _stream(stream)))


def _prune_opts(mode, head_keep, weights):
    """(prune_opts_t, keep-alive objects) for the _ex calls."""
    o = prune_opts_t()
    o.mode = int(mode)
    keep = None
    if head_keep is not None:
        keep = (ctypes.c_int32 * len(head_keep))(*[int(v) for v in head_keep])
        o.head_keep = ctypes.cast(keep, ctypes.c_void_p)
    o.weights = _dptr(weights)
    return o, keep


def mustafar_prune_compress_ex(cache: CompressedCache, x, mode: int = 0, head_keep=None,
                               weights=None, ws=None, stream=None) -> None:
    """mustafar_prune_compress under a pruner variant (PRUNE_MAGNITUDE with optional
    per-head counts, PRUNE_2_4, PRUNE_OUTPUT_AWARE with fp32 weights [B][H][n_new][d];
    on per-channel caches PRUNE_CHANNEL, PRUNE_CHANNEL_OUTPUT_AWARE with fp32 token
    weights [B][H][n_new])."""
    import torch
    n_new = int(x.shape[2])
    need = mustafar_compress_workspace_bytes(cache.desc.B, cache.desc.H, n_new)
    if ws is None:
        ws = torch.empty(max(need, 4), dtype=torch.uint8, device=x.device)
    o, _keep = _prune_opts(mode, head_keep, weights)
    _check("mustafar_prune_compress_ex", lib().mustafar_prune_compress_ex(
        ctypes.byref(cache.desc), _dptr(x), n_new, ctypes.byref(o), _dptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def mustafar_append_ex(cache: CompressedCache, x_new, mode: int = 0, head_keep=None, weights=None,
                       stream=None) -> None:
    """mustafar_append under a pruner variant (weights fp32 [B][H][d] when output-aware)."""
    o, _keep = _prune_opts(mode, head_keep, weights)
    _check("mustafar_append_ex", lib().mustafar_append_ex(
        ctypes.byref(cache.desc), _dptr(x_new), ctypes.byref(o), _stream(stream)))


def mustafar_query_lookahead(q, Hkv: int, L: int = 32, out=None, stream=None):
    """Output-aware channel weights from queries q [B][Hq][n_q][d] fp16: fp32
    [B][Hkv][n_q][d]."""
    import torch
    B, Hq, n_q, d = (int(s) for s in q.shape)
    if out is None:
        out = torch.empty((B, Hkv, n_q, d), dtype=torch.float32, device=q.device)
    _check("mustafar_query_lookahead", lib().mustafar_query_lookahead(
        _dptr(q), B, Hq, int(Hkv), n_q, d, int(L), _dptr(out), _stream(stream)))
    return out


def _attn_ws(B, Hq, Hkv, d, n, n_splits, ws, device):
    import torch
    need = mustafar_attn_workspace_bytes(B, Hq, Hkv, d, n, n_splits)
    if ws is None:
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=device)
    return ws


def mustafar_sparse_attn_splits(Kc: CompressedCache, Vc: CompressedCache, Hq: int, window: bool, ws) -> int:
    """Segments that a sparse call with n_splits = 0 and this workspace takes."""
    n = lib().mustafar_sparse_attn_splits(ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), int(Hq), int(bool(window)),
                                          ws.numel() * ws.element_size())
    _check("mustafar_sparse_attn_splits", min(n, 0))
    return n


def mustafar_sparse_decode_attn(q, Kc: CompressedCache, Vc: CompressedCache, k_tail=None,
                                v_tail=None, scale: float = 0.0, out=None, n_splits: int = 0,
                                ws=None, stream=None):
    """Algorithm 1: attention of q [B][Hq][d] over the compressed caches plus the dense
    window [B][Hkv][n_tail][d]. Returns out [B][Hq][d] fp16."""
    import torch
    B, Hq, d = (int(s) for s in q.shape)
    Hkv = Kc.desc.H
    n_tail = 0 if k_tail is None else int(k_tail.shape[2])
    if out is None:
        out = torch.empty((B, Hq, d), dtype=torch.float16, device=q.device)
    ws = _attn_ws(B, Hq, Hkv, d, Kc.n_tokens, n_splits, ws, q.device)
    _check("mustafar_sparse_decode_attn", lib().mustafar_sparse_decode_attn(
        _dptr(q), B, Hq, ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), _dptr(k_tail),
        _dptr(v_tail), n_tail, float(scale), _dptr(out), int(n_splits), _dptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))
    return out


def mustafar_sparse_decode_attn_static(q, Kc: CompressedCache, Vc: CompressedCache, k_tail=None,
                                       v_tail=None, scale: float = 0.0, out=None, n_splits: int = 0,
                                       stream=None):
    """mustafar_sparse_decode_attn with its partials in the library's static device
    buffer (no workspace; for callers that cannot allocate). out may be preallocated."""
    import torch
    B, Hq, d = (int(s) for s in q.shape)
    n_tail = 0 if k_tail is None else int(k_tail.shape[2])
    if out is None:
        out = torch.empty((B, Hq, d), dtype=torch.float16, device=q.device)
    _check("mustafar_sparse_decode_attn_static", lib().mustafar_sparse_decode_attn_static(
        _dptr(q), B, Hq, ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), _dptr(k_tail), _dptr(v_tail),
        n_tail, float(scale), _dptr(out), int(n_splits), _stream(stream)))
    return out


def mustafar_dense_decode_attn(q, k, v, scale: float = 0.0, out=None, n_splits: int = 0, ws=None,
                               stream=None):
    """Dense baseline: q [B][Hq][d] over k, v [B][Hkv][N][d] fp16. Returns out fp16."""
    import torch
    B, Hq, d = (int(s) for s in q.shape)
    Hkv, N = int(k.shape[1]), int(k.shape[2])
    if out is None:
        out = torch.empty((B, Hq, d), dtype=torch.float16, device=q.device)
    ws = _attn_ws(B, Hq, Hkv, d, N, n_splits, ws, q.device)
    _check("mustafar_dense_decode_attn", lib().mustafar_dense_decode_attn(
        _dptr(q), B, Hq, Hkv, _dptr(k), _dptr(v), N, d, float(scale), _dptr(out), int(n_splits),
        _dptr(ws), ws.numel() * ws.element_size(), _stream(stream)))
    return out


# ---- the dense local window (lifecycle) -------------------------------------------------
class DenseWindow:
    """The dense window of the W most recent tokens of every stream: ring slots
    k, v [B][H][W][d] fp16 and int32 device state len, head, n_comp [B]."""

    def __init__(self, B: int, H: int, d: int, W: int, device="cuda"):
        import torch
        self.k = torch.zeros((B, H, W, d), dtype=torch.float16, device=device)
        self.v = torch.zeros((B, H, W, d), dtype=torch.float16, device=device)
        self.len = torch.zeros(B, dtype=torch.int32, device=device)
        self.head = torch.zeros(B, dtype=torch.int32, device=device)
        self.n_comp = torch.zeros(B, dtype=torch.int32, device=device)
        self.desc = window_t()
        _check("mustafar_window_init", lib().mustafar_window_init(
            ctypes.byref(self.desc), self.k.data_ptr(), self.v.data_ptr(), self.len.data_ptr(),
            self.head.data_ptr(), self.n_comp.data_ptr(), B, H, d, W, 0))

    @property
    def W(self) -> int:
        return self.desc.W

    @property
    def max_len(self) -> int:
        return self.desc.max_len


def mustafar_window_prefill(win: DenseWindow, Kc: CompressedCache, Vc: CompressedCache, x_k, x_v,
                            seq_len, ws=None, stream=None) -> None:
    """Prompts of seq_len[b] tokens (host ints) in x_k, x_v [B][H][n_max][d] fp16: the
    tokens before each entry's last min(seq_len[b], W) are compressed, the rest fill
    its window."""
    import torch
    n_max = int(x_k.shape[2])
    lens = (ctypes.c_int32 * len(seq_len))(*[int(n) for n in seq_len])
    need = mustafar_compress_workspace_bytes(win.desc.B, win.desc.H, max(n_max, 1))  # every entry at once
    if ws is None:
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=x_k.device)
    _check("mustafar_window_prefill", lib().mustafar_window_prefill(
        ctypes.byref(win.desc), ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), _dptr(x_k),
        _dptr(x_v), n_max, lens, _dptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def mustafar_window_step(win: DenseWindow, Kc: CompressedCache, Vc: CompressedCache, k_new, v_new,
                         active=None, stream=None) -> None:
    """One decode step: k_new, v_new [B][H][d] enter the windows of the active entries
    (active: int32 device [B] or None); full windows first hand their oldest token
    to the compressed caches."""
    _check("mustafar_window_step", lib().mustafar_window_step(
        ctypes.byref(win.desc), ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), _dptr(k_new),
        _dptr(v_new), _dptr(active), _stream(stream)))


def mustafar_window_step_weighted(win: DenseWindow, Kc: CompressedCache, Vc: CompressedCache, k_new,
                                  v_new, kacc, active=None, stream=None) -> None:
    """mustafar_window_step whose leaving key is pruned output-aware with its window
    slot's weights in kacc [B][H][W][d] (fp32, device); the new token's weights start
    at 0."""
    _check("mustafar_window_step_weighted", lib().mustafar_window_step_weighted(
        ctypes.byref(win.desc), ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), _dptr(k_new),
        _dptr(v_new), _dptr(active), _dptr(kacc), _stream(stream)))


def mustafar_window_key_weights(q, win: DenseWindow, kacc, active=None, stream=None) -> None:
    """kacc[b][h][slot] += |q| of the query heads of kv-head h (one after the other, in
    fp32) for the newest 32 window tokens of every active entry (active: int32 device
    [B] or None for all); q [B][Hq][d] fp16."""
    B, Hq, _ = (int(s) for s in q.shape)
    _check("mustafar_window_key_weights", lib().mustafar_window_key_weights(
        _dptr(q), B, Hq, ctypes.byref(win.desc), _dptr(active), _dptr(kacc), _stream(stream)))


def mustafar_window_decode_attn(q, Kc: CompressedCache, Vc: CompressedCache, win: DenseWindow,
                                scale: float = 0.0, out=None, n_splits: int = 0, ws=None,
                                stream=None):
    """Algorithm 1 per batch entry over its compressed tokens and its window."""
    import torch
    B, Hq, d = (int(s) for s in q.shape)
    if out is None:
        out = torch.empty((B, Hq, d), dtype=torch.float16, device=q.device)
    ws = _attn_ws(B, Hq, Kc.desc.H, d, Kc.n_tokens, n_splits, ws, q.device)
    _check("mustafar_window_decode_attn", lib().mustafar_window_decode_attn(
        _dptr(q), B, Hq, ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), ctypes.byref(win.desc),
        float(scale), _dptr(out), int(n_splits), _dptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))
    return out


def mustafar_window_decode_attn_scores(q, Kc: CompressedCache, Vc: CompressedCache,
                                       win: DenseWindow, acc, scale: float = 0.0, out=None,
                                       n_splits: int = 0, ws=None, active=None, stream=None):
    """mustafar_window_decode_attn, then acc [B][H][W] (fp32, device) += the attention
    probability, summed over each kv-head's query heads, of every window token
    younger than 32 steps, for the active entries (active: int32 device [B] or None)."""
    import torch
    B, Hq, d = (int(s) for s in q.shape)
    if out is None:
        out = torch.empty((B, Hq, d), dtype=torch.float16, device=q.device)
    ws = _attn_ws(B, Hq, Kc.desc.H, d, Kc.n_tokens, n_splits, ws, q.device)
    _check("mustafar_window_decode_attn_scores", lib().mustafar_window_decode_attn_scores(
        _dptr(q), B, Hq, ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), ctypes.byref(win.desc),
        _dptr(active), _dptr(acc), float(scale), _dptr(out), int(n_splits), _dptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))
    return out


def mustafar_window_step_grouped(win: DenseWindow, Kc: CompressedCache, Vc: CompressedCache,
                                 k_new, v_new, active=None, acc=None, stream=None) -> None:
    """One step of the grouped lifecycle: full windows first hand their oldest 32
    tokens to Kc (per token) and the per-channel cache Vc (one group, scored by acc
    [B][H][W] fp32, or by magnitude when acc is None)."""
    _check("mustafar_window_step_grouped", lib().mustafar_window_step_grouped(
        ctypes.byref(win.desc), ctypes.byref(Kc.desc), ctypes.byref(Vc.desc), _dptr(k_new),
        _dptr(v_new), _dptr(active), _dptr(acc), _stream(stream)))


# ---- the paged dense cache ----------------------------------------------------------------
class PagedCache:
    """Dense keys and values of B requests in pages of a shared pool, with the C descriptor.

    k, v [n_pages][H][page_tokens][d] (fp16 or bf16), table [B][max_pages], state [B + 2]
    (the requests' lengths, the free pages, a word of the library's) and free [n_pages] (the
    stack of free pages), int32. Tensors that are given are used as they are (k and v in any
    order of pages, heads and tokens whose channels are contiguous); the others are made, for an
    empty cache: a state that holds tokens comes with its table and its stack. max_pages: pages of the
    longest request (default: all). status [1] (int32): 0, or why the newest plan that was not
    given a status of its own was refused. A model has a cache a layer, each with k and v of its own and
    the first one's table, state and free, and a step one plan, taken on the first.
    """

    def __init__(self, B: int, H: int, d: int, n_pages: int, page_tokens: int = 64, max_pages: int | None = None,
                 dtype=None, device="cuda", k=None, v=None, table=None, state=None, free=None):
        import torch
        dtype = dtype or (k.dtype if k is not None else torch.float16)
        types = {torch.float16: FP16, torch.bfloat16: BF16}
        if dtype not in types:
            raise ValueError(f"pages hold float16 or bfloat16, not {dtype}")
        device = k.device if k is not None else device
        if max_pages is None:
            max_pages = table.shape[1] if table is not None else n_pages
        if k is None:
            k = torch.zeros((n_pages, H, page_tokens, d), dtype=dtype, device=device)
        if v is None:
            v = torch.zeros_like(k)
        table, state, free = _page_state(B, n_pages, max_pages, k.device, table, state, free)
        for name, x in (("k", k), ("v", v)):
            if tuple(x.shape) != (n_pages, H, page_tokens, d) or x.dtype != dtype or x.stride(3) != 1:
                raise ValueError(f"{name}: [{n_pages}][{H}][{page_tokens}][{d}] of {dtype} with contiguous channels expected")
        if k.stride() != v.stride():
            raise ValueError("k and v have the same strides")
        _want("v", v, tuple(k.shape), dtype, k.device, dense=False)
        self.k, self.v, self.table, self.state, self.free = k, v, table, state, free
        self.dtype, self.device = dtype, k.device
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.desc = pages_t()
        _check("mustafar_paged_init", lib().mustafar_paged_init(
            ctypes.byref(self.desc), _dptr(k), _dptr(v), _dptr(table), _dptr(state), _dptr(free), B, H, d,
            int(page_tokens), int(n_pages), int(max_pages), types[dtype], k.stride(0), k.stride(1), k.stride(2)))

    @property
    def B(self) -> int:
        return self.desc.B

    @property
    def page_tokens(self) -> int:
        return self.desc.page_tokens

    @property
    def lens(self):
        """The requests' lengths (a view of the state)."""
        return self.state[:self.desc.B]


def _want(name, x, shape, dtype, device, dense=True):
    """Raises unless x is a tensor of this shape, type and device, contiguous if `dense`."""
    if x.shape != shape or x.dtype != dtype or (dense and not x.is_contiguous()):
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} expected, "
                         f"not {x.dtype} {tuple(x.shape)}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, the cache on {device}")


def _page_state(B, n_pages, max_pages, device, table, state, free):
    """The tables, the state and the stack that are given, or those of an empty cache."""
    import torch
    if table is None:
        table = torch.zeros((B, max_pages), dtype=torch.int32, device=device)
    if state is None:
        state = torch.zeros(B + 2, dtype=torch.int32, device=device)
        state[B] = n_pages
    if free is None:
        free = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
    for name, x, shape in (("table", table, (B, max_pages)), ("state", state, (B + 2,)), ("free", free, (n_pages,))):
        _want(name, x, shape, torch.int32, device)
    return table, state, free


def _launch(owner, stream, what="the cache is") -> int | None:
    """Raw handle of `stream`, or of torch's current stream, for a call on tensors of the owner's device, which has to be the
    current one (one look-up of it for both)."""
    import torch
    index = torch.cuda.current_device()
    if owner.device.index != index:
        raise ValueError(f"{what} on {owner.device}, the current device is cuda:{index}")
    if stream is not None:
        if getattr(stream, "device_index", index) != index:
            raise ValueError(f"the stream is on cuda:{stream.device_index}, the current device is cuda:{index}")
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return _stream(None) if raw is None else raw(index)


def _rows(name, x, n, heads, cache):
    """Stride of the rows of x [n][heads][d] of the cache's type and device, whose rows are contiguous."""
    return _row_stride(name, x, n, heads, cache.desc.d, cache.dtype, cache.device)


def _row_stride(name, x, n, heads, d, dtype, device):
    if x.shape != (n, heads, d) or x.dtype != dtype:
        raise ValueError(f"{name}: [{n}][{heads}][{d}] of {dtype} expected, not {tuple(x.shape)} of {x.dtype}")
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, the cache on {device}")
    rows, head, channel = x.stride()
    if n and (channel != 1 or (heads > 1 and head != d)):
        raise ValueError(f"{name}: rows of {heads} x {d} contiguous elements expected")
    return rows if n > 1 else heads * d


def _int32(x) -> int:
    """A number of tokens as the C call takes it: behind 32 bits it would see another, and no cache holds more."""
    return max(-1, min(int(x), 0x7fffffff))


def _on_stream(stream):
    """Allocations of a call go to the stream that it works on."""
    import contextlib
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def mustafar_paged_plan(cache: PagedCache, new_len, n_slots: int, keep=None, state_out=None, cu=None, slots=None,
                        status=None, stream=None):
    """A step's pages, sequence starts and slots: new_len [B] (int32, device) new tokens behind the
    first keep [B] of every request (None: all it holds). Returns cu [B + 1] and slots [n_slots]. The
    cache's state advances in place, or is written to state_out [B + 2]. status [1] (None: cache.status) is
    0, or the PLAN_ bits of a step that was refused: it changed nothing, cu is 0 and slots are -1, so that the
    step's write and attention leave everything as it is. Too few free pages are such a step; look at the
    status before the results."""
    import torch
    B, i32 = cache.desc.B, torch.int32
    handle = _launch(cache, stream)
    with _on_stream(stream):
        cu = torch.empty(B + 1, dtype=i32, device=cache.device) if cu is None else cu
        slots = torch.empty(n_slots, dtype=i32, device=cache.device) if slots is None else slots
    status = cache.status if status is None else status
    state_out = cache.state if state_out is None else state_out
    for name, x, n in (("new_len", new_len, B), ("keep", keep, B), ("state_out", state_out, B + 2), ("cu", cu, B + 1),
                       ("slots", slots, n_slots), ("status", status, 1)):
        if x is not None:
            _want(name, x, (n,), i32, cache.device)
    _check("mustafar_paged_plan", lib().mustafar_paged_plan(
        ctypes.byref(cache.desc), _dptr(keep), _dptr(new_len), _dptr(state_out), _dptr(cu), _dptr(slots),
        int(n_slots), _dptr(status), handle))
    return cu, slots


def mustafar_paged_write(cache: PagedCache, k_new, v_new, slots, stream=None) -> None:
    """k_new, v_new [n][H][d] (the cache's type; rows of a packed projection too) into their slots
    [n] (int32; negative: left out)."""
    import torch
    n, H = k_new.shape[0], cache.desc.H
    handle = _launch(cache, stream)
    ks, vs = _rows("k_new", k_new, n, H, cache), _rows("v_new", v_new, n, H, cache)
    _want("slots", slots, (n,), torch.int32, cache.device)
    _check("mustafar_paged_write", lib().mustafar_paged_write(
        ctypes.byref(cache.desc), _dptr(k_new), ks, _dptr(v_new), vs, _dptr(slots), n, handle))


def mustafar_paged_gather(cache: PagedCache, n_max: int, first=None, x_k=None, x_v=None, stream=None):
    """The requests' tokens first[b] (int32 [B], None: 0) .. as dense fp16 x_k, x_v [B][H][n_max][d], the
    input of mustafar_window_prefill; rows behind a request's last are left as they were (0 in
    tensors that the call makes)."""
    return _gather("mustafar_paged_gather", cache, cache.desc, n_max, first, x_k, x_v, stream)


def _gather(fn, cache, desc, n_max, first, x_k, x_v, stream):
    import torch
    pages = cache.desc
    shape = (pages.B, pages.H, int(n_max), pages.d)
    handle = _launch(cache, stream)
    if x_k is None or x_v is None:
        with _on_stream(stream):
            x_k = torch.zeros(shape, dtype=torch.float16, device=cache.device) if x_k is None else x_k
            x_v = torch.zeros(shape, dtype=torch.float16, device=cache.device) if x_v is None else x_v
    _want("x_k", x_k, shape, torch.float16, cache.device)
    _want("x_v", x_v, shape, torch.float16, cache.device)
    if first is not None:
        _want("first", first, (shape[0],), torch.int32, cache.device)
    _check(fn, getattr(lib(), fn)(
        ctypes.byref(desc), None if first is None else first.data_ptr(), x_k.data_ptr(), x_v.data_ptr(), shape[2], handle))
    return x_k, x_v


def mustafar_paged_attn_workspace_bytes(cache: PagedCache, Hq: int, n_q: int, max_q: int, max_tokens: int,
                                        n_splits: int = 0) -> int:
    return lib().mustafar_paged_attn_workspace_bytes(ctypes.byref(cache.desc), int(Hq), int(n_q), _int32(max_q),
                                                     _int32(max_tokens), int(n_splits))


def mustafar_paged_attn(q, cache: PagedCache, cu, max_q: int | None = None, max_tokens: int | None = None,
                        window: int = 0, sinks: int = 0, scale: float = 0.0, out=None, n_splits: int = 0, ws=None,
                        stream=None):
    """Causal attention of q [n_q][Hq][d] (the cache's type; rows of a packed projection too), the last
    cu[b+1] - cu[b] tokens of every request b, over its pages; window > 0: the newest `window` tokens
    and the first `sinks`. max_q and max_tokens: bounds of a request's rows and length (default: one
    row each if n_q <= B, else n_q; all that a table can hold); with bounds near the truth calls are faster.
    Returns out [n_q][Hq][d]; rows from cu[B] on (all of a refused plan's) are left as they were, 0 in a tensor that
    the call makes."""
    return _paged_attn("mustafar_paged_attn", mustafar_paged_attn_workspace_bytes, q, cache, cache.desc, cu, max_q, max_tokens,
                       window, sinks, scale, out, n_splits, ws, stream)


def _paged_attn(fn, workspace_bytes, q, cache, desc, cu, max_q, max_tokens, window, sinks, scale, out, n_splits, ws, stream):
    import torch
    if q.dim() != 3:
        raise ValueError(f"q: [n_q][Hq][{cache.desc.d}] expected, not {tuple(q.shape)}")
    n_q, Hq, d = q.shape
    B = cache.desc.B
    max_q = (1 if n_q <= B else n_q) if max_q is None else max_q
    if max_tokens is None:
        max_tokens = min(cache.desc.max_pages, cache.desc.n_pages) * cache.desc.page_tokens
    max_q, max_tokens, window, sinks = _int32(max_q), _int32(max_tokens), _int32(window), _int32(sinks)
    handle = _launch(cache, stream)
    qs = _rows("q", q, n_q, Hq, cache)
    _want("cu", cu, (B + 1,), torch.int32, cache.device)
    if ws is None:
        need = workspace_bytes(cache, Hq, n_q, max_q, max_tokens, n_splits)
        if need > 0:
            with _on_stream(stream):
                ws = torch.empty(need, dtype=torch.uint8, device=cache.device)
    elif ws.device != cache.device or not ws.is_contiguous():
        raise ValueError(f"ws: contiguous memory on {cache.device} expected")
    if out is None:
        with _on_stream(stream):
            out = torch.zeros((n_q, Hq, d), dtype=cache.dtype, device=cache.device)
    os_ = _rows("out", out, n_q, Hq, cache)
    _check(fn, getattr(lib(), fn)(
        q.data_ptr(), qs, n_q, Hq, ctypes.byref(desc), cu.data_ptr(), window, sinks, float(scale), out.data_ptr(),
        os_, max_q, max_tokens, int(n_splits), None if ws is None else ws.data_ptr(), 0 if ws is None else ws.nbytes,
        handle))
    return out


class PagedCache8:
    """PagedCache in 8 bits: codes with a power of two for block_tokens tokens of a head.

    k, v [n_pages][H][page_tokens][d] are codes (`code`: torch.float8_e4m3fn or torch.int8), k_scale and v_scale
    [n_pages][H][page_tokens / block_tokens] (uint8) 127 + the exponents: a value is code * 2**(scale - 127), and
    one of `dtype` (float16 or bfloat16), the type of the tokens written, of queries and outputs. table, state, free
    and max_pages are PagedCache's, and mustafar_paged_plan and mustafar_rope take either.
    """

    def __init__(self, B: int, H: int, d: int, n_pages: int, page_tokens: int = 64, max_pages: int | None = None,
                 dtype=None, device="cuda", code=None, block_tokens: int = 16, k=None, v=None, k_scale=None, v_scale=None,
                 table=None, state=None, free=None):
        import torch
        dtype = dtype or torch.float16
        code = code or (k.dtype if k is not None else torch.float8_e4m3fn)
        types, codes = {torch.float16: FP16, torch.bfloat16: BF16}, {torch.float8_e4m3fn: E4M3, torch.int8: INT8}
        if dtype not in types:
            raise ValueError(f"tokens are float16 or bfloat16, not {dtype}")
        if code not in codes:
            raise ValueError(f"codes are float8_e4m3fn or int8, not {code}")
        if block_tokens not in (16, 32, 64) or block_tokens > page_tokens:
            raise ValueError(f"a block has 16, 32 or 64 tokens and no more than a page, not {block_tokens}")
        device = k.device if k is not None else device
        if max_pages is None:
            max_pages = table.shape[-1] if table is not None and table.dim() else n_pages
        shape, blocks = (n_pages, H, page_tokens, d), (n_pages, H, page_tokens // block_tokens)
        if k is None:
            k = torch.zeros(shape, dtype=torch.uint8, device=device).view(code)
        if v is None:
            v = torch.zeros_like(k.view(torch.uint8)).view(code)
        if k_scale is None:
            k_scale = torch.zeros(blocks, dtype=torch.uint8, device=device)
        if v_scale is None:
            v_scale = torch.zeros(blocks, dtype=torch.uint8, device=device)
        table, state, free = _page_state(B, n_pages, max_pages, k.device, table, state, free)
        for name, x in (("k", k), ("v", v)):
            if tuple(x.shape) != shape or x.dtype != code or x.stride(3) != 1:
                raise ValueError(f"{name}: [{n_pages}][{H}][{page_tokens}][{d}] of {code} with contiguous channels expected")
        if k.stride() != v.stride():
            raise ValueError("k and v have the same strides")
        _want("v", v, shape, code, k.device, dense=False)
        for name, x in (("k_scale", k_scale), ("v_scale", v_scale)):
            _want(name, x, blocks, torch.uint8, k.device)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.table, self.state, self.free = table, state, free
        self.dtype, self.device, self.code = dtype, k.device, code
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.desc8 = pages8_t()
        _check("mustafar_paged8_init", lib().mustafar_paged8_init(
            ctypes.byref(self.desc8), _dptr(k), _dptr(v), _dptr(k_scale), _dptr(v_scale), _dptr(table), _dptr(state),
            _dptr(free), B, H, d, int(page_tokens), int(n_pages), int(max_pages), types[dtype], codes[code],
            int(block_tokens), k.stride(0), k.stride(1), k.stride(2)))
        self.desc = self.desc8.pages    # (a view: what the plan takes)

    B, page_tokens, lens = PagedCache.B, PagedCache.page_tokens, PagedCache.lens

    @property
    def block_tokens(self) -> int:
        return self.desc8.block_tokens


def _codes(cache):
    if not isinstance(cache, PagedCache8):
        raise ValueError(f"a PagedCache8 expected, not {type(cache).__name__}")


def mustafar_paged8_write(cache: PagedCache8, k_new, v_new, cu, stream=None) -> None:
    """k_new, v_new [n][H][d] (the cache's dtype; rows of a packed projection too), the last cu[b+1] - cu[b] tokens of
    every request b of a planned step, quantised into its pages. A block that holds earlier tokens keeps its exponent, or
    gets the larger one that the new tokens need and its codes are rounded to it. Rows from cu[B] on are left out."""
    import torch
    _codes(cache)
    n, H = k_new.shape[0], cache.desc.H
    handle = _launch(cache, stream)
    ks, vs = _rows("k_new", k_new, n, H, cache), _rows("v_new", v_new, n, H, cache)
    _want("cu", cu, (cache.desc.B + 1,), torch.int32, cache.device)
    _check("mustafar_paged8_write", lib().mustafar_paged8_write(
        ctypes.byref(cache.desc8), k_new.data_ptr(), ks, v_new.data_ptr(), vs, cu.data_ptr(), n, handle))


def mustafar_paged8_gather(cache: PagedCache8, n_max: int, first=None, x_k=None, x_v=None, stream=None):
    """As mustafar_paged_gather: the values of the requests' tokens first[b] .. as dense fp16 [B][H][n_max][d]."""
    _codes(cache)
    return _gather("mustafar_paged8_gather", cache, cache.desc8, n_max, first, x_k, x_v, stream)


def mustafar_paged8_attn_workspace_bytes(cache: PagedCache8, Hq: int, n_q: int, max_q: int, max_tokens: int,
                                         n_splits: int = 0) -> int:
    return lib().mustafar_paged8_attn_workspace_bytes(ctypes.byref(cache.desc8), int(Hq), int(n_q), _int32(max_q),
                                                      _int32(max_tokens), int(n_splits))


def mustafar_paged8_attn(q, cache: PagedCache8, cu, max_q: int | None = None, max_tokens: int | None = None,
                         window: int = 0, sinks: int = 0, scale: float = 0.0, out=None, n_splits: int = 0, ws=None,
                         stream=None):
    """As mustafar_paged_attn, over the values that the codes stand for."""
    _codes(cache)
    return _paged_attn("mustafar_paged8_attn", mustafar_paged8_attn_workspace_bytes, q, cache, cache.desc8, cu, max_q, max_tokens,
                       window, sinks, scale, out, n_splits, ws, stream)


def mustafar_rope_rates(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                        original_len: float = 0.0, low_turns: float = 1.0, high_turns: float = 32.0) -> list:
    """Radians per position of the rot / 2 pairs. scaling: "plain" (base**(-2 i / rot)), "linear" (divided by factor),
    "base" (a larger base, so that the slowest is divided by factor) or "turns" (pairs of up to low_turns turns in original_len
    tokens are divided by factor, those of high_turns and more stay, the others lie between, linearly in their turns). A model
    whose rule is another, such as a ramp in the pair's index between two rounded bounds, passes its own rates to Rope."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling is one of {', '.join(ROPE_SCALINGS)}, not {scaling!r}")
    rates = (ctypes.c_double * max(1, int(rot) // 2))()
    _check("mustafar_rope_rates", lib().mustafar_rope_rates(rates, int(rot), float(base), ROPE_SCALINGS[scaling], float(factor),
                                                            float(original_len), float(low_turns), float(high_turns)))
    return list(rates)


class Rope:
    """Rotary positions of a model: the first rot channels of a head, in pairs `half` a rotation apart or `interleaved`,
    with the rates of mustafar_rope_rates (or `rates` [rot / 2], float64) and a magnitude that the rotated channels are
    multiplied by."""

    def __init__(self, rot: int, base: float = 10000.0, layout: str = "half", scaling: str = "plain", factor: float = 1.0,
                 original_len: float = 0.0, low_turns: float = 1.0, high_turns: float = 32.0, magnitude: float = 1.0,
                 rates=None, device="cuda"):
        import torch
        if layout not in ROPE_LAYOUTS:
            raise ValueError(f"layout is one of {', '.join(ROPE_LAYOUTS)}, not {layout!r}")
        if rates is None:
            rates = torch.tensor(mustafar_rope_rates(rot, base, scaling, factor, original_len, low_turns, high_turns),
                                 dtype=torch.float64, device=device)
        _want("rates", rates, (int(rot) // 2,), torch.float64, rates.device)
        self.rates, self.device = rates, rates.device
        self.desc = rotation_t(_dptr(rates), int(rot), ROPE_LAYOUTS[layout], float(magnitude))


def mustafar_rope(rope: Rope, q, k=None, positions=None, cache=None, cu=None, inverse: bool = False, out_q=None, out_k=None,
                  stream=None):
    """q [n][Hq][d] and k [n][H][d] (float16 or bfloat16; rows of a packed projection too; k may be None) turned by
    their positions [n] (int32), or by those of a planned step's new tokens: cache (a PagedCache or PagedCache8) and cu. Rows
    from cu[B] on are left as they were, 0 in tensors that the call makes. inverse: turned back, which is the gradient (autograd
    does not see the call: what it returns requires no gradient, so that training calls it in a torch.autograd.Function of its
    own, whose backward is the call with inverse=True).
    Returns (out_q, out_k), new tensors unless given; out_q=q, out_k=k turns in place."""
    import torch
    dtype, device = q.dtype, rope.device
    if q.dim() != 3 or (dtype is not torch.float16 and dtype is not torch.bfloat16):
        raise ValueError(f"q: [n][Hq][d] of float16 or bfloat16 expected, not {tuple(q.shape)} of {dtype}")
    n, Hq, d = q.shape
    handle = _launch(rope, stream, "rates are")
    if positions is not None:
        if cache is not None or cu is not None:
            raise ValueError("positions, or a cache and cu")
        _want("positions", positions, (n,), torch.int32, device)
        where = positions.data_ptr(), None, None
    else:
        if cache is None or cu is None:
            raise ValueError("positions, or a cache and cu")
        if cache.device != device:
            raise ValueError(f"rates are on {device}, the cache on {cache.device}")
        _want("cu", cu, (cache.desc.B + 1,), torch.int32, device)
        where = None, ctypes.byref(cache.desc), cu.data_ptr()
    qs = _row_stride("q", q, n, Hq, d, dtype, device)
    if out_q is None:
        out_q = _rope_out(q, cache, stream)
    oqs = _row_stride("out_q", out_q, n, Hq, d, dtype, device)
    if k is None:
        if out_k is not None:
            raise ValueError("out_k without k")
        keys = outs = None, 0
        H = 0
    else:
        if k.dim() != 3:
            raise ValueError(f"k: [{n}][H][{d}] expected, not {tuple(k.shape)}")
        H = k.shape[1]
        keys = k.data_ptr(), _row_stride("k", k, n, H, d, dtype, device)
        if out_k is None:
            out_k = _rope_out(k, cache, stream)
        outs = out_k.data_ptr(), _row_stride("out_k", out_k, n, H, d, dtype, device)
    _check("mustafar_rope", lib().mustafar_rope(
        ctypes.byref(rope.desc), q.data_ptr(), qs, Hq, *keys, H, d, n, FP16 if dtype is torch.float16 else BF16, *where,
        1 if inverse else 0, out_q.data_ptr(), oqs, *outs, handle))
    return out_q, out_k


def _rope_out(x, cache, stream):
    import torch
    with _on_stream(stream):
        return (torch.empty if cache is None else torch.zeros)(x.shape, dtype=x.dtype, device=x.device)


ROUTE_DEFAULT, ROUTE_WALKS, ROUTE_MATRIX_CORES = 0, 1, 2


def mustafar_attn_set_route(route: int) -> None:
    """Kernel route of the sparse calls (ROUTE_DEFAULT, ROUTE_WALKS, ROUTE_MATRIX_CORES)."""
    _check("mustafar_attn_set_route", lib().mustafar_attn_set_route(int(route)))


def mustafar_attn_route() -> int:
    return lib().mustafar_attn_route()


def mustafar_stream_mix(src, dst, write_16ths: int, sink=None, stream=None):
    """Measurement helper: stream device tensor `src`, write write_16ths/16 of it to `dst`."""
    import torch
    need = src.numel() * src.element_size() * write_16ths // 16
    if dst.numel() * dst.element_size() < need:
        raise ValueError(f"dst holds {dst.numel() * dst.element_size()} bytes, {need} needed")
    if sink is None:
        sink = torch.empty(lib().mustafar_stream_read_sink_bytes(), dtype=torch.uint8, device=src.device)
    _check("mustafar_stream_mix", lib().mustafar_stream_mix(
        _dptr(src), src.numel() * src.element_size(), _dptr(dst), int(write_16ths), _dptr(sink),
        _stream(stream)))
    return sink


STREAM_CHUNK_BYTES = 16384  # MUSTAFAR_STREAM_CHUNK_BYTES


def mustafar_stream_chunks(src, n_streams: int, dst, write_16ths: int, sink=None, stream=None):
    """Measurement helper: the bulk compression's access order over device tensor
    `src` (n_streams streams of 16 KiB chunks), write_16ths/16 of every chunk to `dst`;
    returns the per-chunk checksums (uint32 as int32, workgroup order)."""
    import torch
    nbytes = src.numel() * src.element_size()
    if n_streams < 1 or nbytes % (n_streams * STREAM_CHUNK_BYTES) != 0:
        raise ValueError(f"{nbytes} bytes are not {n_streams} streams of whole {STREAM_CHUNK_BYTES}-byte chunks")
    n_chunks = nbytes // (n_streams * STREAM_CHUNK_BYTES)
    need = nbytes * write_16ths // 16
    if dst.numel() * dst.element_size() < need:
        raise ValueError(f"dst holds {dst.numel() * dst.element_size()} bytes, {need} needed")
    if sink is None:
        sink = torch.empty(n_streams * n_chunks, dtype=torch.int32, device=src.device)
    _check("mustafar_stream_chunks", lib().mustafar_stream_chunks(
        _dptr(src), int(n_streams), int(n_chunks), _dptr(dst), int(write_16ths), _dptr(sink), _stream(stream)))
    return sink


def mustafar_stream_read(buf, sink=None, stream=None):
    """Measurement helper: stream the bytes of device tensor `buf` through 16-byte loads."""
    import torch
    if sink is None:
        sink = torch.empty(lib().mustafar_stream_read_sink_bytes(), dtype=torch.uint8,
                           device=buf.device)
    _check("mustafar_stream_read", lib().mustafar_stream_read(
        _dptr(buf), buf.numel() * buf.element_size(), _dptr(sink), _stream(stream)))
    return sink
