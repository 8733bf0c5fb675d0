"""ctypes marshalling for the C ABI declared in include/laser.h (same names, same arguments).

There is no fallback of any kind: if liblaser.so is missing or a call fails, LaserError is raised.
"""
from __future__ import annotations

import ctypes as C
from array import array
import sys
import os
import weakref

import numpy as np
import torch

MODE_RV, MODE_RV_OR_TOP1, MODE_TOPK_ONLY, MODE_TOPP_ONLY = 0, 1, 2, 3
MAX_NGRAM, MAX_DRAFT, MAX_TOPK, MAX_TREE, MAX_OWN_TEXT = 8, 63, 8, 32, 4096      # LASER_MAX_* of include/laser.h

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None


class LaserError(RuntimeError):
    pass


def lib_path() -> str:
    return os.path.join(_HERE, "liblaser.so")


class _ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "ffn", "vocab",
                                         "max_rows", "max_batch", "max_pos")] + \
               [("eps", C.c_float), ("rope_base", C.c_float)] + \
               [(n, C.c_void_p) for n in ("wqkv", "wo", "wgu", "wdown", "g1", "g2", "emb", "wlm", "gf")]


class _KVDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "n_heads", "head_dim", "page_size", "n_pages",
                                         "max_seqs", "max_pages_per_seq")]


class _Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("seq", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


F16, BF16, F32 = 0, 1, 2                                                         # LASER_F16 .. of include/laser.h
_DTYPES = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}


def lib():
    """Load liblaser.so once and declare the prototypes."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise LaserError(f"{path} is not built; run `python -m paper_2408_05676_amd.build` "
                         "(or __graft_entry__.build()) first. There is no fallback path.")
    L = C.CDLL(path)
    vp, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
    L.laser_last_error.restype = C.c_char_p
    L.laser_version.restype = C.c_char_p
    protos = {
        "laser_pool_build": [vp, vp, vp, i64, i32, vp, C.POINTER(vp)],
        "laser_pool_build_with": [vp, vp, vp, i64, i32, i32, i64, vp, C.POINTER(vp)],
        "laser_pool_destroy": [vp],
        "laser_pool_info": [vp, C.POINTER(i64), C.POINTER(i64), C.POINTER(i64), C.POINTER(i64)],
        "laser_pool_read_tokens": [vp, i64, i64, vp],
        "laser_retrieve_drafts": [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp],
        "laser_retrieve_drafts_temp": [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp],
        "laser_own_text_append": [vp, vp, i32, vp, vp, i32, i32, vp],
        "laser_model_create": [C.POINTER(_ModelDesc), vp, C.POINTER(vp)],
        "laser_model_destroy": [vp],
        "laser_kv_create": [C.POINTER(_KVDesc), vp, C.POINTER(vp)],
        "laser_kv_create_4bit": [C.POINTER(_KVDesc), vp, C.POINTER(vp)],
        "laser_rope_table": [vp, i32, i32, C.c_double, vp],
        "laser_kv_append": [vp, i32, vp, vp, vp, i32, i32, i32, C.POINTER(_Heads), C.POINTER(_Heads), C.POINTER(_Heads), C.POINTER(_Heads),
                            i32, vp, i32, i32, vp],
        "laser_kv_attend": [vp, i32, vp, vp, vp, i32, i32, i32, i32, C.POINTER(_Heads), f32, C.POINTER(_Heads), vp],
        "laser_kv_read": [vp, i32, vp, i32, i32, i32, i32, C.POINTER(_Heads), C.POINTER(_Heads), vp],
        "laser_w4_create": [vp, vp, vp, i32, i32, i32, vp, C.POINTER(vp)],
        "laser_w4_destroy": [vp],
        "laser_model_set_w4": [vp, i32, i32, vp],
        "laser_w4_quantize": [vp, i32, i32, i32, vp, vp, vp, vp],
        "laser_w4_matmul": [vp, vp, i64, i32, i32, vp, i64, vp],
        "laser_q8_rows": [vp, i64, i32, i32, i32, vp, i64, vp, vp],
        "laser_q8_norm": [vp, i64, i32, vp, i64, vp, i64, i32, vp, f32, i32, i32, vp, i64, vp, vp],
        "laser_q8_read": [vp, i64, vp, i32, i32, i32, vp, i64, vp],
        "laser_model_set_w8": [vp, i32, i32, vp],
        "laser_w8_create": [vp, vp, i32, i32, i32, vp, C.POINTER(vp)],
        "laser_w8_destroy": [vp],
        "laser_w8_quantize": [vp, i32, i32, vp, vp, vp],
        "laser_w8_matmul": [vp, vp, i64, vp, i32, i32, vp, i64, vp],
        "laser_kv_destroy": [vp],
        "laser_kv_seq_reserve": [vp, i32, i32, vp],
        "laser_kv_seq_release": [vp, i32, vp],
        "laser_kv_import": [vp, i32, i32, vp, vp, i32, vp],
        "laser_kv_seq_set_len": [vp, i32, i32, vp],
        "laser_kv_read_lens": [vp, vp, i32, vp, vp],
        "laser_verify_step": [vp, vp, vp, vp, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp],
        "laser_verify_head": [vp, vp, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp],
        "laser_verify_head_static": [vp, vp, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp],
        "laser_kv_commit": [vp, vp, vp, i32, vp],
        "laser_kv_commit_tree": [vp, vp, vp, vp, i32, i32, vp],
        "laser_generate": [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, C.POINTER(C.c_int), C.POINTER(C.c_float), vp],
        "laser_retrieve_tree": [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp],
        "laser_verify_tree": [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp],
        "laser_ctx_advance": [vp, vp, vp, vp, i32, i32, i32, vp],
        "laser_profile_begin": [vp, i32],
        "laser_model_set_option": [vp, C.c_char_p, i32],
        "laser_model_status": [vp, vp, C.POINTER(C.c_int)],
        "laser_model_read_trace": [vp, vp, vp, i32, C.POINTER(C.c_int), C.POINTER(C.c_int)],
        "laser_profile_end": [vp, vp, C.POINTER(C.c_float), C.POINTER(C.c_int)],
        "laser_probe_hbm": [vp, C.c_size_t, i32, vp, C.POINTER(C.c_float), C.POINTER(C.c_float)],
        "laser_probe_mfma_f16": [vp, i32, vp, C.POINTER(C.c_float)],
        "laser_probe_launch": [i32, i32, vp, C.POINTER(C.c_float)],
        "laser_probe_exchange": [vp, C.c_size_t, i32, vp, C.POINTER(C.c_float), C.POINTER(C.c_int)],
    }
    for name, args in protos.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = C.c_int
    _LIB = L
    return L


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise LaserError(f"{what} failed with code {rc}: {lib().laser_last_error().decode()}")


def _stream(stream=None) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise LaserError(f"{name} must be a contiguous CUDA tensor of {dtype}")
    return t.data_ptr()


def _host_i32(a, name: str) -> np.ndarray:
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.int32))
    if arr.ndim != 1:
        raise LaserError(f"{name} must be one-dimensional")
    return arr


class Pool:
    """laser_pool_build / laser_pool_destroy. builder ("auto", "host" or "device") and mem_limit are laser_pool_build_with's."""

    def __init__(self, tokens, seq_off, seq_key, n_max: int, stream=None, builder: str = "auto", mem_limit: int = -1):
        tokens = np.ascontiguousarray(tokens, dtype=np.int32)
        seq_off = np.ascontiguousarray(seq_off, dtype=np.int64)
        seq_key = np.ascontiguousarray(seq_key, dtype=np.int64)
        if seq_off.size != seq_key.size + 1:
            raise LaserError("seq_off must have n_seq + 1 entries")
        if seq_key.size and int(seq_off[-1]) != tokens.size:
            raise LaserError("seq_off[-1] must equal the number of tokens")
        self._h = C.c_void_p()
        self.n_max = n_max
        _check(lib().laser_pool_build_with(tokens.ctypes.data, seq_off.ctypes.data, seq_key.ctypes.data, seq_key.size, n_max,
                                           ("auto", "host", "device").index(builder), mem_limit, _stream(stream), C.byref(self._h)),
               "laser_pool_build")

    def info(self) -> dict:
        v = [C.c_int64() for _ in range(4)]
        _check(lib().laser_pool_info(self._h, *[C.byref(x) for x in v]), "laser_pool_info")
        return dict(zip(("n_tokens", "n_keys", "n_index_entries", "device_bytes"), (x.value for x in v)))

    def read_tokens(self, start: int, count: int) -> np.ndarray:
        out = np.empty(count, dtype=np.int32)
        _check(lib().laser_pool_read_tokens(self._h, start, count, out.ctypes.data), "laser_pool_read_tokens")
        return out

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().laser_pool_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone; the process frees everything
        if not sys.is_finalizing():
            self.close()


def retrieve_drafts(pool: Pool, keys: torch.Tensor, ctx_tail: torch.Tensor, n_min: int, n_max: int,
                    K: int, min_tokens: int = 1, out=None, stream=None):
    """laser_retrieve_drafts. Returns (drafts [B][K], draft_len [B], match_n [B], pool_index [B])."""
    B = keys.shape[0]
    if ctx_tail.shape != (B, n_max):
        raise LaserError("ctx_tail must be [B][n_max]")
    dev = keys.device
    if out is None:
        out = (torch.empty((B, K), dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int64, device=dev))
    drafts, dl, mn, pi = out
    _check(lib().laser_retrieve_drafts(pool._h, _dev(keys, torch.int64, "keys"), _dev(ctx_tail, torch.int32, "ctx_tail"),
                                       B, n_min, n_max, K, min_tokens,
                                       _dev(drafts, torch.int32, "drafts") if K > 0 else None,
                                       _dev(dl, torch.int32, "draft_len"), _dev(mn, torch.int32, "match_n"),
                                       _dev(pi, torch.int64, "pool_index"), _stream(stream)),
           "laser_retrieve_drafts")
    return drafts, dl, mn, pi


def retrieve_drafts_temp(pool: Pool, keys: torch.Tensor, ctx_tail: torch.Tensor, own_tokens: torch.Tensor,
                         own_len: torch.Tensor, n_min: int, n_max: int, K: int, min_tokens: int = 1, out=None, stream=None):
    """laser_retrieve_drafts_temp: the lookup with each sequence's own text [B][own_cap] as a temporary branch."""
    B = keys.shape[0]
    if ctx_tail.shape != (B, n_max):
        raise LaserError("ctx_tail must be [B][n_max]")
    if own_tokens.dim() != 2 or own_tokens.shape[0] != B or own_len.shape != (B,):
        raise LaserError("own_tokens must be [B][own_cap] and own_len [B]")
    dev = keys.device
    if out is None:
        out = (torch.empty((B, K), dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int64, device=dev))
    drafts, dl, mn, pi = out
    _check(lib().laser_retrieve_drafts_temp(pool._h, _dev(keys, torch.int64, "keys"), _dev(ctx_tail, torch.int32, "ctx_tail"),
                                            _dev(own_tokens, torch.int32, "own_tokens"), _dev(own_len, torch.int32, "own_len"),
                                            own_tokens.shape[1], B, n_min, n_max, K, min_tokens,
                                            _dev(drafts, torch.int32, "drafts") if K > 0 else None,
                                            _dev(dl, torch.int32, "draft_len"), _dev(mn, torch.int32, "match_n"),
                                            _dev(pi, torch.int64, "pool_index"), _stream(stream)),
           "laser_retrieve_drafts_temp")
    return drafts, dl, mn, pi


def own_text_append(own_tokens: torch.Tensor, own_len: torch.Tensor, out_tokens: torch.Tensor, accept_len: torch.Tensor,
                    stream=None):
    """laser_own_text_append."""
    B, cap = own_tokens.shape
    K = out_tokens.shape[1] - 1
    _check(lib().laser_own_text_append(_dev(own_tokens, torch.int32, "own_tokens"), _dev(own_len, torch.int32, "own_len"), cap,
                                       _dev(out_tokens, torch.int32, "out_tokens"), _dev(accept_len, torch.int32, "accept_len"),
                                       B, K, _stream(stream)), "laser_own_text_append")


class Model:
    """laser_model_create / laser_model_destroy. `weights` maps the names of laser_model_desc to
    CUDA tensors (bf16 matrices stacked over layers, float32 gains); they are borrowed, and kept
    alive by this object."""

    def __init__(self, n_layers, d_model, n_heads, ffn, vocab, weights: dict, max_rows: int, max_batch: int,
                 max_pos: int, eps: float = 1e-6, rope_base: float = 10000.0, stream=None):
        self.n_layers, self.d, self.n_heads, self.ffn, self.vocab = n_layers, d_model, n_heads, ffn, vocab
        self.max_rows, self.max_batch = max_rows, max_batch
        self._keep, self._w4 = dict(weights), set()
        d = _ModelDesc(n_layers, d_model, n_heads, ffn, vocab, max_rows, max_batch, max_pos, eps, rope_base)
        for name in ("wqkv", "wo", "wgu", "wdown", "emb", "wlm"):
            t = weights.get(name)
            if t is None:
                if n_layers == 0 and name != "wlm":
                    continue
                raise LaserError(f"missing weight {name}")
            setattr(d, name, _dev(t, torch.bfloat16, name))
        for name in ("g1", "g2", "gf"):
            t = weights.get(name)
            if t is None:
                if n_layers == 0:
                    continue
                raise LaserError(f"missing weight {name}")
            setattr(d, name, _dev(t, torch.float32, name))
        self.device = weights["wlm"].get_device()
        self._h = C.c_void_p()
        _check(lib().laser_model_create(C.byref(d), _stream(stream), C.byref(self._h)), "laser_model_create")

    def set_option(self, name: str, value: int):
        _check(lib().laser_model_set_option(self._h, name.encode(), value), "laser_model_set_option")

    def set_w4(self, layer: int, name: str, w4) -> None:
        """laser_model_set_w4: name is wqkv, wo, wgu or wdown, w4 a W4 or None. A W4 is kept alive until this object is closed, also after
        another has taken its place: a captured graph may still read it."""
        self._set(layer, name, w4, W4, lib().laser_model_set_w4)

    def set_w8(self, layer: int, name: str, w8) -> None:
        """laser_model_set_w8: the same with a W8 (wgu: a gated one)."""
        self._set(layer, name, w8, W8, lib().laser_model_set_w8)

    def _set(self, layer: int, name: str, w, kind, call) -> None:
        names = ("wqkv", "wo", "wgu", "wdown")
        if name not in names:
            raise LaserError(f"no matrix {name!r}: {', '.join(names)}")
        if w is not None:
            if not isinstance(w, kind) or not w._h:
                raise LaserError(f"the matrix must be a {kind.__name__} that has not been closed, or None")
            if w.device != self.device:
                raise LaserError(f"the matrix is on device {w.device}, the model on {self.device}")
        with torch.cuda.device(self.device):                                     # (the first W8 allocates)
            _check(call(self._h, layer, names.index(name), w._h if w is not None else None), call.__name__)
        if w is not None:
            self._w4.add(w)
            w._models.add(self)

    def aborted(self, stream=None) -> bool:
        v = C.c_int()
        _check(lib().laser_model_status(self._h, _stream(stream), C.byref(v)), "laser_model_status")
        return bool(v.value)

    def read_trace(self, stream=None) -> np.ndarray:
        """int64[nwg][cap] wall-clock stamps (100 MHz) of the last traced persistent-kernel launch."""
        buf = np.zeros(1 << 20, dtype=np.int64)
        nwg, cap = C.c_int(), C.c_int()
        _check(lib().laser_model_read_trace(self._h, _stream(stream), buf.ctypes.data, buf.size, C.byref(nwg), C.byref(cap)),
               "laser_model_read_trace")
        return buf[:nwg.value * cap.value].reshape(nwg.value, cap.value)

    def profile_begin(self, max_records: int):
        _check(lib().laser_profile_begin(self._h, max_records), "laser_profile_begin")

    def profile_end(self, stream=None):
        ms, n = C.c_float(), C.c_int()
        _check(lib().laser_profile_end(self._h, _stream(stream), C.byref(ms), C.byref(n)), "laser_profile_end")
        return ms.value, n.value

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().laser_model_destroy(self._h)
            self._h = C.c_void_p()
            self._w4.clear()

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone; the process frees everything
        if not sys.is_finalizing():
            self.close()


class KVCache:
    """laser_kv_create and the per-slot calls."""

    def __init__(self, n_layers, n_heads, head_dim, n_pages, max_seqs, max_pages_per_seq, page_size=16,
                 stream=None):
        self.page_size = page_size
        d = _KVDesc(n_layers, n_heads, head_dim, page_size, n_pages, max_seqs, max_pages_per_seq)
        self._h = C.c_void_p()
        _check(lib().laser_kv_create(C.byref(d), _stream(stream), C.byref(self._h)), "laser_kv_create")

    def reserve(self, seq: int, n_tokens: int, stream=None):
        _check(lib().laser_kv_seq_reserve(self._h, seq, n_tokens, _stream(stream)), "laser_kv_seq_reserve")

    def release(self, seq: int, stream=None):
        _check(lib().laser_kv_seq_release(self._h, seq, _stream(stream)), "laser_kv_seq_release")

    def import_layer(self, seq: int, layer: int, k: torch.Tensor, v: torch.Tensor, stream=None):
        n = k.shape[0]
        _check(lib().laser_kv_import(self._h, seq, layer, _dev(k, torch.float16, "k"), _dev(v, torch.float16, "v"),
                                     n, _stream(stream)), "laser_kv_import")

    def set_len(self, seq: int, n: int, stream=None):
        _check(lib().laser_kv_seq_set_len(self._h, seq, n, _stream(stream)), "laser_kv_seq_set_len")

    def read_lens(self, seq_ids, stream=None) -> np.ndarray:
        ids = _host_i32(seq_ids, "seq_ids")
        out = np.empty(ids.size, dtype=np.int32)
        _check(lib().laser_kv_read_lens(self._h, ids.ctypes.data, ids.size, out.ctypes.data, _stream(stream)),
               "laser_kv_read_lens")
        return out

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().laser_kv_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone; the process frees everything
        if not sys.is_finalizing():
            self.close()


class KVCache4(KVCache):
    """laser_kv_create_4bit: a KVCache whose keys and values are held in four bits. n_heads: its key/value heads."""

    def __init__(self, n_layers, n_heads, head_dim, n_pages, max_seqs, max_pages_per_seq, page_size=16, stream=None):
        self.page_size, self.n_heads, self.head_dim, self.device = page_size, n_heads, head_dim, torch.cuda.current_device()
        d = _KVDesc(n_layers, n_heads, head_dim, page_size, n_pages, max_seqs, max_pages_per_seq)
        self._h = C.c_void_p()
        _check(lib().laser_kv_create_4bit(C.byref(d), _stream(stream), C.byref(self._h)), "laser_kv_create_4bit")


def _heads(t: torch.Tensor, name: str, shape, dtype, dev: int) -> _Heads:
    """A [B][R][H][dh] tensor, in any order of its first three dimensions, as laser_heads."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != dtype or t.shape != shape:
        raise LaserError(f"{name} must be a CUDA tensor {list(shape)} of {dtype} with contiguous channels")
    s = t.stride()
    if s[3] != 1 and t.numel():
        raise LaserError(f"{name} must have contiguous channels")
    _here(t, name, dev)
    return _Heads(t.data_ptr(), s[0], s[1], s[2])


def _here(t: torch.Tensor, name: str, dev: int) -> None:
    if t.get_device() != dev:
        raise LaserError(f"{name} is on {t.device}, not on the current device")


def _device() -> int:
    return torch._C._cuda_getDevice()


def _on(stream, dev: int) -> int:
    """_stream() at a tenth of its host time where the current stream is meant (a small call takes less than that on the device)."""
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)


def _ids(seq_ids):
    """Sequence slots as a host int32 array."""
    return _host_i32(seq_ids, "seq_ids") if isinstance(seq_ids, (np.ndarray, torch.Tensor)) else array("i", seq_ids)


def _ids_ptr(ids) -> int:
    return ids.ctypes.data if isinstance(ids, np.ndarray) else ids.buffer_info()[0]


def _out(shape, dtype, device, stream) -> torch.Tensor:
    """A result's memory, allocated for the stream that writes it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(_stream(stream)))
    with torch.cuda.stream(s):
        return torch.empty(shape, dtype=dtype, device=device)


def _cache_device(kv) -> int:
    if not isinstance(kv, KVCache4):
        raise LaserError("kv must be a KVCache4")
    dev = _device()
    if kv.device != dev:
        raise LaserError(f"the cache is on device {kv.device}, not on the current one")
    return dev


def _step_args(n_ids, n_rows, tree_parent, B, R, dev):
    if n_ids != B:
        raise LaserError(f"seq_ids must name {B} sequences")
    if n_rows is not None:
        if n_rows.shape != (B,):
            raise LaserError("n_rows must be [B]")
        _here(n_rows, "n_rows", dev)
        n_rows = _dev(n_rows, torch.int32, "n_rows")
    if tree_parent is not None:
        if tree_parent.shape != (B, R - 1):
            raise LaserError("tree_parent must be [B][R - 1]")
        _here(tree_parent, "tree_parent", dev)
        tree_parent = _dev(tree_parent, torch.int32, "tree_parent")
    return n_rows, tree_parent


def rope_table(max_pos: int, dim: int, base: float = 10000.0, stream=None) -> torch.Tensor:
    """laser_rope_table: (cos, sin) float32 [max_pos][dim / 2][2]."""
    t = _out((max_pos, dim // 2, 2), torch.float32, "cuda", stream)
    _check(lib().laser_rope_table(t.data_ptr(), max_pos, dim, base, _stream(stream)), "laser_rope_table")
    return t


def kv_append(kv: KVCache4, layer: int, seq_ids, k: torch.Tensor, v: torch.Tensor, q=None, rope=None, tree_parent=None, n_rows=None,
              q_out=None, stream=None):
    """laser_kv_append: keys and values [B][R][heads][head_dim] of a step's rows into the cache, rotated by `rope`
    (rope_table; None: not rotated). Returns the rotated queries (q [B][R][query heads][head_dim], may be q_out itself) or None."""
    dev, ids = _cache_device(kv), _ids(seq_ids)
    if not isinstance(k, torch.Tensor) or k.dim() != 4:
        raise LaserError("k must be [B][R][heads][head_dim]")
    B, R = k.shape[:2]
    nr, tp = _step_args(len(ids), n_rows, tree_parent, B, R, dev)
    dt = k.dtype
    if dt not in _DTYPES:
        raise LaserError(f"k: {dt} is not float16, bfloat16 or float32")
    shape = (B, R, kv.n_heads, kv.head_dim)
    hk, hv = _heads(k, "k", shape, dt, dev), _heads(v, "v", shape, dt, dev)
    hq = ho = None
    n_heads = 0
    if q is not None:
        if not isinstance(q, torch.Tensor) or q.dim() != 4:
            raise LaserError("q must be [B][R][heads][head_dim]")
        n_heads = q.shape[2]
        if q_out is None:
            q_out = _out(q.shape, dt, q.device, stream)
        shape = (B, R, n_heads, kv.head_dim)
        hq, ho = _heads(q, "q", shape, dt, dev), _heads(q_out, "q_out", shape, dt, dev)
    rope_p, rope_dim, max_pos = None, 0, 0
    if rope is not None:
        if rope.dim() != 3 or rope.shape[2] != 2:
            raise LaserError("rope must be [max_pos][rope_dim / 2][2]")
        _here(rope, "rope", dev)
        rope_p, max_pos, rope_dim = _dev(rope, torch.float32, "rope"), rope.shape[0], 2 * rope.shape[1]
    _check(lib().laser_kv_append(kv._h, layer, _ids_ptr(ids), nr, tp, B, R, _DTYPES[dt], hk, hv, hq, ho, n_heads, rope_p, rope_dim, max_pos,
                                 _on(stream, dev)), "laser_kv_append")
    return q_out


def kv_attend(kv: KVCache4, layer: int, seq_ids, q: torch.Tensor, tree_parent=None, n_rows=None, scale=None, out=None, stream=None) -> torch.Tensor:
    """laser_kv_attend: q [B][R][query heads][head_dim] -> the same shape. scale: 1 / sqrt(head_dim) unless given."""
    dev, ids = _cache_device(kv), _ids(seq_ids)
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise LaserError("q must be [B][R][heads][head_dim]")
    B, R, H, dh = q.shape
    nr, tp = _step_args(len(ids), n_rows, tree_parent, B, R, dev)
    if q.dtype not in _DTYPES:
        raise LaserError(f"q: {q.dtype} is not float16, bfloat16 or float32")
    shape = (B, R, H, kv.head_dim)
    hq = _heads(q, "q", shape, q.dtype, dev)
    if out is None:
        out = _out(q.shape, q.dtype, q.device, stream)
    ho = _heads(out, "out", shape, q.dtype, dev)
    _check(lib().laser_kv_attend(kv._h, layer, _ids_ptr(ids), nr, tp, B, R, H, _DTYPES[q.dtype], hq, dh ** -0.5 if scale is None else scale, ho,
                                 _on(stream, dev)), "laser_kv_attend")
    return out


def kv_read(kv: KVCache4, layer: int, seq_ids, n: int, start: int = -1, dtype=torch.float16, out=None, stream=None):
    """laser_kv_read: the keys and values [B][n][heads][head_dim] that tokens start .. start + n - 1 (-1: those behind the committed
    length) stand for."""
    dev, ids = _cache_device(kv), _ids(seq_ids)
    B = len(ids)
    shape = (B, n, kv.n_heads, kv.head_dim)
    if out is None:
        out = _out(shape, dtype, "cuda", stream), _out(shape, dtype, "cuda", stream)
    k, v = out
    if k.dtype not in _DTYPES:
        raise LaserError(f"{k.dtype} is not float16, bfloat16 or float32")
    _check(lib().laser_kv_read(kv._h, layer, _ids_ptr(ids), B, start, n, _DTYPES[k.dtype], _heads(k, "k", shape, k.dtype, dev),
                               _heads(v, "v", shape, k.dtype, dev), _on(stream, dev)), "laser_kv_read")
    return k, v


def w4_quantize(w: torch.Tensor, group: int = 128, stream=None):
    """laser_w4_quantize: bf16 [N][Kd] -> (codes uint8 [N][Kd / 2], scales and offsets fp16 [N][Kd / group])."""
    p = _dev(w, torch.bfloat16, "w")
    if w.dim() != 2:
        raise LaserError("w must be [N][Kd]")
    _here(w, "w", _device())
    N, Kd = w.shape
    if group not in (32, 64, 128) or Kd % group:
        raise LaserError(f"group {group}: 32, 64 or 128, and Kd {Kd} a multiple of it")
    out = (_out((N, Kd // 2), torch.uint8, w.device, stream), *(_out((N, Kd // group), torch.float16, w.device, stream) for _ in range(2)))
    _check(lib().laser_w4_quantize(p, N, Kd, group, *(t.data_ptr() for t in out), _stream(stream)), "laser_w4_quantize")
    return out


class W4:
    """laser_w4_create / laser_w4_destroy: a matrix of 4-bit weights laid out for w4_matmul (see laser.h for the three arrays)."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, offsets: torch.Tensor, stream=None):
        self._h, self._models = C.c_void_p(), weakref.WeakSet()
        if codes.dim() != 2 or scales.dim() != 2 or scales.shape != offsets.shape or scales.shape[0] != codes.shape[0] or not scales.shape[1]:
            raise LaserError("codes must be [N][Kd / 2], scales and offsets [N][Kd / group]")
        for t, n in ((codes, "codes"), (scales, "scales"), (offsets, "offsets")):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                _here(t, n, _device())
        self.N, self.Kd = codes.shape[0], 2 * codes.shape[1]
        self.group = self.Kd // scales.shape[1]
        if self.group * scales.shape[1] != self.Kd:
            raise LaserError("Kd is not a multiple of the number of groups")
        self.device = codes.get_device()
        _check(lib().laser_w4_create(_dev(codes, torch.uint8, "codes"), _dev(scales, torch.float16, "scales"), _dev(offsets, torch.float16, "offsets"),
                                     self.N, self.Kd, self.group, _stream(stream), C.byref(self._h)), "laser_w4_create")

    def close(self):
        if any(m._h for m in getattr(self, "_models", ())):
            raise LaserError("the matrix is in use by a model: close that first")
        self._free()

    def _free(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().laser_w4_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone; the process frees everything
        if not sys.is_finalizing():
            self._free()


def w4_matmul(w: W4, x: torch.Tensor, out=None, stream=None) -> torch.Tensor:
    """laser_w4_matmul: x [M][Kd] (float16 or bfloat16, contiguous within a row) -> [M][N] of the same type."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in (torch.float16, torch.bfloat16) or x.dim() != 2 or x.shape[1] != w.Kd or x.stride(1) != 1:
        raise LaserError(f"x must be a CUDA tensor [M][{w.Kd}] of float16 or bfloat16 with contiguous rows")
    M, dev = x.shape[0], _device()
    if out is None:
        out = _out((M, w.N), x.dtype, x.device, stream)
    elif not isinstance(out, torch.Tensor) or not out.is_cuda or out.dtype != x.dtype or out.shape != (M, w.N) or (out.stride(1) != 1 and w.N > 1):
        raise LaserError(f"out must be a CUDA tensor [{M}][{w.N}] of {x.dtype} with contiguous rows")
    if x.get_device() != dev or out.get_device() != dev or w.device != dev:
        raise LaserError(f"x, out and the weights must be on the current device, not on {x.device}, {out.device} and {w.device}")
    _check(lib().laser_w4_matmul(w._h, x.data_ptr(), x.stride(0) if M > 1 else w.Kd, M, _DTYPES[x.dtype], out.data_ptr(),
                                 out.stride(0) if M > 1 else w.N, _on(stream, dev)), "laser_w4_matmul")
    return out


Q8_PAD = 128                                                                     # rows of codes lie multiples of this many bytes apart


# A small call takes less than the checks of its arguments would attribute by attribute: the helpers below read each of a tensor's once, and calls in between are left out.
_current, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _matrix(t, name: str, types):
    """(device, M, N, types[its dtype], row stride, address) of a [M][N] tensor with contiguous rows on the current device."""
    try:
        (M, N), (step, one), dt, dev = t.shape, t.stride(), types[t.dtype], t.get_device()
    except (AttributeError, ValueError, KeyError, TypeError):
        raise LaserError(f"{name} must be a CUDA tensor [M][N] of {', '.join(str(k)[6:] for k in types)}") from None
    if dev < 0 or dev != _current_device():
        raise LaserError(f"{name} is on {t.device}, not on the current device")
    if one != 1 and N > 1 and M:
        raise LaserError(f"{name} must have contiguous rows")
    return dev, M, N, dt, step if M > 1 else -(-N // Q8_PAD) * Q8_PAD, t.data_ptr()


def _like(t, name: str, M: int, N: int, types, dev: int):
    """(types[its dtype], row stride, address) of a [M][N] tensor with contiguous rows on device dev."""
    try:
        dt, shape, (step, one), on = types[t.dtype], t.shape, t.stride(), t.get_device()
    except (AttributeError, ValueError, KeyError, TypeError):
        shape = None
    if shape != (M, N) or on != dev:
        raise LaserError(f"{name} must be a tensor [{M}][{N}] of {', '.join(str(k)[6:] for k in types)} on the current device")
    if one != 1 and N > 1 and M:
        raise LaserError(f"{name} must have contiguous rows")
    return dt, step if M > 1 else -(-N // Q8_PAD) * Q8_PAD, t.data_ptr()


def _line(t, name: str, M: int, dev: int) -> int:
    """The address of a contiguous float32 [M] on device dev."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.shape != (M,) or t.get_device() != dev or not t.is_contiguous():
        raise LaserError(f"{name} must be a contiguous tensor [{M}] of float32 on the current device")
    return t.data_ptr()


_CODES = {torch.int8: 0}


def _q8_out(M: int, N: int, device, stream):
    """Memory for the codes and scales of M rows of N."""
    return _out((M, -(-N // Q8_PAD) * Q8_PAD), torch.int8, device, stream)[:, :N], _out((M,), torch.float32, device, stream)


def q8_rows(x: torch.Tensor, out=None, stream=None):
    """laser_q8_rows: x [M][N] -> (codes int8 [M][N], scales float32 [M]). The codes' rows are Q8_PAD bytes' multiples apart, as w8_matmul wants them;
    out: two such tensors to write to (codes of any row stride, if they are for q8_read only)."""
    dev, M, N, dt, step, xp = _matrix(x, "x", _DTYPES)
    codes, scales = _q8_out(M, N, x.device, stream) if out is None else out
    _, cs, cp = _like(codes, "codes", M, N, _CODES, dev)
    rc = lib().laser_q8_rows(xp, step, M, N, dt, cp, cs, _line(scales, "scales", M, dev), _current(dev) if stream is None else _stream(stream))
    if rc:
        _check(rc, "laser_q8_rows")
    return codes, scales


def q8_norm(x: torch.Tensor, gain: torch.Tensor, eps: float = 1e-6, residual=None, residual_out=None, out=None, stream=None):
    """laser_q8_norm: (codes, scales) of the root-mean-square norm of x + residual times gain (float32 [N]); the sum goes to residual_out (None: to
    residual itself). residual: float32 or x's type, or None."""
    dev, M, N, dt, step, xp = _matrix(x, "x", _DTYPES)
    rs, rp, os_, op, rdt = 0, None, 0, None, dt
    if residual is not None:
        rdt, rs, rp = _like(residual, "residual", M, N, _DTYPES, dev)
        odt, os_, op = (rdt, rs, rp) if residual_out is None else _like(residual_out, "residual_out", M, N, _DTYPES, dev)
        if odt != rdt:
            raise LaserError("residual_out is not of residual's type")
    elif residual_out is not None:
        raise LaserError("residual_out without a residual")
    codes, scales = _q8_out(M, N, x.device, stream) if out is None else out
    _, cs, cp = _like(codes, "codes", M, N, _CODES, dev)
    rc = lib().laser_q8_norm(xp, step, dt, rp, rs, op, os_, rdt, _line(gain, "gain", N, dev), eps, M, N, cp, cs, _line(scales, "scales", M, dev),
                             _current(dev) if stream is None else _stream(stream))
    if rc:
        _check(rc, "laser_q8_norm")
    return codes, scales


def q8_read(codes: torch.Tensor, scales: torch.Tensor, dtype=torch.float16, out=None, stream=None) -> torch.Tensor:
    """laser_q8_read: what rows of codes stand for, [M][N] of dtype (or of out's)."""
    dev, M, N, _, cs, cp = _matrix(codes, "codes", _CODES)
    if out is None:
        out = _out((M, N), dtype, codes.device, stream)
    dt, os_, op = _like(out, "out", M, N, _DTYPES, dev)
    rc = lib().laser_q8_read(cp, cs, _line(scales, "scales", M, dev), M, N, dt, op, os_, _current(dev) if stream is None else _stream(stream))
    if rc:
        _check(rc, "laser_q8_read")
    return out


def w8_quantize(w: torch.Tensor, stream=None):
    """laser_w8_quantize: bf16 [N][Kd] -> (codes int8 [N][Kd], scales float32 [N])."""
    p = _dev(w, torch.bfloat16, "w")
    if w.dim() != 2:
        raise LaserError("w must be [N][Kd]")
    _here(w, "w", _device())
    N, Kd = w.shape
    out = _out((N, Kd), torch.int8, w.device, stream), _out((N,), torch.float32, w.device, stream)
    _check(lib().laser_w8_quantize(p, N, Kd, *(t.data_ptr() for t in out), _stream(stream)), "laser_w8_quantize")
    return out


class W8:
    """laser_w8_create / laser_w8_destroy: a matrix of 8-bit weights laid out for w8_matmul, codes int8 [N][Kd] and scales float32 [N] (w8_quantize).
    gated: rows 0 .. N / 2 - 1 are gates, the others the up projection; a product then has N / 2 columns, silu(gate) * up."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, gated: bool = False, stream=None):
        self._h, self._models = C.c_void_p(), weakref.WeakSet()
        if codes.dim() != 2 or scales.shape != codes.shape[:1]:
            raise LaserError("codes must be [N][Kd] and scales [N]")
        for t, n in ((codes, "codes"), (scales, "scales")):
            if t.is_cuda:
                _here(t, n, _device())
        self.N, self.Kd = codes.shape
        self.gated, self.outs, self.device = bool(gated), self.N // 2 if gated else self.N, codes.get_device()
        _check(lib().laser_w8_create(_dev(codes, torch.int8, "codes"), _dev(scales, torch.float32, "scales"), self.N, self.Kd, int(self.gated),
                                     _stream(stream), C.byref(self._h)), "laser_w8_create")

    def close(self):
        if any(m._h for m in getattr(self, "_models", ())):
            raise LaserError("the matrix is in use by a model: close that first")
        self._free()

    def _free(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().laser_w8_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        # at interpreter shutdown the HIP runtime may already be gone; the process frees everything
        if sys is not None and not sys.is_finalizing():
            self._free()


def w8_matmul(w: W8, x: torch.Tensor, scales: torch.Tensor, dtype=torch.float16, out=None, stream=None) -> torch.Tensor:
    """laser_w8_matmul: rows of codes x int8 [M][Kd] with their scales (q8_rows, q8_norm) -> [M][w.outs] of dtype (or of out's)."""
    if not isinstance(w, W8) or not w._h:
        raise LaserError("w must be a W8 that has not been closed")
    dev, M, Kd, _, step, xp = _matrix(x, "x", _CODES)
    if w.device != dev or w.Kd != Kd:
        raise LaserError(f"the weights are [{w.N}][{w.Kd}] on device {w.device}, the rows [{M}][{Kd}] on {dev}")
    # a row's bytes up to the next multiple of Q8_PAD are read
    if Kd % Q8_PAD and M and x.storage_offset() + (M - 1) * step + -(-Kd // Q8_PAD) * Q8_PAD > x.untyped_storage().nbytes():
        raise LaserError(f"rows of x must lie multiples of {Q8_PAD} bytes apart, and the memory of the last one reach as far")
    if out is None:
        out = _out((M, w.outs), dtype, x.device, stream)
    dt, os_, op = _like(out, "out", M, w.outs, _DTYPES, dev)
    rc = lib().laser_w8_matmul(w._h, xp, step, _line(scales, "scales", M, dev), M, dt, op, os_, _current(dev) if stream is None else _stream(stream))
    if rc:
        _check(rc, "laser_w8_matmul")
    return out


def verify_step(model: Model, kv: KVCache, seq_ids, pending: torch.Tensor, drafts: torch.Tensor,
                draft_len: torch.Tensor, topk: int, p: float, mode: int = MODE_RV, want_logits: bool = False,
                out=None, stream=None):
    """laser_verify_step. Returns (accept_len [B], out_tokens [B][K+1], logits [B][K+1][V] or None)."""
    ids = _host_i32(seq_ids, "seq_ids")
    B, K = drafts.shape
    dev = pending.device
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty((B, K + 1), dtype=torch.int32, device=dev))
    acc, toks = out
    logits = torch.empty((B, K + 1, model.vocab), dtype=torch.float32, device=dev) if want_logits else None
    _check(lib().laser_verify_step(model._h, kv._h, ids.ctypes.data, _dev(pending, torch.int32, "pending"),
                                   _dev(drafts, torch.int32, "drafts") if K > 0 else None,
                                   _dev(draft_len, torch.int32, "draft_len"), B, K, topk, p, mode,
                                   _dev(acc, torch.int32, "accept_len"), _dev(toks, torch.int32, "out_tokens"),
                                   logits.data_ptr() if want_logits else None, _stream(stream)),
           "laser_verify_step")
    return acc, toks, logits


def verify_head(model: Model, h: torch.Tensor, drafts: torch.Tensor, draft_len: torch.Tensor, topk: int,
                p: float, mode: int = MODE_RV, want_logits: bool = False, out=None, stream=None):
    """laser_verify_head on final-normed hidden states h fp16 [B][K+1][d]."""
    B, K = drafts.shape
    if h.shape != (B, K + 1, model.d):
        raise LaserError("h must be [B][K+1][d]")
    dev = h.device
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty((B, K + 1), dtype=torch.int32, device=dev))
    acc, toks = out
    logits = torch.empty((B, K + 1, model.vocab), dtype=torch.float32, device=dev) if want_logits else None
    _check(lib().laser_verify_head(model._h, _dev(h, torch.float16, "h"),
                                   _dev(drafts, torch.int32, "drafts") if K > 0 else None,
                                   _dev(draft_len, torch.int32, "draft_len"), B, K, topk, p, mode,
                                   _dev(acc, torch.int32, "accept_len"), _dev(toks, torch.int32, "out_tokens"),
                                   logits.data_ptr() if want_logits else None, _stream(stream)),
           "laser_verify_head")
    return acc, toks, logits


def retrieve_tree(pool: "Pool", keys: torch.Tensor, ctx_tail: torch.Tensor, n_min: int, n_max: int, K: int,
                  min_tokens: int = 1, out=None, stream=None):
    """laser_retrieve_tree. Returns (tree_tokens [B][K], tree_parent [B][K], tree_freq [B][K], tree_len [B], match_n [B])."""
    B = keys.shape[0]
    dev = keys.device
    if out is None:
        out = (torch.empty((B, K), dtype=torch.int32, device=dev), torch.empty((B, K), dtype=torch.int32, device=dev),
               torch.empty((B, K), dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev),
               torch.empty(B, dtype=torch.int32, device=dev))
    tok, par, freq, tl, mn = out
    _check(lib().laser_retrieve_tree(pool._h, _dev(keys, torch.int64, "keys"), _dev(ctx_tail, torch.int32, "ctx_tail"),
                                     B, n_min, n_max, K, min_tokens,
                                     _dev(tok, torch.int32, "tree_tokens") if K > 0 else None,
                                     _dev(par, torch.int32, "tree_parent") if K > 0 else None,
                                     (_dev(freq, torch.int32, "tree_freq") if K > 0 else None) if freq is not None else None,
                                     _dev(tl, torch.int32, "tree_len"), _dev(mn, torch.int32, "match_n"), _stream(stream)),
           "laser_retrieve_tree")
    return tok, par, freq, tl, mn


def verify_tree(model: "Model", kv: "KVCache", seq_ids, pending: torch.Tensor, tree_tokens: torch.Tensor,
                tree_parent: torch.Tensor, tree_len: torch.Tensor, topk: int, p: float, mode: int = MODE_RV,
                want_logits: bool = False, out=None, stream=None):
    """laser_verify_tree. Returns (accept_len [B], out_tokens [B][K+1], accept_path [B][K], logits or None)."""
    ids = _host_i32(seq_ids, "seq_ids")
    B, K = tree_tokens.shape
    dev = pending.device
    if out is None:
        out = (torch.empty(B, dtype=torch.int32, device=dev), torch.empty((B, K + 1), dtype=torch.int32, device=dev),
               torch.empty((B, K), dtype=torch.int32, device=dev))
    acc, toks, path = out
    logits = torch.empty((B, K + 1, model.vocab), dtype=torch.float32, device=dev) if want_logits else None
    _check(lib().laser_verify_tree(model._h, kv._h, ids.ctypes.data, _dev(pending, torch.int32, "pending"),
                                   _dev(tree_tokens, torch.int32, "tree_tokens") if K > 0 else None,
                                   _dev(tree_parent, torch.int32, "tree_parent") if K > 0 else None,
                                   _dev(tree_len, torch.int32, "tree_len"), B, K, topk, p, mode,
                                   _dev(acc, torch.int32, "accept_len"), _dev(toks, torch.int32, "out_tokens"),
                                   _dev(path, torch.int32, "accept_path") if K > 0 else None,
                                   logits.data_ptr() if want_logits else None, _stream(stream)), "laser_verify_tree")
    return acc, toks, path, logits


def kv_commit_tree(kv: "KVCache", seq_ids, accept_len: torch.Tensor, accept_path: torch.Tensor, stream=None):
    """laser_kv_commit_tree."""
    ids = _host_i32(seq_ids, "seq_ids")
    K = accept_path.shape[1]
    _check(lib().laser_kv_commit_tree(kv._h, ids.ctypes.data, _dev(accept_len, torch.int32, "accept_len"),
                                      _dev(accept_path, torch.int32, "accept_path") if K > 0 else None, ids.size, K,
                                      _stream(stream)), "laser_kv_commit_tree")


class GenerateOpts(C.Structure):
    _fields_ = [("K", C.c_int32), ("n_min", C.c_int32), ("n_max", C.c_int32), ("min_tokens", C.c_int32), ("tree", C.c_int32),
                ("topk", C.c_int32), ("p", C.c_float), ("mode", C.c_int32), ("max_new_tokens", C.c_int32), ("eos_token", C.c_int32),
                ("check_every", C.c_int32), ("own_cap", C.c_int32)]


def generate(model: "Model", kv: "KVCache", pool, seq_ids, keys, ctx_tail: torch.Tensor, pending: torch.Tensor, K: int, n_min: int,
             topk: int, p: float, mode: int = MODE_RV, max_new_tokens: int = 64, eos_token: int = -1, tree: bool = False,
             min_tokens: int = 1, check_every: int = 8, own_tokens=None, own_len=None, time_retrieval: bool = False, stream=None):
    """laser_generate. Returns (gen_tokens int32 [B][max_new_tokens] (-1 padded), gen_len int32 [B], counters int32 [B][4],
    steps run, summed retrieval-kernel milliseconds or None)."""
    ids = _host_i32(seq_ids, "seq_ids")
    B, n_max = ctx_tail.shape
    dev = pending.device
    gen = torch.empty((B, max_new_tokens), dtype=torch.int32, device=dev)
    glen = torch.empty(B, dtype=torch.int32, device=dev)
    cnt = torch.empty((B, 4), dtype=torch.int32, device=dev)
    own_cap = own_tokens.shape[1] if own_tokens is not None else 0
    o = GenerateOpts(K, n_min, n_max, min_tokens, int(tree), topk, p, mode, max_new_tokens, eos_token, check_every, own_cap)
    steps, ms = C.c_int(0), C.c_float(0.0)
    _check(lib().laser_generate(model._h, kv._h, pool._h if pool is not None else None, ids.ctypes.data,
                                _dev(keys, torch.int64, "keys") if keys is not None else None,
                                _dev(ctx_tail, torch.int32, "ctx_tail"), _dev(pending, torch.int32, "pending"),
                                _dev(own_tokens, torch.int32, "own_tokens") if own_tokens is not None else None,
                                _dev(own_len, torch.int32, "own_len") if own_len is not None else None,
                                ids.size, C.byref(o), gen.data_ptr(), glen.data_ptr(), cnt.data_ptr(), C.byref(steps),
                                C.byref(ms) if time_retrieval else None, _stream(stream)), "laser_generate")
    return gen, glen, cnt, steps.value, (ms.value if time_retrieval else None)


def verify_head_static(model: Model, h: torch.Tensor, drafts: torch.Tensor, draft_len: torch.Tensor, topk: int,
                       p: float, mode: int, out, stream=None):
    """laser_verify_head_static: laser_verify_head without any allocation (at most 16 rows); out = (accept_len
    int32 [B], out_tokens int32 [B][K+1]) must be given."""
    B, K = drafts.shape
    if h.shape != (B, K + 1, model.d):
        raise LaserError("h must be [B][K+1][d]")
    acc, toks = out
    _check(lib().laser_verify_head_static(model._h, _dev(h, torch.float16, "h"),
                                          _dev(drafts, torch.int32, "drafts") if K > 0 else None,
                                          _dev(draft_len, torch.int32, "draft_len"), B, K, topk, p, mode,
                                          _dev(acc, torch.int32, "accept_len"), _dev(toks, torch.int32, "out_tokens"),
                                          _stream(stream)), "laser_verify_head_static")
    return acc, toks


def kv_commit(kv: KVCache, seq_ids, accept_len: torch.Tensor, stream=None):
    """laser_kv_commit."""
    ids = _host_i32(seq_ids, "seq_ids")
    _check(lib().laser_kv_commit(kv._h, ids.ctypes.data, _dev(accept_len, torch.int32, "accept_len"), ids.size,
                                 _stream(stream)), "laser_kv_commit")


def ctx_advance(ctx_tail: torch.Tensor, pending: torch.Tensor, out_tokens: torch.Tensor, accept_len: torch.Tensor,
                stream=None):
    """laser_ctx_advance."""
    B, n_max = ctx_tail.shape
    K = out_tokens.shape[1] - 1
    _check(lib().laser_ctx_advance(_dev(ctx_tail, torch.int32, "ctx_tail"), _dev(pending, torch.int32, "pending"),
                                   _dev(out_tokens, torch.int32, "out_tokens"), _dev(accept_len, torch.int32, "accept_len"),
                                   B, K, n_max, _stream(stream)), "laser_ctx_advance")


def probe_hbm(buf: torch.Tensor, reps: int = 10, stream=None):
    """laser_probe_hbm on a caller-owned CUDA scratch tensor: (read GB/s, copy GB/s)."""
    if not (isinstance(buf, torch.Tensor) and buf.is_cuda and buf.is_contiguous()):
        raise LaserError("buf must be a contiguous CUDA tensor")
    nbytes = buf.numel() * buf.element_size()
    r, c = C.c_float(), C.c_float()
    _check(lib().laser_probe_hbm(buf.data_ptr(), nbytes - nbytes % 32, reps, _stream(stream), C.byref(r), C.byref(c)),
           "laser_probe_hbm")
    return r.value, c.value


def probe_mfma_f16(scratch: torch.Tensor, reps: int = 10, stream=None) -> float:
    """laser_probe_mfma_f16: executed TFLOP/s of a register-resident fp16 matrix-instruction loop."""
    if not (isinstance(scratch, torch.Tensor) and scratch.is_cuda and scratch.numel() * scratch.element_size() >= 4):
        raise LaserError("scratch must be a CUDA tensor of at least 4 bytes")
    t = C.c_float()
    _check(lib().laser_probe_mfma_f16(scratch.data_ptr(), reps, _stream(stream), C.byref(t)), "laser_probe_mfma_f16")
    return t.value


def probe_launch(blocks: int, reps: int = 200, stream=None) -> float:
    """laser_probe_launch: microseconds per launch of an empty kernel of `blocks` wavefronts."""
    t = C.c_float()
    _check(lib().laser_probe_launch(blocks, reps, _stream(stream), C.byref(t)), "laser_probe_launch")
    return t.value


def probe_exchange(scratch: torch.Tensor, iters: int = 200, stream=None):
    """laser_probe_exchange: (microseconds per all-to-all exchange of a cooperative launch, error count)."""
    if not (isinstance(scratch, torch.Tensor) and scratch.is_cuda and scratch.is_contiguous()):
        raise LaserError("scratch must be a contiguous CUDA tensor")
    t, e = C.c_float(), C.c_int()
    _check(lib().laser_probe_exchange(scratch.data_ptr(), scratch.numel() * scratch.element_size(), iters, _stream(stream),
                                      C.byref(t), C.byref(e)), "laser_probe_exchange")
    return t.value, e.value
