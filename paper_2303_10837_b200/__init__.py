"""Python binding of ``libfedhe.so``: the sm_100a CUDA library for the hot path of
FedML-HE secure aggregation (mask selection, CKKS encode + encrypt, weighted
ciphertext aggregation with rescale, decrypt + decode, pack/unpack).

The functions have the names of the C entry points in ``include/fedhe.h`` and do
argument marshalling only: torch owns device memory and streams, every step of
the path runs in the library's kernels.  There is no CPU fallback: importing
this package without the built library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfedhe.so")

HE_MAX_LIMBS = 16
HE_MAX_CLIENTS = 256
HE_OK = 0
HE_ERR_INVALID_ARG, HE_ERR_PARAMS, HE_ERR_ALLOC, HE_ERR_CUDA = -1, -2, -3, -4
HE_ERR_OVERFLOW, HE_ERR_LEVEL, HE_ERR_SIZE = -5, -6, -7


class HeError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (where, he_strerror(code), code))


class he_params(C.Structure):
    _fields_ = [("N", C.c_uint32), ("L", C.c_uint32), ("q", C.c_uint64 * HE_MAX_LIMBS),
                ("log2_delta", C.c_int32)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libfedhe.so is missing: build it with `python paper_2303_10837_b200/build.py` "
            "(there is no fallback path)")
    return C.CDLL(LIB_PATH)


_lib = _load()
_vp, _sz, _u64, _u32 = C.c_void_p, C.c_size_t, C.c_uint64, C.c_uint32

_SIGS = {
    "he_strerror": (C.c_char_p, [C.c_int]),
    "he_launch_count": (_u64, []),
    "he_ctx_create": (C.c_int, [C.POINTER(he_params), C.POINTER(_vp)]),
    "he_ctx_destroy": (C.c_int, [_vp]),
    "he_ctx_status": (C.c_int, [_vp, C.POINTER(C.c_int)]),
    "he_ctx_reserve": (C.c_int, [_vp, _sz]),
    "he_slots": (_sz, [_vp]),
    "he_num_ct": (_sz, [_vp, _sz]),
    "he_ct_words": (_sz, [_vp, _u32]),
    "he_keygen": (C.c_int, [_vp, _u64, C.POINTER(_vp), _vp]),
    "he_keys_destroy": (C.c_int, [_vp]),
    "he_keys_export": (C.c_int, [_vp, _vp, _vp, _vp, _vp]),
    "he_select_mask": (C.c_int, [_vp, _vp, _sz, _sz, C.POINTER(_vp), _vp]),
    "he_select_mask_ranges": (C.c_int, [_vp, _vp, _sz, _sz, _vp, _sz, C.POINTER(_vp), _vp]),
    "he_mask_indices": (C.c_int, [_vp, C.POINTER(_vp), C.POINTER(_sz)]),
    "he_mask_copy_indices": (C.c_int, [_vp, _vp, _vp]),
    "he_mask_destroy": (C.c_int, [_vp]),
    "he_pack": (C.c_int, [_vp, _vp, _vp, _sz, _vp, _vp, _vp]),
    "he_encode": (C.c_int, [_vp, _vp, _sz, _vp, _vp]),
    "he_encrypt": (C.c_int, [_vp, _vp, _vp, _sz, _u64, _u32, _vp, _vp]),
    "he_encrypt_range": (C.c_int, [_vp, _vp, _vp, _sz, _sz, _u64, _u32, _vp, _vp]),
    "he_weighted_aggregate": (C.c_int, [_vp, _vp, _vp, C.c_int, _sz, _vp, _vp]),
    "he_weighted_partial": (C.c_int, [_vp, _vp, _vp, C.c_int, _sz, _vp, _vp]),
    "he_rescale_partial_sum": (C.c_int, [_vp, _vp, _u32, _sz, _vp, _vp]),
    "he_rescale_partial_parts": (C.c_int, [_vp, _vp, C.c_int, _sz, _vp, _vp]),
    "he_encrypt_ntt": (C.c_int, [_vp, _vp, _vp, _sz, _u64, _u32, _vp, _vp]),
    "he_weighted_aggregate_ntt": (C.c_int, [_vp, _vp, _vp, C.c_int, _sz, _vp, _vp]),
    "he_decrypt_level_ntt": (C.c_int, [_vp, _vp, _vp, _u32, _sz, _vp, _vp]),
    "he_plain_aggregate": (C.c_int, [_vp, _vp, _vp, C.c_int, _sz, _vp, _vp]),
    "he_decrypt": (C.c_int, [_vp, _vp, _vp, _sz, _vp, _vp]),
    "he_decrypt_level": (C.c_int, [_vp, _vp, _vp, _u32, _sz, _vp, _vp]),
    "he_decrypt_noalloc": (C.c_int, [_vp, _vp, _vp, _sz, _vp, _vp]),
    "he_threshold_split": (C.c_int, [_vp, _vp, _u64, C.POINTER(_vp), C.POINTER(_vp), _vp]),
    "he_partial_decrypt": (C.c_int, [_vp, _vp, _u32, _vp, _u32, _sz, _u64, _u32, _vp, _vp]),
    "he_threshold_combine": (C.c_int, [_vp, _vp, _u32, _vp, C.c_int, _sz, _vp, _vp]),
    "he_unpack": (C.c_int, [_vp, _vp, _vp, _vp, _sz, _vp, _vp]),
    "he_ntt_forward": (C.c_int, [_vp, _vp, _sz, _vp]),
    "he_ntt_inverse": (C.c_int, [_vp, _vp, _sz, _vp]),
    "he_round_host": (C.c_int, [_vp, _vp, _vp, _vp, _vp, C.c_int, _sz, _u64, _vp, _vp]),
    "he_token_log_probs": (C.c_int, [_vp, _vp, C.c_int, _sz, _sz, _sz, _vp, _u32, _vp, _vp, _vp, _vp, _vp, _vp]),
    "he_token_log_probs_backward": (C.c_int, [_vp, _vp, C.c_int, _sz, _sz, _sz, _vp, _vp, _vp, _vp, _vp, _u32, _vp, _vp, _vp, _sz, _vp]),
    "he_layer_norm": (C.c_int, [_vp, _vp, C.c_int, _sz, _sz, _sz, _vp, _vp, C.c_int, C.c_float, _vp, _sz, _vp, _vp, _vp]),
    "he_layer_norm_backward_work_bytes": (_sz, [_vp, _sz, _sz]),
    "he_layer_norm_backward": (C.c_int, [_vp, _vp, _sz, _vp, _sz, C.c_int, _sz, _sz, _vp, _vp, _vp, C.c_int, _vp, _sz, _vp, _sz, _vp, _vp,
                                         _vp, _sz, _vp]),
    "he_linear_sensitivity_work_bytes": (_sz, [_vp, C.c_int, _sz, _sz, _sz, C.c_int, C.c_int]),
    "he_linear_sensitivity": (C.c_int, [_vp, _vp, _sz, _vp, _sz, C.c_int, _sz, _sz, _sz, _vp, _sz, C.c_int, _vp, _vp, _vp, _sz, _vp]),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTS = tuple(_SIGS)


def he_strerror(code: int) -> str:
    return _lib.he_strerror(code).decode()


def he_launch_count() -> int:
    return int(_lib.he_launch_count())


def _check(code: int, where: str) -> None:
    if code != HE_OK:
        raise HeError(code, where)


# The current stream's handle without making a stream object: 0.2 us instead of 3.2, of 14 us that a short call (packing or encrypting
# a ciphertext) takes the host.  Private names of torch, so the public call stands in where one of them is absent.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> int:
    """The current stream's handle."""
    if _raw_stream and _raw_device and torch.cuda.is_initialized():
        return _raw_stream(_raw_device())
    return torch.cuda.current_stream().cuda_stream


def _dev(t: torch.Tensor, dtype: torch.dtype) -> int:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError("expected a contiguous CUDA tensor of dtype %s" % dtype)
    return t.data_ptr()


# The C ABI takes plain pointers and cannot know how large a buffer is, so this
# layer is where a short buffer is caught: before the call, on the host, as an
# error instead of an out-of-bounds access on the device.
def _sized(t: torch.Tensor, count: int, what: str, exact: bool = False) -> None:
    have = t.numel()
    if have != count if exact else have < count:
        raise HeError(HE_ERR_INVALID_ARG, "%s: %d entries, %s%d needed" % (what, have, "" if exact else "at least ", count))


def _same_len(a, b, what: str) -> None:
    if len(a) != len(b) or len(a) < 1:
        raise HeError(HE_ERR_INVALID_ARG, "%s: %d and %d entries" % (what, len(a), len(b)))


def _whole_cts(ctx: "Ctx", sel: torch.Tensor, what: str) -> int:
    """Number of ciphertexts of a slot buffer, which must hold whole ciphertexts."""
    if sel.numel() % ctx.n:
        raise HeError(HE_ERR_INVALID_ARG, "%s: %d slots is not a multiple of n = %d" % (what, sel.numel(), ctx.n))
    return sel.numel() // ctx.n


def _ct_count(ctx: "Ctx", ct: torch.Tensor, level: int, what: str) -> int:
    """T of a ciphertext tensor [T][2][level][N] (taken from its first extent, checked against its size)."""
    if not 1 <= level <= ctx.L:
        raise HeError(HE_ERR_LEVEL, what)
    T = ct.shape[0] if ct.dim() else 0
    _sized(ct, T * 2 * level * ctx.N, what, exact=True)
    return T


class Ctx:
    """Owner of a ``he_ctx*``."""

    def __init__(self, handle: int, N: int, L: int, log2_delta: int):
        self.handle, self.N, self.L, self.log2_delta = handle, N, L, log2_delta
        self.n = N // 2

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:     # _lib is gone at interpreter exit
            _lib.he_ctx_destroy(self.handle)
            self.handle = None


class Keys:
    def __init__(self, handle: int, ctx: Ctx):
        self.handle, self.ctx = handle, ctx

    def __del__(self):
        if getattr(self, "handle", None) and getattr(self.ctx, "handle", None) and _lib is not None:
            _lib.he_keys_destroy(self.handle)
            self.handle = None


class Mask:
    def __init__(self, handle: int, P: int, k: int, idx_ptr: int):
        self.handle, self.P, self.k, self.idx_ptr = handle, P, k, idx_ptr

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.he_mask_destroy(self.handle)
            self.handle = None


def he_ctx_create(N: int, primes: Sequence[int], log2_delta: int) -> Ctx:
    p = he_params()
    p.N, p.L, p.log2_delta = N, len(primes), log2_delta
    if len(primes) > HE_MAX_LIMBS:
        raise HeError(HE_ERR_PARAMS, "he_ctx_create")
    for j, q in enumerate(primes):
        p.q[j] = q
    h = _vp()
    _check(_lib.he_ctx_create(C.byref(p), C.byref(h)), "he_ctx_create")
    return Ctx(h.value, N, len(primes), log2_delta)


def he_ctx_status(ctx: Ctx) -> int:
    st = C.c_int(0)
    _check(_lib.he_ctx_status(ctx.handle, C.byref(st)), "he_ctx_status")
    return st.value


def he_ctx_reserve(ctx: Ctx, max_k: int) -> None:
    _check(_lib.he_ctx_reserve(ctx.handle, max_k), "he_ctx_reserve")


def he_slots(ctx: Ctx) -> int:
    return int(_lib.he_slots(ctx.handle))


def he_num_ct(ctx: Ctx, k: int) -> int:
    return int(_lib.he_num_ct(ctx.handle, k))


def he_ct_words(ctx: Ctx, level: int) -> int:
    return int(_lib.he_ct_words(ctx.handle, level))


def he_keygen(ctx: Ctx, seed: int) -> Keys:
    h = _vp()
    _check(_lib.he_keygen(ctx.handle, seed, C.byref(h), _stream()), "he_keygen")
    return Keys(h.value, ctx)


def he_keys_export(ctx: Ctx, keys: Keys):
    """(pk uint64-as-int64 [2][L][N], s int8 [N]) on the device."""
    pk = torch.empty((2, ctx.L, ctx.N), dtype=torch.int64, device="cuda")
    s = torch.empty(ctx.N, dtype=torch.int8, device="cuda")
    _check(_lib.he_keys_export(ctx.handle, keys.handle, pk.data_ptr(), s.data_ptr(), _stream()),
           "he_keys_export")
    return pk, s


def _finish_mask(h: _vp, P: int) -> Mask:
    ip, k = _vp(), _sz()
    _check(_lib.he_mask_indices(h.value, C.byref(ip), C.byref(k)), "he_mask_indices")
    return Mask(h.value, P, int(k.value), ip.value or 0)


def he_select_mask(ctx: Ctx, score: torch.Tensor, k: int) -> Mask:
    h = _vp()
    _check(_lib.he_select_mask(ctx.handle, _dev(score, torch.float32), score.numel(), k, C.byref(h),
                               _stream()), "he_select_mask")
    return _finish_mask(h, score.numel())


def he_select_mask_ranges(ctx: Ctx, score: torch.Tensor, k: int, ranges: Sequence[Sequence[int]]) -> Mask:
    flat = (C.c_uint64 * (2 * len(ranges)))(*[int(v) for r in ranges for v in r])
    h = _vp()
    _check(_lib.he_select_mask_ranges(ctx.handle, _dev(score, torch.float32), score.numel(), k,
                                      C.cast(flat, _vp), len(ranges), C.byref(h), _stream()),
           "he_select_mask_ranges")
    return _finish_mask(h, score.numel())


def he_mask_indices(mask: Mask) -> torch.Tensor:
    """Copy of the ascending index list (int32 view of the uint32 values)."""
    out = torch.empty(mask.k, dtype=torch.int32, device="cuda")
    _check(_lib.he_mask_copy_indices(mask.handle, out.data_ptr() if mask.k else None, _stream()),
           "he_mask_copy_indices")
    return out


def he_pack(ctx: Ctx, mask: Optional[Mask], x: torch.Tensor):
    """(sel float32 [T*n], rest float32 [P-k] or None)."""
    P = x.numel()
    if mask is not None and mask.P != P:
        raise HeError(HE_ERR_INVALID_ARG, "he_pack: the mask was built for %d parameters, x has %d" % (mask.P, P))
    k = mask.k if mask is not None else P
    sel = torch.empty(he_num_ct(ctx, k) * ctx.n, dtype=torch.float32, device="cuda")
    rest = torch.empty(P - k, dtype=torch.float32, device="cuda") if mask is not None else None
    _check(_lib.he_pack(ctx.handle, mask.handle if mask else None, _dev(x, torch.float32), P,
                        sel.data_ptr(), rest.data_ptr() if rest is not None else None, _stream()),
           "he_pack")
    return sel, rest


def he_encode(ctx: Ctx, sel: torch.Tensor) -> torch.Tensor:
    T = _whole_cts(ctx, sel, "he_encode sel")
    m = torch.empty((T, ctx.N), dtype=torch.int64, device="cuda")
    _check(_lib.he_encode(ctx.handle, _dev(sel, torch.float32), sel.numel(), m.data_ptr(), _stream()),
           "he_encode")
    return m


def he_encrypt(ctx: Ctx, keys: Keys, sel: torch.Tensor, seed: int, client_id: int,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Fresh ciphertexts uint64-as-int64 [T][2][L][N]."""
    T = _whole_cts(ctx, sel, "he_encrypt sel")
    if out is None:
        out = torch.empty((T, 2, ctx.L, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * ctx.L * ctx.N, "he_encrypt out")
    _check(_lib.he_encrypt(ctx.handle, keys.handle, _dev(sel, torch.float32), sel.numel(), seed, client_id,
                           _dev(out, torch.int64), _stream()), "he_encrypt")
    return out


def he_encrypt_ntt(ctx: Ctx, keys: Keys, sel: torch.Tensor, seed: int, client_id: int,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The same ciphertexts in the transform-domain wire format."""
    T = _whole_cts(ctx, sel, "he_encrypt_ntt sel")
    if out is None:
        out = torch.empty((T, 2, ctx.L, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * ctx.L * ctx.N, "he_encrypt_ntt out")
    _check(_lib.he_encrypt_ntt(ctx.handle, keys.handle, _dev(sel, torch.float32), sel.numel(), seed, client_id,
                               _dev(out, torch.int64), _stream()), "he_encrypt_ntt")
    return out


def he_encrypt_range(ctx: Ctx, keys: Keys, sel: torch.Tensor, t_begin: int, t_count: int, seed: int,
                     client_id: int, out: torch.Tensor) -> torch.Tensor:
    """`sel` holds the slots of ciphertexts t_begin .. t_begin+t_count-1."""
    _sized(sel, t_count * ctx.n, "he_encrypt_range sel")
    _sized(out, t_count * 2 * ctx.L * ctx.N, "he_encrypt_range out")
    _check(_lib.he_encrypt_range(ctx.handle, keys.handle, _dev(sel, torch.float32), t_begin, t_count, seed,
                                 client_id, _dev(out, torch.int64), _stream()), "he_encrypt_range")
    return out


def he_weighted_aggregate(ctx: Ctx, cts: List[torch.Tensor], alpha: Sequence[float],
                          out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _same_len(cts, alpha, "he_weighted_aggregate cts and alpha")
    Cn = len(cts)
    T = _ct_count(ctx, cts[0], ctx.L, "he_weighted_aggregate cts[0]")
    for i, c in enumerate(cts):
        _sized(c, T * 2 * ctx.L * ctx.N, "he_weighted_aggregate cts[%d]" % i, exact=True)
    if out is None:
        out = torch.empty((T, 2, ctx.L - 1, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * (ctx.L - 1) * ctx.N, "he_weighted_aggregate out")
    ptrs = (_vp * Cn)(*[_dev(c, torch.int64) for c in cts])
    al = (C.c_double * Cn)(*[float(a) for a in alpha])
    _check(_lib.he_weighted_aggregate(ctx.handle, C.cast(ptrs, _vp), C.cast(al, _vp), Cn, T,
                                      _dev(out, torch.int64), _stream()), "he_weighted_aggregate")
    return out


def he_weighted_partial(ctx: Ctx, cts: List[torch.Tensor], alpha: Sequence[float],
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Weighted sum of a subset of the clients on all L limbs, no rescale: int64 [T][2][L][N]."""
    _same_len(cts, alpha, "he_weighted_partial cts and alpha")
    Cn = len(cts)
    T = _ct_count(ctx, cts[0], ctx.L, "he_weighted_partial cts[0]")
    for i, c in enumerate(cts):
        _sized(c, T * 2 * ctx.L * ctx.N, "he_weighted_partial cts[%d]" % i, exact=True)
    if out is None:
        out = torch.empty((T, 2, ctx.L, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * ctx.L * ctx.N, "he_weighted_partial out")
    ptrs = (_vp * Cn)(*[_dev(c, torch.int64) for c in cts])
    al = (C.c_double * Cn)(*[float(a) for a in alpha])
    _check(_lib.he_weighted_partial(ctx.handle, C.cast(ptrs, _vp), C.cast(al, _vp), Cn, T,
                                    _dev(out, torch.int64), _stream()), "he_weighted_partial")
    return out


def he_rescale_partial_sum(ctx: Ctx, summed: torch.Tensor, parts: int,
                           out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rescale of the word-by-word sum of `parts` results of he_weighted_partial."""
    T = _ct_count(ctx, summed, ctx.L, "he_rescale_partial_sum summed")
    if out is None:
        out = torch.empty((T, 2, ctx.L - 1, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * (ctx.L - 1) * ctx.N, "he_rescale_partial_sum out")
    _check(_lib.he_rescale_partial_sum(ctx.handle, _dev(summed, torch.int64), int(parts), T,
                                       _dev(out, torch.int64), _stream()), "he_rescale_partial_sum")
    return out


def he_rescale_partial_parts(ctx: Ctx, parts: List[torch.Tensor], out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rescale of the sum of several results of he_weighted_partial, added by the kernel itself."""
    if len(parts) < 1:
        raise HeError(HE_ERR_INVALID_ARG, "he_rescale_partial_parts: no parts")
    T = _ct_count(ctx, parts[0], ctx.L, "he_rescale_partial_parts parts[0]")
    for i, p in enumerate(parts):
        _sized(p, T * 2 * ctx.L * ctx.N, "he_rescale_partial_parts parts[%d]" % i, exact=True)
    if out is None:
        out = torch.empty((T, 2, ctx.L - 1, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * (ctx.L - 1) * ctx.N, "he_rescale_partial_parts out")
    ptrs = (_vp * len(parts))(*[_dev(p, torch.int64) for p in parts])
    _check(_lib.he_rescale_partial_parts(ctx.handle, C.cast(ptrs, _vp), len(parts), T,
                                         _dev(out, torch.int64), _stream()), "he_rescale_partial_parts")
    return out


def he_weighted_aggregate_ntt(ctx: Ctx, cts: List[torch.Tensor], alpha: Sequence[float],
                              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _same_len(cts, alpha, "he_weighted_aggregate_ntt cts and alpha")
    Cn = len(cts)
    T = _ct_count(ctx, cts[0], ctx.L, "he_weighted_aggregate_ntt cts[0]")
    for i, c in enumerate(cts):
        _sized(c, T * 2 * ctx.L * ctx.N, "he_weighted_aggregate_ntt cts[%d]" % i, exact=True)
    if out is None:
        out = torch.empty((T, 2, ctx.L - 1, ctx.N), dtype=torch.int64, device="cuda")
    _sized(out, T * 2 * (ctx.L - 1) * ctx.N, "he_weighted_aggregate_ntt out")
    ptrs = (_vp * Cn)(*[_dev(c, torch.int64) for c in cts])
    al = (C.c_double * Cn)(*[float(a) for a in alpha])
    _check(_lib.he_weighted_aggregate_ntt(ctx.handle, C.cast(ptrs, _vp), C.cast(al, _vp), Cn, T,
                                          _dev(out, torch.int64), _stream()), "he_weighted_aggregate_ntt")
    return out


def he_plain_aggregate(ctx: Ctx, rests: List[torch.Tensor], alpha: Sequence[float]) -> torch.Tensor:
    _same_len(rests, alpha, "he_plain_aggregate rests and alpha")
    Cn = len(rests)
    n = rests[0].numel()
    for i, r in enumerate(rests):
        _sized(r, n, "he_plain_aggregate rests[%d]" % i, exact=True)
    ptrs = (_vp * Cn)(*[_dev(r, torch.float32) if n else 1 for r in rests])
    al = (C.c_double * Cn)(*[float(a) for a in alpha])
    out = torch.empty(n, dtype=torch.float64, device="cuda")
    _check(_lib.he_plain_aggregate(ctx.handle, C.cast(ptrs, _vp), C.cast(al, _vp), Cn, n, out.data_ptr(),
                                   _stream()), "he_plain_aggregate")
    return out


def he_decrypt(ctx: Ctx, keys: Keys, agg: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    T = _ct_count(ctx, agg, ctx.L - 1, "he_decrypt agg")
    if out is None:
        out = torch.empty(T * ctx.n, dtype=torch.float64, device="cuda")
    _sized(out, T * ctx.n, "he_decrypt out")
    _check(_lib.he_decrypt(ctx.handle, keys.handle, _dev(agg, torch.int64), T, _dev(out, torch.float64),
                           _stream()), "he_decrypt")
    return out


def he_decrypt_level(ctx: Ctx, keys: Keys, ct: torch.Tensor, level: int) -> torch.Tensor:
    T = _ct_count(ctx, ct, level, "he_decrypt_level ct")
    z = torch.empty(T * ctx.n, dtype=torch.float64, device="cuda")
    _check(_lib.he_decrypt_level(ctx.handle, keys.handle, _dev(ct, torch.int64), level, T, z.data_ptr(),
                                 _stream()), "he_decrypt_level")
    return z


def he_decrypt_level_ntt(ctx: Ctx, keys: Keys, ct: torch.Tensor, level: int,
                         out: Optional[torch.Tensor] = None) -> torch.Tensor:
    T = _ct_count(ctx, ct, level, "he_decrypt_level_ntt ct")
    if out is None:
        out = torch.empty(T * ctx.n, dtype=torch.float64, device="cuda")
    _sized(out, T * ctx.n, "he_decrypt_level_ntt out")
    _check(_lib.he_decrypt_level_ntt(ctx.handle, keys.handle, _dev(ct, torch.int64), level, T,
                                     _dev(out, torch.float64), _stream()), "he_decrypt_level_ntt")
    return out


def he_threshold_split(ctx: Ctx, keys: Keys, seed: int):
    """Two additive shares of the secret key (handles accepted by he_partial_decrypt only)."""
    a, b = _vp(), _vp()
    _check(_lib.he_threshold_split(ctx.handle, keys.handle, seed, C.byref(a), C.byref(b), _stream()),
           "he_threshold_split")
    return Keys(a.value, ctx), Keys(b.value, ctx)


def he_partial_decrypt(ctx: Ctx, share: Keys, party: int, ct: torch.Tensor, level: int, seed: int,
                       smudge_bits: int) -> torch.Tensor:
    """Residues mod q_0, uint64-as-int64 [T][N]."""
    T = _ct_count(ctx, ct, level, "he_partial_decrypt ct")
    part = torch.empty((T, ctx.N), dtype=torch.int64, device="cuda")
    _check(_lib.he_partial_decrypt(ctx.handle, share.handle, party, _dev(ct, torch.int64) or None, level, T,
                                   seed, smudge_bits, part.data_ptr() or None, _stream()), "he_partial_decrypt")
    return part


def he_threshold_combine(ctx: Ctx, ct: torch.Tensor, level: int, parts: List[torch.Tensor]) -> torch.Tensor:
    T = _ct_count(ctx, ct, level, "he_threshold_combine ct")
    for i, p in enumerate(parts):
        _sized(p, T * ctx.N, "he_threshold_combine parts[%d]" % i, exact=True)
    ptrs = (_vp * len(parts))(*[_dev(p, torch.int64) for p in parts])
    z = torch.empty(T * ctx.n, dtype=torch.float64, device="cuda")
    _check(_lib.he_threshold_combine(ctx.handle, _dev(ct, torch.int64) or None, level, C.cast(ptrs, _vp),
                                     len(parts), T, z.data_ptr() or None, _stream()), "he_threshold_combine")
    return z


HE_NOALLOC_MAX_WORDS = 1 << 21


def he_decrypt_noalloc(ctx: Ctx, keys: Keys, agg: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """he_decrypt without any allocation inside the library: the work buffer is a fixed array
    in the library image, so T * N must not exceed HE_NOALLOC_MAX_WORDS and N must be <= 16384.
    `out` (float64 [T*n]) is supplied by the caller for the same reason."""
    T = _ct_count(ctx, agg, ctx.L - 1, "he_decrypt_noalloc agg")
    _sized(out, T * ctx.n, "he_decrypt_noalloc out")
    _check(_lib.he_decrypt_noalloc(ctx.handle, keys.handle, _dev(agg, torch.int64) or None, T,
                                   _dev(out, torch.float64) or None, _stream()), "he_decrypt_noalloc")
    return out


def he_unpack(ctx: Ctx, mask: Optional[Mask], z: torch.Tensor, rest_avg: Optional[torch.Tensor], P: int,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    k = P
    if mask is not None:
        if mask.P != P:
            raise HeError(HE_ERR_INVALID_ARG, "he_unpack: the mask was built for %d parameters, P is %d" % (mask.P, P))
        k = mask.k
        if k < P:
            if rest_avg is None:
                raise HeError(HE_ERR_INVALID_ARG, "he_unpack: rest_avg is missing")
            _sized(rest_avg, P - k, "he_unpack rest_avg")
    _sized(z, k, "he_unpack z")
    if out is None:
        out = torch.empty(P, dtype=torch.float64, device="cuda")
    _sized(out, P, "he_unpack out")
    _check(_lib.he_unpack(ctx.handle, mask.handle if mask else None, _dev(z, torch.float64) or None,
                          _dev(rest_avg, torch.float64) if (rest_avg is not None and rest_avg.numel()) else None,
                          P, _dev(out, torch.float64), _stream()), "he_unpack")
    return out


def he_ntt_forward(ctx: Ctx, polys: torch.Tensor) -> torch.Tensor:
    """In place on uint64-as-int64 [B][L][N]."""
    _sized(polys, (polys.shape[0] if polys.dim() else 0) * ctx.L * ctx.N, "he_ntt_forward polys", exact=True)
    _check(_lib.he_ntt_forward(ctx.handle, _dev(polys, torch.int64), polys.shape[0], _stream()),
           "he_ntt_forward")
    return polys


def he_ntt_inverse(ctx: Ctx, polys: torch.Tensor) -> torch.Tensor:
    _sized(polys, (polys.shape[0] if polys.dim() else 0) * ctx.L * ctx.N, "he_ntt_inverse polys", exact=True)
    _check(_lib.he_ntt_inverse(ctx.handle, _dev(polys, torch.int64), polys.shape[0], _stream()),
           "he_ntt_inverse")
    return polys


def he_round_host(ctx: Ctx, keys: Keys, mask: Optional[Mask], xs: List[torch.Tensor],
                  alpha: Sequence[float], enc_seed: int, out: torch.Tensor) -> torch.Tensor:
    """Whole round with HOST tensors in (float32 [P] each, ideally pinned) and out (float64 [P])."""
    _same_len(xs, alpha, "he_round_host xs and alpha")
    Cn = len(xs)
    P = xs[0].numel()
    if mask is not None and mask.P != P:
        raise HeError(HE_ERR_INVALID_ARG, "he_round_host: the mask was built for %d parameters, xs have %d" % (mask.P, P))
    for x in xs:
        if x.is_cuda or x.dtype != torch.float32 or not x.is_contiguous() or x.numel() != P:
            raise TypeError("xs must be contiguous host float32 tensors of one size")
    if out.is_cuda or out.dtype != torch.float64 or out.numel() != P:
        raise TypeError("out must be a host float64 tensor of P entries")
    ptrs = (_vp * Cn)(*[x.data_ptr() for x in xs])
    al = (C.c_double * Cn)(*[float(a) for a in alpha])
    _check(_lib.he_round_host(ctx.handle, keys.handle, mask.handle if mask else None, C.cast(ptrs, _vp),
                              C.cast(al, _vp), Cn, P, enc_seed, out.data_ptr(), _stream()), "he_round_host")
    return out


# ---------------------------------------------------------------------------
# the sensitivity map's operators (Step 1 of Selective Parameter Encryption)
# ---------------------------------------------------------------------------

HE_F32, HE_BF16, HE_F16 = 0, 1, 2
HE_MAX_TOP = 64
_DTYPES = {torch.float32: HE_F32, torch.bfloat16: HE_BF16, torch.float16: HE_F16}


def _dtype(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise HeError(HE_ERR_INVALID_ARG, "%s: %s, not float32, bfloat16 or float16" % (what, t.dtype))
    return code


def _matrix(t: torch.Tensor, rows: Optional[int], cols: Optional[int], dtype: Optional[torch.dtype], what: str, out: bool = False) -> int:
    """Row stride of a matrix whose rows are contiguous; its sizes and type are checked (None: any)."""
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        raise HeError(HE_ERR_INVALID_ARG, "%s: shape %s, [%s][%s] needed" % (what, tuple(shape), "rows" if rows is None else rows,
                                                                             "columns" if cols is None else cols))
    if dtype is not None and t.dtype != dtype:
        raise HeError(HE_ERR_INVALID_ARG, "%s: %s, %s needed" % (what, t.dtype, dtype))
    stride, step = t.stride()
    if step != 1 and shape[1] > 1:
        raise HeError(HE_ERR_INVALID_ARG, "%s: the elements of a row do not lie together" % what)
    if shape[0] < 2:
        stride = shape[1]
    if out and stride < shape[1]:
        raise HeError(HE_ERR_INVALID_ARG, "%s: rows overlap" % what)
    return stride


def _vector(t: torch.Tensor, count: int, dtype: torch.dtype, what: str, dtype2: Optional[torch.dtype] = None) -> None:
    if len(t.shape) != 1 or t.shape[0] != count or (t.dtype != dtype and t.dtype != dtype2) or (count > 1 and t.stride(0) != 1):
        raise HeError(HE_ERR_INVALID_ARG, "%s: %s %s, a contiguous vector of %d needed" % (what, t.dtype, tuple(t.shape), count))


def _on_gpu(*tensors: Optional[torch.Tensor]) -> int:
    """All tensors lie on the current device (None: absent)."""
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise TypeError("expected CUDA tensors")
    device = _raw_device() if _raw_device else torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise HeError(HE_ERR_INVALID_ARG, "a tensor on cuda:%d, the current device is cuda:%d" % (t.get_device(), device))
    return device


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr() or None


def _offsets(samples: Optional[torch.Tensor], what: str) -> int:
    """Number of samples of a vector of offsets."""
    if samples is None:
        return 0
    if samples.dim() != 1 or samples.shape[0] < 1 or samples.dtype != torch.int32 or not samples.is_contiguous():
        raise HeError(HE_ERR_INVALID_ARG, "%s: %s %s, contiguous int32 offsets needed" % (what, samples.dtype, tuple(samples.shape)))
    return samples.shape[0] - 1


def he_token_log_probs(ctx: Ctx, logits: torch.Tensor, targets: torch.Tensor, top: int = 0):
    """(logp, lse, entropy: float32 [rows]; top_logp float32, top_ids int64: [rows][top], None for top = 0) of logits [rows][vocab]
    and int64 targets, of which a negative one is none."""
    what = "he_token_log_probs "
    code, stride = _dtype(logits, what + "logits"), _matrix(logits, None, None, None, what + "logits")
    rows, vocab = logits.shape
    _vector(targets, rows, torch.int64, what + "targets")
    if vocab < 1 or not 0 <= top <= min(vocab, HE_MAX_TOP):
        raise HeError(HE_ERR_INVALID_ARG, what + "top: %d of %d" % (top, vocab))
    _on_gpu(logits, targets)
    logp, lse, entropy = logits.new_empty((3, rows), dtype=torch.float32).unbind(0)
    top_logp = logits.new_empty((rows, top), dtype=torch.float32) if top else None
    top_ids = logits.new_empty((rows, top), dtype=torch.int64) if top else None
    _check(_lib.he_token_log_probs(ctx.handle, _ptr(logits), code, rows, vocab, stride, _ptr(targets), top, _ptr(logp), _ptr(lse),
                                   _ptr(entropy), _ptr(top_logp), _ptr(top_ids), _stream()), "he_token_log_probs")
    return logp, lse, entropy, top_logp, top_ids


def he_token_log_probs_backward(ctx: Ctx, logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, dlogp: torch.Tensor,
                                entropy: Optional[torch.Tensor] = None, dentropy: Optional[torch.Tensor] = None,
                                top_ids: Optional[torch.Tensor] = None, dtop: Optional[torch.Tensor] = None,
                                out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of the logits, of their type, from those of logp and, where given, of the entropy and of the alternatives; `out` may
    be the logits themselves."""
    what = "he_token_log_probs_backward "
    code, stride = _dtype(logits, what + "logits"), _matrix(logits, None, None, None, what + "logits")
    rows, vocab = logits.shape
    _vector(targets, rows, torch.int64, what + "targets")
    _vector(lse, rows, torch.float32, what + "lse")
    _vector(dlogp, rows, torch.float32, what + "dlogp")
    if dentropy is not None:
        if entropy is None:
            raise HeError(HE_ERR_INVALID_ARG, what + "dentropy needs the entropy")
        _vector(entropy, rows, torch.float32, what + "entropy")
        _vector(dentropy, rows, torch.float32, what + "dentropy")
    top = 0
    if (top_ids is None) != (dtop is None):
        raise HeError(HE_ERR_INVALID_ARG, what + "top_ids and dtop go together")
    if top_ids is not None:
        top = top_ids.shape[1] if top_ids.dim() == 2 else -1
        if not 0 <= top <= min(vocab, HE_MAX_TOP) or top_ids.shape != (rows, top) or dtop.shape != (rows, top) or top_ids.dtype != torch.int64 or \
                dtop.dtype != torch.float32 or not top_ids.is_contiguous() or not dtop.is_contiguous():
            raise HeError(HE_ERR_INVALID_ARG, what + "top_ids %s and dtop %s" % (tuple(top_ids.shape), tuple(dtop.shape)))
    if vocab < 1:
        raise HeError(HE_ERR_INVALID_ARG, what + "logits: no columns")
    if out is not None:
        _matrix(out, rows, vocab, logits.dtype, what + "out", out=True)
    _on_gpu(logits, targets, lse, dlogp, entropy, dentropy, top_ids, dtop, out)
    if out is None:
        out = logits.new_empty((rows, vocab))
    _check(_lib.he_token_log_probs_backward(ctx.handle, _ptr(logits), code, rows, vocab, stride, _ptr(targets), _ptr(lse), _ptr(dlogp),
                                            _ptr(entropy) if dentropy is not None else None, _ptr(dentropy), top, _ptr(top_ids) if top else None,
                                            _ptr(dtop) if top else None, _ptr(out), out.stride(0) if rows > 1 else vocab, _stream()),
           "he_token_log_probs_backward")
    return out


def _norm_weights(weight: Optional[torch.Tensor], bias: Optional[torch.Tensor], width: int, x: torch.Tensor, what: str) -> int:
    """Type of the weights: float32 or x's, both the same."""
    first = weight if weight is not None else bias
    if first is None:
        return HE_F32
    _vector(first, width, torch.float32, what + "weights", x.dtype)
    if bias is not None and bias is not first:
        _vector(bias, width, torch.float32, what + "bias", x.dtype)
        if bias.dtype != first.dtype:
            raise HeError(HE_ERR_INVALID_ARG, what + "weight and bias: %s and %s" % (first.dtype, bias.dtype))
    return _DTYPES[first.dtype]


def he_layer_norm(ctx: Ctx, x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                  out: Optional[torch.Tensor] = None):
    """(y of x's type, mean, rstd: float32 [rows]) of the rows of x; `out` may be x itself."""
    what = "he_layer_norm "
    code, stride = _dtype(x, what + "x"), _matrix(x, None, None, None, what + "x")
    rows, width = x.shape
    kind = _norm_weights(weight, bias, width, x, what)
    if width < 1 or not eps >= 0:
        raise HeError(HE_ERR_INVALID_ARG, what + "width %d, eps %g" % (width, eps))
    if out is not None:
        _matrix(out, rows, width, x.dtype, what + "out", out=True)
    _on_gpu(x, weight, bias, out)
    if out is None:
        out = x.new_empty((rows, width))
    mean, rstd = x.new_empty((2, rows), dtype=torch.float32).unbind(0)
    _check(_lib.he_layer_norm(ctx.handle, _ptr(x), code, rows, width, stride, _ptr(weight), _ptr(bias), kind, eps, _ptr(out),
                              out.stride(0) if rows > 1 else width, _ptr(mean), _ptr(rstd), _stream()), "he_layer_norm")
    return out, mean, rstd


def he_layer_norm_backward(ctx: Ctx, dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                           weight: Optional[torch.Tensor] = None, samples: Optional[torch.Tensor] = None):
    """(dx of x's type, dweight, dbias: float32 [width]).  With the offsets of samples the last two are the map's entries, sums over
    samples of magnitudes; without, gradients over all rows."""
    what = "he_layer_norm_backward "
    code, stride = _dtype(x, what + "x"), _matrix(x, None, None, None, what + "x")
    rows, width = x.shape
    dy_stride = _matrix(dy, rows, width, x.dtype, what + "dy")
    _vector(mean, rows, torch.float32, what + "mean")
    _vector(rstd, rows, torch.float32, what + "rstd")
    kind = _norm_weights(weight, None, width, x, what)
    count = _offsets(samples, what + "samples")
    if width < 1:
        raise HeError(HE_ERR_INVALID_ARG, what + "x: no columns")
    _on_gpu(x, dy, mean, rstd, weight, samples)
    dx = x.new_empty((rows, width))
    dweight, dbias = x.new_empty((2, width), dtype=torch.float32).unbind(0)
    room = max(_lib.he_layer_norm_backward_work_bytes(ctx.handle, rows, width), 16)
    work = x.new_empty(room, dtype=torch.uint8)
    _check(_lib.he_layer_norm_backward(ctx.handle, _ptr(dy), dy_stride, _ptr(x), stride, code, rows, width, _ptr(mean), _ptr(rstd), _ptr(weight),
                                       kind, _ptr(samples), count, _ptr(dx), width, _ptr(dweight), _ptr(dbias), _ptr(work), room,
                                       _stream()), "he_layer_norm_backward")
    return dx, dweight, dbias


def _rows_aligned(t: torch.Tensor, stride: int, width: int) -> bool:
    return stride >= width and t.data_ptr() % 16 == 0 and stride * t.element_size() % 16 == 0


def he_linear_sensitivity(ctx: Ctx, x: torch.Tensor, dy: torch.Tensor, samples: Optional[torch.Tensor] = None,
                          out: Optional[torch.Tensor] = None, out_bias: Optional[torch.Tensor] = None, accumulate: bool = False,
                          bias: bool = True):
    """(float32 [outputs][inputs], float32 [outputs] or None without bias): a linear layer's entries of the map from its inputs
    x [rows][inputs] and its outputs' gradients dy [rows][outputs], summed over samples, or over rows without offsets; with `accumulate`
    added to what out and out_bias hold."""
    what = "he_linear_sensitivity "
    code, stride = _dtype(x, what + "x"), _matrix(x, None, None, None, what + "x")
    rows, inputs = x.shape
    dy_stride = _matrix(dy, rows, None, x.dtype, what + "dy")
    outputs = dy.shape[1]
    count = _offsets(samples, what + "samples")
    if inputs < 1 or outputs < 1:
        raise HeError(HE_ERR_INVALID_ARG, what + "%d inputs, %d outputs" % (inputs, outputs))
    if accumulate and (out is None or (bias and out_bias is None)):
        raise HeError(HE_ERR_INVALID_ARG, what + "nothing to add to")
    if out is not None:
        _matrix(out, outputs, inputs, torch.float32, what + "out", out=True)
        if not out.is_contiguous():
            raise HeError(HE_ERR_INVALID_ARG, what + "out is not contiguous")
    if out_bias is not None:
        _vector(out_bias, outputs, torch.float32, what + "out_bias")
    _on_gpu(x, dy, samples, out, out_bias)
    if out is None:
        out = x.new_empty((outputs, inputs), dtype=torch.float32)
    if bias and out_bias is None:
        out_bias = x.new_empty(outputs, dtype=torch.float32)
    aligned = _rows_aligned(x, stride, inputs) and _rows_aligned(dy, dy_stride, outputs)
    room = max(_lib.he_linear_sensitivity_work_bytes(ctx.handle, code, rows, inputs, outputs, samples is not None, aligned), 16)
    work = x.new_empty(room, dtype=torch.uint8)
    _check(_lib.he_linear_sensitivity(ctx.handle, _ptr(x), stride, _ptr(dy), dy_stride, code, rows, inputs, outputs, _ptr(samples), count,
                                      1 if accumulate else 0, _ptr(out), _ptr(out_bias) if bias else None, _ptr(work), room, _stream()),
           "he_linear_sensitivity")
    return out, out_bias if bias else None
