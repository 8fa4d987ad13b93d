"""Binding of libmixllm_hip.so: argument marshalling only - ctypes, and for the calls a model makes for every
layer the native module _calls (csrc/pycalls.cpp).

PyTorch supplies device memory (tensors) and the current HIP stream; every step of the
quantized linear runs in the library's own kernels.  There is no fallback: if the shared
library is missing the import of `lib()` raises."""
import ctypes as C
import os
from copy import copy
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree build; MIXLLM_LIB names another build of the same sources (say one made with other launch
# constants through MIXLLM_EXTRA_FLAGS / MIXLLM_LIB_OUT of the build script, to be measured with bench.py)
LIB_PATH = os.environ.get("MIXLLM_LIB") or os.path.join(HERE, "libmixllm_hip.so")
GROUP = 128

PATH_AUTO, PATH_GENERIC, PATH_DECODE, PATH_PREFILL = 0, 1, 2, 3
PATH_DECODE_STREAM, PATH_DECODE_RESIDENT, PATH_DECODE_SPLIT, PATH_MID = 4, 5, 6, 7
PATH_PREFILL_32, PATH_PREFILL_64, PATH_PREFILL_128 = 8, 9, 10


class MixllmError(RuntimeError):
    """A call into the library returned a status other than MIXLLM_OK (kept in .status)."""

    def __init__(self, message: str, status: int = 0):
        super().__init__(message)
        self.status = status


class _Desc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("M", "K", "N", "n8", "group", "act_group", "w8_group")]


class _Sizes(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("w8_bytes", "w4_bytes", "scales8_bytes", "scales4_bytes",
                                          "zeros4_bytes", "perm_bytes", "xq_bytes", "xscale_bytes",
                                          "y_bytes", "workspace_bytes", "linear_workspace_bytes")]


class _Epilogue(C.Structure):
    _fields_ = [("bias", C.c_void_p), ("residual", C.c_void_p), ("activation", C.c_int32), ("gated", C.c_int32)]


class _RouteDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("T", "E", "top_k", "logits_fp16", "logits_stride", "score", "groups", "top_groups",
                                         "group_score", "renormalize")] + [("scale", C.c_float)]


class _Expert(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("packed_w4", "packed_w8", "scales4", "scales8", "zeros4", "feature_perm")] + \
               [("n8", C.c_int32), ("reserved", C.c_int32)]


_lib = None
_native = None
_VP = C.c_void_p


def lib():
    """Load the shared library (built in-tree by paper_2412_14590_amd/build.py)."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MixllmError(f"{LIB_PATH} is missing: build it with `python -m paper_2412_14590_amd.build` "
                              "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(LIB_PATH)
        L.mixllm_status_string.restype = C.c_char_p
        L.mixllm_status_string.argtypes = [C.c_int]
        L.mixllm_abi_version.restype = C.c_int
        L.mixllm_query_sizes.argtypes = [C.POINTER(_Desc), C.POINTER(_Sizes)]
        L.mixllm_build_feature_perm.argtypes = [C.c_int32, C.c_int32, _VP, _VP]
        L.mixllm_quantize_weights.argtypes = [C.POINTER(_Desc)] + [_VP] * 9
        L.mixllm_pack_weights.argtypes = [C.POINTER(_Desc)] + [_VP] * 13
        L.mixllm_unpack_weights.argtypes = [C.POINTER(_Desc)] + [_VP] * 13
        L.mixllm_quantize_activations.argtypes = [C.POINTER(_Desc)] + [_VP] * 4
        L.mixllm_mixed_linear.argtypes = [C.POINTER(_Desc)] + [_VP] * 10 + [C.c_size_t, _VP]
        L.mixllm_mixed_linear_path.argtypes = [C.POINTER(_Desc)] + [_VP] * 10 + [C.c_size_t, C.c_int, _VP]
        L.mixllm_debug_group_partials.argtypes = [C.POINTER(_Desc)] + [_VP] * 6 + [C.c_int, _VP]
        L.mixllm_debug_channel_sums.argtypes = [C.POINTER(_Desc)] + [_VP] * 9 + [C.c_int, _VP]
        L.mixllm_mixed_linear_fp16.argtypes = [C.POINTER(_Desc)] + [_VP] * 9 + [C.c_size_t, _VP]
        L.mixllm_mixed_linear_fp16_static.argtypes = [C.POINTER(_Desc)] + [_VP] * 9
        L.mixllm_channel_salience.argtypes = [C.POINTER(_Desc), _VP, _VP, C.c_float, C.c_int, _VP, _VP]
        L.mixllm_select_salient_workspace.argtypes = [C.c_int32]
        L.mixllm_select_salient_workspace.restype = C.c_size_t
        L.mixllm_select_salient.argtypes = [_VP, _VP, C.c_int32, C.c_int64, _VP, _VP, _VP, C.c_size_t, _VP]
        L.mixllm_debug_check_fast_division.argtypes = [_VP, _VP]
        L.mixllm_debug_check_fast_division.restype = C.c_int
        L.mixllm_debug_work_split.argtypes = [C.POINTER(_Desc), C.c_int, _VP]
        L.mixllm_debug_work_split.restype = C.c_int
        L.mixllm_mixed_linear_epilogue.argtypes = [C.POINTER(_Desc)] + [_VP] * 8 + [C.POINTER(_Epilogue)] + [_VP] * 2 + [C.c_size_t, _VP]
        L.mixllm_mixed_linear_fp16_epilogue.argtypes = [C.POINTER(_Desc)] + [_VP] * 7 + [C.POINTER(_Epilogue)] + [_VP] * 2 + [C.c_size_t, _VP]
        L.mixllm_route_workspace.argtypes = [C.POINTER(_RouteDesc)]
        L.mixllm_route_workspace.restype = C.c_size_t
        L.mixllm_route_experts.argtypes = [C.POINTER(_RouteDesc)] + [_VP] * 9 + [C.c_size_t, _VP]
        L.mixllm_experts_table_bytes.argtypes = [C.c_int32]
        L.mixllm_experts_table_bytes.restype = C.c_size_t
        L.mixllm_experts_table.argtypes = [C.POINTER(_Desc), C.c_int32, C.POINTER(_Expert), _VP, _VP]
        L.mixllm_experts_workspace.argtypes = [C.POINTER(_Desc)]
        L.mixllm_experts_workspace.restype = C.c_size_t
        L.mixllm_experts_linear.argtypes = [C.POINTER(_Desc), C.c_int32] + [_VP] * 5 + [C.c_int32, C.POINTER(_Epilogue)] + [_VP] * 2
        L.mixllm_experts_linear_fp16.argtypes = [C.POINTER(_Desc), C.c_int32] + [_VP] * 4 + [C.c_int32, C.POINTER(_Epilogue)] + \
            [_VP] * 2 + [C.c_size_t, _VP]
        L.mixllm_experts_combine.argtypes = [C.c_int32] * 4 + [_VP] * 6
        L.mixllm_channel_salience.restype = C.c_int
        L.mixllm_select_salient.restype = C.c_int
        for name in ("mixllm_mixed_linear_epilogue", "mixllm_mixed_linear_fp16_epilogue", "mixllm_route_experts", "mixllm_experts_table",
                     "mixllm_experts_linear", "mixllm_experts_linear_fp16", "mixllm_experts_combine",
                     "mixllm_query_sizes", "mixllm_build_feature_perm", "mixllm_quantize_weights",
                     "mixllm_pack_weights", "mixllm_unpack_weights", "mixllm_quantize_activations",
                     "mixllm_mixed_linear", "mixllm_mixed_linear_path", "mixllm_debug_group_partials",
                     "mixllm_mixed_linear_fp16", "mixllm_mixed_linear_fp16_static", "mixllm_debug_channel_sums"):
            getattr(L, name).restype = C.c_int
        try:
            from . import _calls
        except ImportError as e:
            raise MixllmError(f"{os.path.join(HERE, '_calls.so')} is missing or does not load ({e}): build it with "
                              "`python -m paper_2412_14590_amd.build` (there is no fallback)") from e
        _calls.bind(*(C.cast(f, _VP).value for f in (L.mixllm_query_sizes, L.mixllm_quantize_activations,
                                                     L.mixllm_mixed_linear_path, L.mixllm_mixed_linear_fp16,
                                                     L.mixllm_mixed_linear_epilogue, L.mixllm_mixed_linear_fp16_epilogue,
                                                     L.mixllm_route_workspace, L.mixllm_route_experts, L.mixllm_experts_workspace,
                                                     L.mixllm_experts_linear, L.mixllm_experts_linear_fp16, L.mixllm_experts_combine,
                                                     L.mixllm_experts_table_bytes)))
        _native = _calls
        _lib = L
    return _lib


def _calls():
    """The native module, bound to the loaded library."""
    if _native is None:
        lib()
    return _native


def _result(r, what: str):
    """What a native call returned: its result, or a status as a number."""
    if type(r) is int:
        _check(r, what)
    return r


def _check(rc: int, what: str):
    if rc != 0:
        raise MixllmError(f"{what}: {lib().mixllm_status_string(rc).decode()} ({rc})", rc)


def abi_version() -> int:
    return int(lib().mixllm_abi_version())


def _desc(M, K, N, n8, act_group=None, w8_group=None) -> _Desc:
    return _Desc(int(M), int(K), int(N), int(n8), GROUP,
                 int(K if act_group is None else act_group), int(K if w8_group is None else w8_group))


def query_sizes(M, K, N, n8, act_group=None, w8_group=None) -> dict:
    d, s = _desc(M, K, N, n8, act_group, w8_group), _Sizes()
    _check(lib().mixllm_query_sizes(C.byref(d), C.byref(s)), "mixllm_query_sizes")
    return {n: int(getattr(s, n)) for n, _ in _Sizes._fields_}


def build_feature_perm(N: int, salient_idx) -> np.ndarray:
    sal = np.ascontiguousarray(salient_idx, dtype=np.int32)
    perm = np.empty(N, np.int32)
    _check(lib().mixllm_build_feature_perm(N, sal.size, sal.ctypes.data, perm.ctypes.data),
           "mixllm_build_feature_perm")
    return perm


def _ptr(t: Optional[torch.Tensor]):
    if t is None or t.numel() == 0:
        return None
    assert t.is_cuda and t.is_contiguous(), "device, contiguous tensors only"
    return t.data_ptr()


def _stream():
    # the current stream of the current device as an integer: the same value as
    # torch.cuda.current_stream().cuda_stream without the Stream object made around it (2.8 us a call).
    # The name is private to torch: a test compares it with the public value
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _version(t: torch.Tensor):
    return None if t.is_inference() else t._version


def _keeps_pairs(perm):
    """Of orders [.., N] with an even number of channels in either part (tensor or numpy array): every even place has an even
    channel, and the place after it the next."""
    return ((perm[..., 0::2] % 2 == 0) & (perm[..., 1::2] == perm[..., 0::2] + 1)).all(-1)


@dataclass
class PackedLayer:
    """Packed, quantized weights of one linear layer, resident in HBM."""
    K: int
    N: int
    n8: int
    w8_group: int
    w8: torch.Tensor        # uint8 buffers in the library's packed layouts
    w4: torch.Tensor
    s8: torch.Tensor
    s4: torch.Tensor
    z4: torch.Tensor
    perm: torch.Tensor      # int32 [N]

    _seen = None   # (perm, its version, n8, whether they keep pairs): what `pairs` found the last time it looked (no field)

    @property
    def pairs(self) -> bool:
        """Whether gated products can be asked for: row 2 j of either part is channel 2 i, and row 2 j + 1 channel 2 i + 1.  The order
        lies on the device: the first look at it waits for it, a later one is free while neither perm nor n8 changes (a list
        that quantize_weights got from the host was looked at there).  During a capture nothing can be waited for."""
        seen, version = self._seen, _version(self.perm)
        if seen is None or seen[0] is not self.perm or seen[1:3] != (version, self.n8):
            if self.N % 2 or self.n8 % 2:
                return False
            assert not (self.perm.is_cuda and torch.cuda.is_current_stream_capturing()), \
                "gated: whether a layer keeps pairs is not known before its first gated call (or a look at .pairs), which cannot be in a capture"
            seen = self._seen = (self.perm, version, self.n8, bool(_keeps_pairs(self.perm)))
        return seen[3]

    def desc(self, M=0, act_group=None):
        return _desc(M, self.K, self.N, self.n8, act_group, self.w8_group)

    def weight_bytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.w8, self.w4, self.s8, self.s4, self.z4, self.perm))

    def clone(self) -> "PackedLayer":
        return PackedLayer(self.K, self.N, self.n8, self.w8_group, self.w8.clone(), self.w4.clone(),
                           self.s8.clone(), self.s4.clone(), self.z4.clone(), self.perm.clone())


def _alloc_layer(K, N, n8, w8_group, device) -> PackedLayer:
    w8_group = K if w8_group is None else w8_group
    sz = query_sizes(0, K, N, n8, None, w8_group)
    u8 = lambda n: torch.empty(n, dtype=torch.uint8, device=device)
    return PackedLayer(K, N, n8, w8_group, u8(sz["w8_bytes"]), u8(sz["w4_bytes"]), u8(sz["scales8_bytes"]),
                       u8(sz["scales4_bytes"]), u8(sz["zeros4_bytes"]),
                       torch.empty(N, dtype=torch.int32, device=device))


def quantize_weights(W: torch.Tensor, salient_idx, w8_group=None) -> PackedLayer:
    """Offline: fp16 W [N,K] on the device + the list of 8-bit channels -> packed layer.  The list is
    an int32 device tensor (say a slice of select_salient's result: nothing crosses to the host), or a
    host sequence / numpy array, which is checked (range, duplicates) and copied to the device here."""
    assert W.dtype == torch.float16 and W.dim() == 2
    N, K = W.shape
    order = None
    if isinstance(salient_idx, torch.Tensor):
        sal = salient_idx.to(device=W.device, dtype=torch.int32).contiguous()
    else:
        host = np.ascontiguousarray(salient_idx, dtype=np.int32)
        order = build_feature_perm(N, host)  # raises on an index out of range or a duplicate
        sal = torch.from_numpy(host).to(W.device)
    L = _alloc_layer(K, N, int(sal.numel()), w8_group, W.device)
    d = L.desc()
    _check(lib().mixllm_quantize_weights(C.byref(d), _ptr(W), _ptr(sal), _ptr(L.w8), _ptr(L.w4), _ptr(L.s8),
                                         _ptr(L.s4), _ptr(L.z4), _ptr(L.perm), _stream()), "mixllm_quantize_weights")
    if order is not None and N % 2 == 0 and L.n8 % 2 == 0:
        L._seen = (L.perm, _version(L.perm), L.n8, bool(_keeps_pairs(order)))
    return L


def pack_weights(q8, s8, q4, s4, z4, perm, K: int, w8_group=None) -> PackedLayer:
    """Canonical device tensors (q8 int8 [n8,K], s8 fp16, q4 uint8 [n4,K], s4 fp16 [n4,K/128],
    z4 uint8 [n4,K/128], perm int32 [N]) -> packed layer."""
    N = perm.numel()
    n8 = 0 if q8 is None else q8.shape[0]
    L = _alloc_layer(K, N, n8, w8_group, perm.device)
    d = L.desc()
    _check(lib().mixllm_pack_weights(C.byref(d), _ptr(q8), _ptr(s8), _ptr(q4), _ptr(s4), _ptr(z4), _ptr(perm),
                                     _ptr(L.w8), _ptr(L.w4), _ptr(L.s8), _ptr(L.s4), _ptr(L.z4), _ptr(L.perm),
                                     _stream()), "mixllm_pack_weights")
    return L


def unpack_weights(L: PackedLayer) -> dict:
    """Packed layer -> canonical device tensors (inverse of pack_weights)."""
    dev = L.perm.device
    n4, ng = L.N - L.n8, L.K // GROUP
    ng8 = L.K // L.w8_group
    out = {
        "q8": torch.empty((L.n8, L.K), dtype=torch.int8, device=dev),
        "s8": torch.empty((L.n8, ng8), dtype=torch.float16, device=dev),
        "q4": torch.empty((n4, L.K), dtype=torch.uint8, device=dev),
        "s4": torch.empty((n4, ng), dtype=torch.float16, device=dev),
        "z4": torch.empty((n4, ng), dtype=torch.uint8, device=dev),
        "perm": torch.empty(L.N, dtype=torch.int32, device=dev),
    }
    d = L.desc()
    _check(lib().mixllm_unpack_weights(C.byref(d), _ptr(L.w8), _ptr(L.w4), _ptr(L.s8), _ptr(L.s4), _ptr(L.z4),
                                       _ptr(L.perm), _ptr(out["q8"]), _ptr(out["s8"]), _ptr(out["q4"]),
                                       _ptr(out["s4"]), _ptr(out["z4"]), _ptr(out["perm"]), _stream()),
           "mixllm_unpack_weights")
    return out


def quantize_activations(x: torch.Tensor, act_group=None, out=None):
    """fp16 x [M,K] -> (xq int8 [M,K], xscale fp16 [M, K/act_group])."""
    return _result(_calls().quantize_activations(x, act_group, out, _stream()), "mixllm_quantize_activations")


def mixed_linear(xq: torch.Tensor, xs: torch.Tensor, L: PackedLayer, path: int = PATH_AUTO, out=None, workspace=None):
    """The quantized linear: (xq, xscale, packed layer) -> y fp16 [M,N] in original channel order.
    `workspace` (optional uint8 tensor, query_sizes()['linear_workspace_bytes']) lets the tiled path split K."""
    return _result(_calls().mixed_linear(xq, xs, L.K, L.N, L.n8, L.w8_group, L.w8, L.w4, L.s8, L.s4, L.z4, L.perm, path, out,
                                         workspace, _stream()), "mixllm_mixed_linear")


def debug_group_partials(xq: torch.Tensor, L: PackedLayer, path: int = PATH_AUTO) -> torch.Tensor:
    """Exact int32 partial sums P [M,N,K/128] (original channel order) from the chosen path."""
    M, K = xq.shape
    assert K == L.K
    P = torch.empty((M, L.N, K // GROUP), dtype=torch.int32, device=xq.device)
    d = L.desc(M)
    _check(lib().mixllm_debug_group_partials(C.byref(d), _ptr(xq), _ptr(L.w4), _ptr(L.w8), _ptr(L.z4),
                                             _ptr(L.perm), _ptr(P), path, _stream()),
           "mixllm_debug_group_partials")
    return P


def debug_channel_sums(xq: torch.Tensor, xs: torch.Tensor, L: PackedLayer, path: int = PATH_PREFILL) -> torch.Tensor:
    """S [M,N] int32 = the per-group partial sums added up over the groups, from the kernels the
    linear launches for this shape (generic or tiled path)."""
    M, K = xq.shape
    assert K == L.K
    S = torch.empty((M, L.N), dtype=torch.int32, device=xq.device)
    d = L.desc(M, K // xs.shape[1])
    _check(lib().mixllm_debug_channel_sums(C.byref(d), _ptr(xq), _ptr(xs), _ptr(L.w4), _ptr(L.w8), _ptr(L.s4),
                                           _ptr(L.s8), _ptr(L.z4), _ptr(L.perm), _ptr(S), path, _stream()),
           "mixllm_debug_channel_sums")
    return S


def linear(x: torch.Tensor, L: PackedLayer, act_group=None, path: int = PATH_AUTO) -> torch.Tensor:
    """fp16 x [M,K] -> fp16 y [M,N]: activation quantizer followed by the quantized linear."""
    xq, xs = quantize_activations(x, act_group)
    return mixed_linear(xq, xs, L, path)


def linear_fp16(x: torch.Tensor, L: PackedLayer, act_group=None, out=None, workspace=None) -> torch.Tensor:
    """fp16 x [M,K] -> fp16 y [M,N] through mixllm_mixed_linear_fp16: one kernel for a single token
    where the decode kernel can quantize its own activations, otherwise quantizer + linear with
    xq / xscale in `workspace` (a uint8 tensor of query_sizes()['workspace_bytes'], allocated here
    when not given)."""
    return _result(_calls().linear_fp16(x, L.K, L.N, L.n8, L.w8_group, L.w8, L.w4, L.s8, L.s4, L.z4, L.perm,
                                        L.K if act_group is None else act_group, out, workspace, _stream()),
                   "mixllm_mixed_linear_fp16")


def linear_fp16_static(x: torch.Tensor, L: PackedLayer, out: torch.Tensor, act_group=None) -> torch.Tensor:
    """mixllm_mixed_linear_fp16_static: the same as linear_fp16 with the scratch inside the library; the
    caller brings the output tensor, and nothing is allocated on the way."""
    assert x.dtype == torch.float16 and x.dim() == 2 and x.shape[1] == L.K
    assert out.dtype == torch.float16 and out.shape == (x.shape[0], L.N)
    d = L.desc(x.shape[0], act_group)
    _check(lib().mixllm_mixed_linear_fp16_static(C.byref(d), _ptr(x), _ptr(L.w4), _ptr(L.w8), _ptr(L.s4), _ptr(L.s8),
                                                 _ptr(L.z4), _ptr(L.perm), _ptr(out), _stream()),
           "mixllm_mixed_linear_fp16_static")
    return out


ACTIVATIONS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
SCORES = {"softmax": 0, "sigmoid": 1}
GROUP_SCORES = {"max": 0, "top2": 1}


def _named(table: dict, name, what: str) -> int:
    if name not in table:
        raise ValueError(f"{what} is one of {', '.join(repr(n) for n in table)}, got {name!r}")
    return table[name]


def _check_pairs(L: PackedLayer):
    # (a layer that is not on the device is refused with the other operands)
    assert not L.perm.is_cuda or L.pairs, "gated: the layer's order keeps channels 2 i and 2 i + 1 next to each other, in one part (PackedLayer.pairs)"


def mixed_linear_epilogue(xq: torch.Tensor, xs: torch.Tensor, L: PackedLayer, bias=None, activation=None, gated: bool = False,
                          residual=None, out=None, workspace=None) -> torch.Tensor:
    """mixed_linear with bias [N], activation (ACTIVATIONS) and residual (of y's shape; may be `out` itself, which otherwise
    overlaps no operand) done on its fp32 sums:
    y = act(x W^T + bias) + residual.  gated: rows 2 i and 2 i + 1 of W are gate and up of output i and next to each other in the
    packed layer (L.pairs: both 8-bit or neither; lists of either part in ascending order do), and
    y [M, N/2] = act(gate) up + residual."""
    if gated:
        _check_pairs(L)
    return _result(_calls().mixed_linear_epilogue(xq, xs, L.K, L.N, L.n8, L.w8_group, L.w8, L.w4, L.s8, L.s4, L.z4, L.perm, bias, residual,
                                                  _named(ACTIVATIONS, activation, "activation"), gated, out, workspace, _stream()),
                   "mixllm_mixed_linear_epilogue")


def linear_fp16_epilogue(x: torch.Tensor, L: PackedLayer, bias=None, activation=None, gated: bool = False, residual=None,
                         act_group=None, out=None, workspace=None) -> torch.Tensor:
    """linear_fp16 with the epilogue of mixed_linear_epilogue: fp16 x [M,K] in, fp16 y out, one kernel for a token."""
    if gated:
        _check_pairs(L)
    return _result(_calls().linear_fp16_epilogue(x, L.K, L.N, L.n8, L.w8_group, L.w8, L.w4, L.s8, L.s4, L.z4, L.perm,
                                                 L.K if act_group is None else act_group, bias, residual,
                                                 _named(ACTIVATIONS, activation, "activation"), gated, out, workspace, _stream()),
                   "mixllm_mixed_linear_fp16_epilogue")


@dataclass
class Route:
    """Which experts every token takes, and the assignments (token * top_k + j) sorted by expert."""
    ids: torch.Tensor       # int32 [T, top_k], -1 = none
    weights: torch.Tensor   # fp32 [T, top_k]
    offsets: torch.Tensor   # int32 [E + 1]: place of every expert's first assignment
    rows: torch.Tensor      # int32 [T * top_k]: assignment at every place, -1 behind the last
    slots: torch.Tensor     # int32 [T, top_k]: place of every assignment, -1 = none


def route_experts(logits: torch.Tensor, top_k: int, score: str = "softmax", bias=None, mask=None, groups: int = 1, top_groups: int = 1,
                  group_score: str = "max", renormalize: bool = True, scale: float = 1.0) -> Route:
    """Router: logits fp16 or fp32 [T,E] -> Route.  score "softmax" or "sigmoid"; bias fp32 [E] moves the choice, not the weights;
    mask [T] (bool): False = padding; with groups > 1 only the experts of the top_groups best groups are chosen from, a group's
    score being its best expert's ("max") or the sum of its two best ("top2").  An expert with a logit of -inf is never taken."""
    return Route(*_result(_calls().route_experts(logits, top_k, _named(SCORES, score, "score"), bias, mask, groups, top_groups,
                                                 _named(GROUP_SCORES, group_score, "group_score"), renormalize, scale, _stream()),
                          "mixllm_route_experts"))


@dataclass
class PackedExperts:
    """The packed layers of one linear of a layer of experts, and the device table through which the kernels reach them.  The table
    holds addresses: the tensors behind them live as long as this does.  Weights written into these tensors are used from then
    on; a PackedLayer that gets other tensors is another layer, and packed into experts anew."""
    K: int
    N: int
    w8_group: int
    layers: tuple           # of PackedLayer: what the table points to
    table: torch.Tensor
    n8: int                 # the most 8-bit channels of any of them
    pairs: bool = True      # all keep pairs (PackedLayer.pairs): gated products can be asked for
    held: tuple = ()        # the tensors whose addresses the table has

    @property
    def E(self) -> int:
        return len(self.layers)


def _all_keep_pairs(layers) -> bool:
    """PackedLayer.pairs of all of them (of one N), with one wait for the device."""
    if any(L.N % 2 or L.n8 % 2 for L in layers):
        return False
    new = [L for L in layers if L._seen is None]
    if new and new[0].perm.is_cuda and torch.cuda.is_current_stream_capturing():
        return False
    if new:
        some = max(1, (1 << 24) // new[0].N)   # orders looked at together: 64 MB of copies
        answers = [_keeps_pairs(torch.stack([L.perm for L in new[i:i + some]])) for i in range(0, len(new), some)]
        for L, keeps in zip(new, torch.cat(answers).tolist()):
            L._seen = (L.perm, _version(L.perm), L.n8, keeps)
    return all(L.pairs for L in layers)


def pack_experts(layers) -> PackedExperts:
    """Packed layers of one K, N and w8_group (each with its own 8-bit channels) -> the experts of one linear."""
    layers = list(layers)
    assert layers and all((L.K, L.N, L.w8_group, L.perm.device) == (layers[0].K, layers[0].N, layers[0].w8_group, layers[0].perm.device)
                          for L in layers), "experts of one size, granularity and device"
    first = layers[0]
    assert not first.perm.is_cuda or first.perm.device.index == torch.cuda.current_device(), "layers of the current device"
    entries = (_Expert * len(layers))(*(_Expert(_ptr(L.w4), _ptr(L.w8), _ptr(L.s4), _ptr(L.s8), _ptr(L.z4), _ptr(L.perm), L.n8, 0)
                                        for L in layers))
    table = torch.empty(int(lib().mixllm_experts_table_bytes(len(layers))), dtype=torch.uint8, device=first.perm.device)
    d = first.desc()
    _check(lib().mixllm_experts_table(C.byref(d), len(layers), entries, _ptr(table), _stream()), "mixllm_experts_table")
    pairs = _all_keep_pairs(layers)
    return PackedExperts(first.K, first.N, first.w8_group, tuple(copy(L) for L in layers), table, max(L.n8 for L in layers), pairs,
                         tuple(t for L in layers for t in (L.w4, L.w8, L.s4, L.s8, L.z4, L.perm)))


_PAIRS = "gated: every expert has an even number of 8-bit channels, and channels 2 i and 2 i + 1 next to each other in its order (PackedLayer.pairs)"


def experts_linear(xq: torch.Tensor, xs: torch.Tensor, L: PackedExperts, route: Route, bias=None, activation=None, gated: bool = False,
                   gather: bool = True, out=None) -> torch.Tensor:
    """The linears of the experts over the rows routed to them: y [T * top_k, N] (gated [.., N/2]), one row per assignment in the
    route's order; rows behind the last assignment are left as they were.  gather: xq has a row per token; otherwise one per
    assignment, in the route's order.  bias fp16 [E,N]; activation and gated as in mixed_linear_epilogue.  out does not overlap the
    activations."""
    assert L.pairs or not gated, _PAIRS
    return _result(_calls().experts_linear(xq, xs, L.K, L.N, L.w8_group, L.E, L.table, L.n8, route.offsets, route.rows, route.slots, gather, bias,
                                           _named(ACTIVATIONS, activation, "activation"), gated, out, _stream()), "mixllm_experts_linear")


def experts_linear_fp16(x: torch.Tensor, L: PackedExperts, route: Route, bias=None, activation=None, gated: bool = False,
                        gather: bool = True, act_group=None, out=None, workspace=None) -> torch.Tensor:
    """experts_linear from fp16 activations x [T,K] (gather) or [T * top_k, K]: quantizer and products."""
    assert L.pairs or not gated, _PAIRS
    return _result(_calls().experts_linear_fp16(x, L.K, L.N, L.w8_group, L.E, L.table, L.n8, route.offsets, route.rows, route.slots, gather,
                                                L.K if act_group is None else act_group, bias,
                                                _named(ACTIVATIONS, activation, "activation"), gated, out, workspace, _stream()),
                   "mixllm_experts_linear_fp16")


def experts_combine(y: torch.Tensor, route: Route, residual=None, out=None) -> torch.Tensor:
    """Sum of every token's rows of y [T * top_k, N] by the route's weights, plus the residual [T,N] (may be `out` itself,
    which otherwise overlaps no operand)."""
    return _result(_calls().experts_combine(y, route.weights, route.slots, residual, out, _stream()), "mixllm_experts_combine")


def experts_mlp(x: torch.Tensor, route: Route, gate_up: PackedExperts, down: PackedExperts, activation="silu", residual=None,
                act_group=None, bias_gate_up=None, bias_down=None) -> torch.Tensor:
    """A layer of experts: x [T,K] -> gated rows act(gate) up of every token's experts -> down -> their weighted sum + residual.
    act_group: None (one activation scale per row) or 128, for both linears."""
    h = experts_linear_fp16(x, gate_up, route, bias_gate_up, activation, gated=True, gather=True, act_group=act_group)
    y = experts_linear_fp16(h, down, route, bias_down, gather=False, act_group=act_group)
    return experts_combine(y, route, residual)


def channel_salience(W: torch.Tensor, G: torch.Tensor, out=None, weight: float = 1.0, accumulate: bool = False) -> torch.Tensor:
    """Salience of every output channel of one layer for one gradient sample (fp16 W, G [N,K] ->
    fp32 [N]); with `out`, weight and accumulate the mean over several samples is built call by call."""
    assert W.dtype == torch.float16 and G.dtype == torch.float16 and W.shape == G.shape and W.dim() == 2
    N, K = W.shape
    W, G = W.contiguous(), G.contiguous()
    sal = torch.empty(N, dtype=torch.float32, device=W.device) if out is None else out
    assert sal.dtype == torch.float32 and sal.numel() == N
    d = _desc(0, K, N, 0, None, None)
    _check(lib().mixllm_channel_salience(C.byref(d), _ptr(W), _ptr(G), C.c_float(weight), int(bool(accumulate)),
                                         _ptr(sal), _stream()), "mixllm_channel_salience")
    return sal


def select_salient(saliences, T: int):
    """The T most salient channels over all layers: `saliences` is a list of fp32 device tensors (one
    per layer); returns one ascending int32 index tensor per layer (on the device) - the salient_idx
    of quantize_weights for that layer.  It takes channels one by one.  Of layers for gated products search the pairs:
    s.view(-1, 2).sum(1) of each, T / 2 of them, and channels 2 p and 2 p + 1 of a pair p."""
    sizes = [int(s.numel()) for s in saliences]
    flat = torch.cat([s.reshape(-1).to(torch.float32) for s in saliences]) if len(saliences) > 1 else \
        saliences[0].reshape(-1).to(torch.float32).contiguous()
    L = len(sizes)
    offsets = (C.c_int64 * (L + 1))(*np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64).tolist())
    selected = torch.empty(max(int(T), 1), dtype=torch.int32, device=flat.device)
    counts = torch.empty(L, dtype=torch.int32, device=flat.device)
    need = int(lib().mixllm_select_salient_workspace(L))
    ws = torch.empty(need, dtype=torch.uint8, device=flat.device)
    _check(lib().mixllm_select_salient(_ptr(flat), C.cast(offsets, _VP), L, int(T), _ptr(selected), _ptr(counts),
                                       _ptr(ws), need, _stream()), "mixllm_select_salient")
    cnt = counts.cpu().tolist()
    out, o = [], 0
    for c in cnt:
        out.append(selected[o:o + c])
        o += c
    return out
