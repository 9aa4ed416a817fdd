"""Python binding of libmkq (MI355X-native W4A4 BERT linear layer).

Argument marshalling only: every step of the path runs in the HIP kernels of
``libmkq.so``.  PyTorch is used for device memory and streams.  There is no
fallback: if the library has not been built, loading it raises.
"""
from __future__ import annotations

import ctypes as C
import os
from array import array
from functools import lru_cache

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmkq.so")

MKQ_OK = 0
MKQ_ERR_NULL, MKQ_ERR_SHAPE, MKQ_ERR_ALIGN, MKQ_ERR_SCALE = -1, -2, -3, -4
MKQ_ERR_DTYPE, MKQ_ERR_WORKSPACE, MKQ_ERR_UNSUPPORTED, MKQ_ERR_HIP = -5, -6, -7, -8
MKQ_F32, MKQ_F16, MKQ_BF16, MKQ_I4, MKQ_I8 = 0, 1, 2, 3, 4
MKQ_ACT_NONE, MKQ_ACT_GELU = 0, 1

EXPORTS = [
    "mkq_status_string", "mkq_version", "mkq_quantize", "mkq_absmax_scale",
    "mkq_packed_weight_bytes", "mkq_pack_weights_int4", "mkq_pack_codes_int4",
    "mkq_padded_k", "mkq_quantize_padded", "mkq_pack_weights_int4_padded",
    "mkq_unpack_weights_int4", "mkq_linear_int4_workspace_bytes", "mkq_linear_int4",
    "mkq_quantize_int8", "mkq_pack_weights_int8", "mkq_linear_int8", "mkq_bert_layer_int8_workspace",
    "mkq_bert_layer_int8", "mkq_layernorm_int8", "mkq_attention_int8",
    "mkq_scale_gradients", "mkq_percentile_scale_workspace_bytes", "mkq_percentile_scale", "mkq_attention_varlen",
    "mkq_quantize_e3m2", "mkq_pack_codes_e3m2", "mkq_pack_weights_e3m2", "mkq_linear_int4_e3m2",
    "mkq_linear_fp16", "mkq_bert_layer_workspace", "mkq_bert_layer_int4",
    "mkq_bert_layer_fp16_workspace_bytes", "mkq_bert_layer_fp16", "mkq_layernorm", "mkq_attention",
    "mkq_splitk_scratch_bytes", "mkq_splitk_scratch_init", "mkq_init",
    "mkq_tuning_linear_int4", "mkq_tuning_linear_int4_e3m2", "mkq_tuning_linear_int4_stream", "mkq_tuning_linear_int8",
    "mkq_stream_weight_bytes", "mkq_repack_weights_int4_stream", "mkq_linear_int4_stream",
    "mkq_linear_int4_stream_static",
    "mkq_group_weight_bytes", "mkq_pack_weights_int4_group", "mkq_linear_int4_group",
    "mkq_embedding", "mkq_embedding_int4_group", "mkq_embedding_gradient_workspace_bytes", "mkq_embedding_gradient",
    "mkq_gradient_norm_workspace_bytes", "mkq_gradient_norm", "mkq_clip_gradients",
    "mkq_token_log_probs_workspace_bytes", "mkq_token_log_probs", "mkq_token_log_probs_gradient",
    "mkq_checkpoint_bytes", "mkq_checkpoint_int8", "mkq_checkpoint_restore", "mkq_checkpoint_gelu_gradient",
    "mkq_low_rank_adapters_workspace_bytes", "mkq_low_rank_adapters", "mkq_low_rank_adapters_gradient_workspace_bytes",
    "mkq_low_rank_adapters_gradient",
    "mkq_measure_stream", "mkq_measure_mfma_i8_operand_bytes", "mkq_measure_mfma_i8_ops", "mkq_measure_mfma_i8",
]


class MkqError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Epilogue(C.Structure):
    _fields_ = [("act", C.c_int), ("residual", C.c_void_p), ("residual_dtype", C.c_int),
                ("s_next", C.c_float), ("q_out", C.c_void_p), ("acc_out", C.c_void_p),
                ("splitk_scratch", C.c_void_p), ("splitk_scratch_bytes", C.c_size_t), ("q_pitch", C.c_int64)]


class BertLayerParams(C.Structure):
    _fields_ = ([(n, C.c_int64) for n in ("batch", "seq", "hidden", "heads", "ffn")]
                + [(n, C.c_void_p) for n in ("Wq_qkv", "Wq_ao", "Wq_up", "Wq_down",
                                             "sw_qkv", "sw_ao", "sw_up", "sw_down",
                                             "b_qkv", "b_ao", "b_up", "b_down")]
                + [(n, C.c_float) for n in ("sx_qkv", "sx_ao", "sx_up", "sx_down")]
                + [(n, C.c_void_p) for n in ("ln1_gamma", "ln1_beta", "ln2_gamma", "ln2_beta")]
                + [("ln_eps", C.c_float), ("s_out_next", C.c_float), ("next_bits", C.c_int),
                   ("cu_seqlens", C.c_void_p), ("total_tokens", C.c_int64)])


class BertLayerWorkspaceLayout(C.Structure):
    _fields_ = [(n, C.c_size_t) for n in ("c0", "qkv", "c1", "u", "h1", "c2", "c3", "d", "total")]


class BertLayerParamsFp16(C.Structure):
    _fields_ = ([(n, C.c_int64) for n in ("batch", "seq", "hidden", "heads", "ffn")]
                + [(n, C.c_void_p) for n in ("W_qkv", "W_ao", "W_up", "W_down",
                                             "b_qkv", "b_ao", "b_up", "b_down",
                                             "ln1_gamma", "ln1_beta", "ln2_gamma", "ln2_beta")]
                + [("ln_eps", C.c_float), ("cu_seqlens", C.c_void_p), ("total_tokens", C.c_int64)])


_lib = None


def load() -> C.CDLL:
    """Loads libmkq.so (built by ``python -m paper_2203_13483_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           f"`python -m paper_2203_13483_amd.build` (there is no fallback path)")
    # torch first: the device memory and streams handed to the library are torch's, so both must sit on the
    # HIP runtime that torch brings; loaded before torch, the library would pull in the system's copy instead
    _torch()
    lib = C.CDLL(LIB_PATH)
    i64, vp, f32, ci, sz = C.c_int64, C.c_void_p, C.c_float, C.c_int, C.c_size_t
    sig = {
        "mkq_status_string": (C.c_char_p, [ci]),
        "mkq_version": (ci, []),
        "mkq_quantize": (ci, [vp, ci, i64, i64, i64, f32, vp, vp]),
        "mkq_absmax_scale": (ci, [vp, ci, i64, i64, i64, ci, vp, vp]),
        "mkq_packed_weight_bytes": (sz, [i64, i64]),
        "mkq_scale_gradients": (ci, [vp, ci, i64, i64, i64, f32, ci, vp, vp]),
        "mkq_percentile_scale_workspace_bytes": (sz, []),
        "mkq_percentile_scale": (ci, [vp, ci, i64, i64, i64, i64, ci, vp, vp, sz, vp]),
        "mkq_pack_weights_int4": (ci, [vp, i64, i64, vp, vp, vp, vp]),
        "mkq_pack_codes_int4": (ci, [vp, i64, i64, vp, vp]),
        "mkq_padded_k": (i64, [i64]),
        "mkq_quantize_padded": (ci, [vp, ci, i64, i64, i64, f32, vp, vp]),
        "mkq_pack_weights_int4_padded": (ci, [vp, i64, i64, vp, vp, vp, vp]),
        "mkq_unpack_weights_int4": (ci, [vp, i64, i64, vp, vp]),
        "mkq_linear_int4_workspace_bytes": (sz, [i64, i64, i64, ci]),
        "mkq_linear_int4": (ci, [vp, ci, f32, vp, vp, vp, i64, i64, i64, vp, ci,
                                 C.POINTER(Epilogue), vp, sz, vp]),
        "mkq_tuning_linear_int4": (ci, [vp, ci, f32, vp, vp, vp, i64, i64, i64, vp, ci,
                                        C.POINTER(Epilogue), vp, sz, vp, ci, ci]),
        "mkq_tuning_linear_int4_e3m2": (ci, [vp, f32, vp, vp, vp, i64, i64, i64, vp, ci, C.POINTER(Epilogue), vp, ci]),
        "mkq_tuning_linear_int4_stream": (ci, [vp, ci, f32, vp, vp, vp, i64, i64, i64, vp, ci,
                                               C.POINTER(Epilogue), vp, sz, vp, ci, ci]),
        "mkq_linear_int4_stream": (ci, [vp, ci, f32, vp, vp, vp, i64, i64, i64, vp, ci,
                                        C.POINTER(Epilogue), vp, sz, vp]),
        "mkq_linear_int4_stream_static": (ci, [vp, f32, vp, vp, vp, i64, i64, i64, vp, ci, C.POINTER(Epilogue), vp]),
        "mkq_measure_stream": (ci, [ci, vp, vp, sz, vp]),
        "mkq_measure_mfma_i8_operand_bytes": (sz, []),
        "mkq_measure_mfma_i8_ops": (i64, [ci]),
        "mkq_measure_mfma_i8": (ci, [vp, sz, ci, vp, vp]),
        "mkq_stream_weight_bytes": (sz, [i64, i64]),
        "mkq_repack_weights_int4_stream": (ci, [vp, i64, i64, vp, vp]),
        "mkq_splitk_scratch_bytes": (sz, []),
        "mkq_splitk_scratch_init": (ci, [vp, sz, vp]),
        "mkq_init": (ci, []),
        "mkq_quantize_int8": (ci, [vp, ci, i64, i64, i64, f32, vp, vp]),
        "mkq_pack_weights_int8": (ci, [vp, i64, i64, vp, vp, vp, vp]),
        "mkq_linear_int8": (ci, [vp, f32, vp, vp, vp, i64, i64, i64, vp, ci, C.POINTER(Epilogue), vp]),
        "mkq_tuning_linear_int8": (ci, [vp, f32, vp, vp, vp, i64, i64, i64, vp, ci, C.POINTER(Epilogue), vp, ci]),
        "mkq_linear_fp16": (ci, [vp, vp, vp, i64, i64, i64, vp, ci, ci, vp, vp]),
        "mkq_quantize_e3m2": (ci, [vp, ci, i64, i64, i64, f32, vp, vp]),
        "mkq_pack_codes_e3m2": (ci, [vp, i64, i64, vp, vp]),
        "mkq_pack_weights_e3m2": (ci, [vp, i64, i64, vp, vp, vp, vp]),
        "mkq_linear_int4_e3m2": (ci, [vp, f32, vp, vp, vp, i64, i64, i64, vp, ci, C.POINTER(Epilogue), vp]),
        "mkq_bert_layer_workspace": (ci, [C.POINTER(BertLayerParams), C.POINTER(BertLayerWorkspaceLayout)]),
        "mkq_bert_layer_int4": (ci, [C.POINTER(BertLayerParams), vp, ci, vp, vp, vp, vp, sz, vp]),
        "mkq_bert_layer_fp16_workspace_bytes": (sz, [C.POINTER(BertLayerParamsFp16)]),
        "mkq_bert_layer_fp16": (ci, [C.POINTER(BertLayerParamsFp16), vp, vp, vp, sz, vp]),
        "mkq_layernorm": (ci, [vp, i64, i64, vp, vp, f32, vp, f32, vp, vp]),
        "mkq_attention": (ci, [vp, i64, i64, i64, i64, vp, f32, vp, vp]),
        "mkq_attention_varlen": (ci, [vp, vp, i64, i64, i64, i64, vp, f32, vp, ci, vp]),
        "mkq_layernorm_int8": (ci, [vp, i64, i64, vp, vp, f32, vp, f32, vp, vp]),
        "mkq_attention_int8": (ci, [vp, i64, i64, i64, i64, vp, f32, vp, vp]),
        "mkq_bert_layer_int8_workspace": (ci, [C.POINTER(BertLayerParams), C.POINTER(BertLayerWorkspaceLayout)]),
        "mkq_bert_layer_int8": (ci, [C.POINTER(BertLayerParams), vp, ci, vp, vp, vp, vp, sz, vp]),
        "mkq_group_weight_bytes": (sz, [i64, i64]),
        "mkq_pack_weights_int4_group": (ci, [vp, ci, i64, i64, i64, ci, vp, vp, vp, vp]),
        "mkq_linear_int4_group": (ci, [vp, ci, i64, vp, vp, ci, vp, i64, i64, i64, vp, ci, C.POINTER(Epilogue), vp]),
        "mkq_embedding": (ci, [vp, ci, i64, vp, ci, i64, i64, i64, f32, vp, ci, i64, vp]),
        "mkq_embedding_int4_group": (ci, [vp, ci, i64, vp, vp, ci, i64, i64, f32, vp, ci, i64, vp]),
        "mkq_embedding_gradient_workspace_bytes": (sz, [i64, i64]),
        "mkq_embedding_gradient": (ci, [vp, ci, i64, vp, ci, i64, i64, i64, f32, i64, ci, vp, ci, i64, vp, sz, vp]),
        "mkq_gradient_norm_workspace_bytes": (sz, [i64]),
        "mkq_gradient_norm": (ci, [i64, vp, vp, vp, vp, vp, sz, vp]),
        "mkq_clip_gradients": (ci, [i64, vp, vp, vp, vp, f32, vp, vp, sz, vp]),
    }
    sig.update({
        "mkq_token_log_probs_workspace_bytes": (sz, [i64, i64, ci]),
        "mkq_token_log_probs": (ci, [vp, ci, i64, i64, i64, f32, vp, ci, vp, vp, vp, ci, vp, vp, vp, sz, vp]),
        "mkq_token_log_probs_gradient": (ci, [vp, ci, i64, i64, i64, f32, vp, ci, vp, vp, vp, vp, vp, ci, i64, vp]),
        "mkq_checkpoint_bytes": (sz, [i64, i64]),
        "mkq_checkpoint_int8": (ci, [vp, ci, i64, i64, i64, ci, vp, vp, vp]),
        "mkq_checkpoint_restore": (ci, [vp, vp, ci, i64, i64, ci, vp, ci, i64, vp]),
        "mkq_checkpoint_gelu_gradient": (ci, [vp, vp, ci, i64, i64, vp, ci, i64, vp, ci, i64, vp]),
        "mkq_low_rank_adapters_workspace_bytes": (sz, [i64, i64, i64, ci, i64]),
        "mkq_low_rank_adapters": (ci, [vp, ci, i64, vp, i64, i64, i64, ci, i64, vp, vp, ci, vp, vp, i64, vp, ci, i64, vp, vp, sz, vp]),
        "mkq_low_rank_adapters_gradient_workspace_bytes": (sz, [i64, i64, i64, ci, i64]),
        "mkq_low_rank_adapters_gradient": (ci, [vp, ci, i64, vp, ci, i64, vp, ci, vp, vp, i64, i64, i64, ci, i64, vp, vp, ci, vp, vp, i64,
                                                vp, ci, i64, vp, vp, ci, ci, vp, sz, vp]),
    })
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().mkq_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != MKQ_OK:
        raise MkqError(status, where)


# What follows runs in every call, and the smallest linears are bound by their calls: addresses go to ctypes as the integers
# they are, and torch's Stream object is not built only to read its handle.  From call to call, us, with the block
# of options passed only where there are any: 128 tokens of binary32 through K = N = 768 10.4 -> 6.1, 16 rows of codes through
# K = N = 4096 9.6 -> 6.1 (the kernels are 5.8).
_torch_module = None
_dtype_codes = {}


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _dtype_codes.update({torch.float32: MKQ_F32, torch.float16: MKQ_F16, torch.bfloat16: MKQ_BF16})
        _torch_module = torch
    return _torch_module


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    if torch.cuda.is_initialized():
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:  # (names that torch does not promise to keep)
            pass
    return torch.cuda.current_stream().cuda_stream


def _dtype_code(t):
    if not _dtype_codes:
        _torch()
    return _dtype_codes[t.dtype]


_torch_dtypes = {}


def _torch_dtype(code):
    if not _torch_dtypes:
        torch = _torch()
        _torch_dtypes.update({MKQ_F32: torch.float32, MKQ_F16: torch.float16, MKQ_BF16: torch.bfloat16})
    return _torch_dtypes[code]


# ----------------------------------------------------------------------------------
# Same names as the C entry points.  Tensors are torch CUDA tensors; outputs are
# allocated with torch when not passed in.

def mkq_version() -> int:
    return int(load().mkq_version())


def mkq_quantize(x, s_x: float, q_out=None, stream=None):
    """x [M,K] float32/float16 -> packed codes uint8 [M,K/2]."""
    torch = _torch()
    M, K = x.shape
    if q_out is None:
        q_out = torch.empty((M, K // 2), dtype=torch.uint8, device=x.device)
    _check(load().mkq_quantize(_ptr(x), _dtype_code(x), M, K, x.stride(0), float(s_x), _ptr(q_out),
                               _stream(stream)), "mkq_quantize")
    return q_out


def mkq_absmax_scale(x, per_row: bool = False, s_out=None, stream=None):
    torch = _torch()
    M, K = x.shape
    if s_out is None:
        s_out = torch.empty(M if per_row else 1, dtype=torch.float32, device=x.device)
    _check(load().mkq_absmax_scale(_ptr(x), _dtype_code(x), M, K, x.stride(0), int(per_row),
                                   _ptr(s_out), _stream(stream)), "mkq_absmax_scale")
    return s_out


def mkq_scale_gradients(x, s: float, bits: int = 4, g_out=None, stream=None):
    """(STE-based, MSE-based) scale-gradient sums of x [M,K] under step s -> float64 tensor [2]."""
    torch = _torch()
    M, K = x.shape
    if g_out is None:
        g_out = torch.empty(2, dtype=torch.float64, device=x.device)
    _check(load().mkq_scale_gradients(_ptr(x), _dtype_code(x), M, K, x.stride(0), float(s), int(bits), _ptr(g_out),
                                      _stream(stream)), "mkq_scale_gradients")
    return g_out


def mkq_percentile_scale_workspace_bytes() -> int:
    return int(load().mkq_percentile_scale_workspace_bytes())


def mkq_percentile_scale(x, top_ppm: int = 100, bits: int = 4, s_out=None, workspace=None, stream=None):
    """Step from the k-th largest |x| (k = max(1, n*top_ppm // 10**6)) -> float32 tensor [1]."""
    torch = _torch()
    M, K = x.shape
    if s_out is None:
        s_out = torch.empty(1, dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = torch.empty(mkq_percentile_scale_workspace_bytes(), dtype=torch.uint8, device=x.device)
    _check(load().mkq_percentile_scale(_ptr(x), _dtype_code(x), M, K, x.stride(0), int(top_ppm), int(bits),
                                       _ptr(s_out), _ptr(workspace), workspace.numel(), _stream(stream)),
           "mkq_percentile_scale")
    return s_out


def mkq_packed_weight_bytes(N: int, K: int) -> int:
    return int(load().mkq_packed_weight_bytes(N, K))


def mkq_pack_weights_int4(W, s_w_in=None, stream=None):
    """W [N,K] float32 -> (Wq uint8 [packed bytes], s_w float32 [N])."""
    torch = _torch()
    N, K = W.shape
    nbytes = mkq_packed_weight_bytes(N, K)
    Wq = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=W.device)
    s_w = torch.empty(N, dtype=torch.float32, device=W.device)
    _check(load().mkq_pack_weights_int4(_ptr(W), N, K, _ptr(s_w_in), _ptr(s_w), _ptr(Wq),
                                        _stream(stream)), "mkq_pack_weights_int4")
    return Wq, s_w


def mkq_padded_k(K: int) -> int:
    """Smallest multiple of 128 >= K: the row length, in codes, of operands stored with zero padding."""
    return int(load().mkq_padded_k(K))


def mkq_quantize_padded(x, s_x: float, q_out=None, stream=None):
    """x [M,K] float32/float16, K % 8 == 0 -> packed codes uint8 [M, mkq_padded_k(K)/2], zero codes past K."""
    torch = _torch()
    M, K = x.shape
    if q_out is None:
        q_out = torch.empty((M, mkq_padded_k(K) // 2), dtype=torch.uint8, device=x.device)
    _check(load().mkq_quantize_padded(_ptr(x), _dtype_code(x), M, K, x.stride(0), float(s_x), _ptr(q_out),
                                      _stream(stream)), "mkq_quantize_padded")
    return q_out


def mkq_pack_weights_int4_padded(W, s_w_in=None, stream=None):
    """W [N,K] float32, K % 8 == 0 -> (Wq uint8 [N * mkq_padded_k(K)/2], s_w float32 [N])."""
    torch = _torch()
    N, K = W.shape
    Wq = torch.empty(max(N * mkq_padded_k(K) // 2, 1), dtype=torch.uint8, device=W.device)
    s_w = torch.empty(N, dtype=torch.float32, device=W.device)
    _check(load().mkq_pack_weights_int4_padded(_ptr(W), N, K, _ptr(s_w_in), _ptr(s_w), _ptr(Wq),
                                               _stream(stream)), "mkq_pack_weights_int4_padded")
    return Wq, s_w


def mkq_pack_codes_int4(codes, stream=None):
    torch = _torch()
    rows, K = codes.shape
    q = torch.empty((rows, K // 2), dtype=torch.uint8, device=codes.device)
    _check(load().mkq_pack_codes_int4(_ptr(codes), rows, K, _ptr(q), _stream(stream)),
           "mkq_pack_codes_int4")
    return q


def mkq_unpack_weights_int4(Wq, N: int, K: int, stream=None):
    torch = _torch()
    codes = torch.empty((N, K), dtype=torch.int8, device=Wq.device)
    _check(load().mkq_unpack_weights_int4(_ptr(Wq), N, K, _ptr(codes), _stream(stream)),
           "mkq_unpack_weights_int4")
    return codes


def mkq_linear_int4_workspace_bytes(M: int, N: int, K: int, a_dtype: int) -> int:
    return int(load().mkq_linear_int4_workspace_bytes(M, N, K, a_dtype))


def mkq_init() -> None:
    _check(load().mkq_init(), "mkq_init")


def mkq_splitk_scratch_bytes() -> int:
    return int(load().mkq_splitk_scratch_bytes())


def mkq_splitk_scratch_init(scratch=None, device="cuda", stream=None):
    """A scratch area for K splits across workgroups, counters cleared (allocated here when not passed in)."""
    torch = _torch()
    if scratch is None:
        scratch = torch.empty(mkq_splitk_scratch_bytes(), dtype=torch.uint8, device=device)
    _check(load().mkq_splitk_scratch_init(_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)),
           "mkq_splitk_scratch_init")
    return scratch


def mkq_linear_int4(a, s_x: float, Wq, s_w, bias, N: int, K: int, out_dtype: int = MKQ_F32, *,
                    a_is_codes: bool | None = None, act: int = MKQ_ACT_NONE, residual=None,
                    s_next: float = 0.0, want_q: bool = False, want_acc: bool = False,
                    out=None, workspace=None, stream=None, splitk_scratch=None,
                    config: int | None = None, k_slices: int = 0, w_stream: bool = False,
                    prefetch_stages: int = 0, q_pitch: int = 0, q_out=None):
    """The quantized linear.  ``a`` is packed codes (uint8 [M,K/2]) or float [M,K].

    Returns a dict with ``out`` (float tensor, or uint8 [M,N/2] for MKQ_I4) and
    optionally ``q`` (packed codes under s_next) and ``acc`` (int32 [M,N]).
    ``config`` / ``k_slices`` call mkq_tuning_linear_int4 (the kernel configuration chosen by the caller).
    ``w_stream``: Wq is in the streaming layout (mkq_linear_int4_stream; ``prefetch_stages`` / ``k_slices``
    call its tuning variant).  ``q_pitch``: codes per row of the code outputs (0 = N; the columns from N on are written
    as zero codes).  ``q_out``: the caller's buffer for the extra codes (implies ``want_q``).
    """
    torch = _torch()
    if a_is_codes is None:
        a_is_codes = a.dtype == torch.uint8
    M = a.size(0)
    a_dtype = MKQ_I4 if a_is_codes else _dtype_code(a)
    code_cols = (int(q_pitch) or N) // 2
    if out is None:
        out = (torch.empty((M, code_cols), dtype=torch.uint8, device=a.device) if out_dtype == MKQ_I4
               else torch.empty((M, N), dtype=_torch_dtype(out_dtype), device=a.device))
    q = q_out if q_out is not None else (torch.empty((M, code_cols), dtype=torch.uint8, device=a.device) if want_q else None)
    acc = torch.empty((M, N), dtype=torch.int32, device=a.device) if want_acc else None
    epi = None  # (what it says when nothing is asked for is what the library takes a null pointer for)
    if act or residual is not None or s_next or q is not None or want_acc or splitk_scratch is not None or q_pitch:
        epi = C.byref(Epilogue(
            act=int(act), residual=_ptr(residual), residual_dtype=_dtype_code(residual) if residual is not None else MKQ_F32,
            s_next=float(s_next), q_out=_ptr(q), acc_out=_ptr(acc), splitk_scratch=_ptr(splitk_scratch),
            splitk_scratch_bytes=splitk_scratch.nbytes if splitk_scratch is not None else 0, q_pitch=int(q_pitch)))
    if workspace is None and not a_is_codes:
        workspace = torch.empty(mkq_linear_int4_workspace_bytes(M, N, K, a_dtype), dtype=torch.uint8, device=a.device)
    ws_bytes = workspace.nbytes if workspace is not None else 0
    if w_stream:
        if not prefetch_stages and not k_slices:
            _check(load().mkq_linear_int4_stream(_ptr(a), a_dtype, float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias),
                                                 M, N, K, _ptr(out), int(out_dtype), epi, _ptr(workspace),
                                                 ws_bytes, _stream(stream)), "mkq_linear_int4_stream")
        else:
            _check(load().mkq_tuning_linear_int4_stream(_ptr(a), a_dtype, float(s_x), _ptr(Wq), _ptr(s_w),
                                                        _ptr(bias), M, N, K, _ptr(out), int(out_dtype),
                                                        epi, _ptr(workspace), ws_bytes, _stream(stream),
                                                        int(prefetch_stages), int(k_slices)),
                   "mkq_tuning_linear_int4_stream")
    elif config is None and not k_slices:
        _check(load().mkq_linear_int4(_ptr(a), a_dtype, float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias),
                                      M, N, K, _ptr(out), int(out_dtype), epi, _ptr(workspace),
                                      ws_bytes, _stream(stream)), "mkq_linear_int4")
    else:
        _check(load().mkq_tuning_linear_int4(_ptr(a), a_dtype, float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias),
                                             M, N, K, _ptr(out), int(out_dtype), epi, _ptr(workspace),
                                             ws_bytes, _stream(stream), -1 if config is None else int(config),
                                             int(k_slices)), "mkq_tuning_linear_int4")
    return {"out": out, "q": q, "acc": acc}


def mkq_linear_int4_stream(a, s_x, Wq_stream, s_w, bias, N, K, out_dtype=MKQ_F32, **kw):
    """mkq_linear_int4 on weights in the streaming layout (M <= 128)."""
    return mkq_linear_int4(a, s_x, Wq_stream, s_w, bias, N, K, out_dtype, w_stream=True, **kw)


def mkq_linear_int4_stream_static(a, s_x: float, Wq_stream, s_w, bias, N: int, K: int, out_dtype: int = MKQ_F32, *,
                                  act: int = MKQ_ACT_NONE, residual=None, s_next: float = 0.0, out=None,
                                  q_out=None, acc_out=None, stream=None):
    """mkq_linear_int4_stream on packed codes with the library's own scratch: nothing is allocated by the C
    call (outputs are the caller's: ``out`` and, optionally, ``q_out`` / ``acc_out`` must be passed in)."""
    M = a.shape[0]
    epi = Epilogue(act=int(act), residual=residual.data_ptr() if residual is not None else None,
                   residual_dtype=_dtype_code(residual) if residual is not None else MKQ_F32,
                   s_next=float(s_next), q_out=q_out.data_ptr() if q_out is not None else None,
                   acc_out=acc_out.data_ptr() if acc_out is not None else None,
                   splitk_scratch=None, splitk_scratch_bytes=0)
    _check(load().mkq_linear_int4_stream_static(_ptr(a), float(s_x), _ptr(Wq_stream), _ptr(s_w), _ptr(bias), M, N, K,
                                                _ptr(out), int(out_dtype), C.byref(epi), _stream(stream)),
           "mkq_linear_int4_stream_static")
    return out


def mkq_measure_stream(kind: int, src, dst, nbytes: int, stream=None):
    _check(load().mkq_measure_stream(int(kind), _ptr(src), _ptr(dst), int(nbytes), _stream(stream)), "mkq_measure_stream")


def mkq_measure_mfma_i8(operands, iters: int, sink, stream=None):
    """One launch of the register-only int8 MFMA loop; returns the integer operations it performs."""
    _check(load().mkq_measure_mfma_i8(_ptr(operands), operands.numel() * operands.element_size(), int(iters),
                                      _ptr(sink), _stream(stream)), "mkq_measure_mfma_i8")
    return int(load().mkq_measure_mfma_i8_ops(int(iters)))


def mkq_stream_weight_bytes(N: int, K: int) -> int:
    return int(load().mkq_stream_weight_bytes(N, K))


def mkq_repack_weights_int4_stream(Wq, N: int, K: int, out=None, stream=None):
    """Canonical packed weights -> the streaming layout (uint8 [mkq_stream_weight_bytes(N, K)])."""
    torch = _torch()
    if out is None:
        out = torch.empty(mkq_stream_weight_bytes(N, K), dtype=torch.uint8, device=Wq.device)
    _check(load().mkq_repack_weights_int4_stream(_ptr(Wq), N, K, _ptr(out), _stream(stream)),
           "mkq_repack_weights_int4_stream")
    return out


def mkq_quantize_int8(x, s_x: float, q_out=None, stream=None):
    """x [M,K] float32/float16 -> int8 codes [M,K] (8-bit range of the quantizer)."""
    torch = _torch()
    M, K = x.shape
    if q_out is None:
        q_out = torch.empty((M, K), dtype=torch.int8, device=x.device)
    _check(load().mkq_quantize_int8(_ptr(x), _dtype_code(x), M, K, x.stride(0), float(s_x), _ptr(q_out),
                                    _stream(stream)), "mkq_quantize_int8")
    return q_out


def mkq_pack_weights_int8(W, s_w_in=None, stream=None):
    """W [N,K] float32 -> (int8 codes [N,K], s_w float32 [N])."""
    torch = _torch()
    N, K = W.shape
    Wq = torch.empty((N, K), dtype=torch.int8, device=W.device)
    s_w = torch.empty(N, dtype=torch.float32, device=W.device)
    _check(load().mkq_pack_weights_int8(_ptr(W), N, K, _ptr(s_w_in), _ptr(s_w), _ptr(Wq),
                                        _stream(stream)), "mkq_pack_weights_int8")
    return Wq, s_w


def mkq_linear_int8(a, s_x: float, Wq, s_w, bias, out_dtype: int = MKQ_F32, *, act: int = MKQ_ACT_NONE,
                    residual=None, s_next: float = 0.0, want_acc: bool = False, out=None, stream=None,
                    config: int | None = None, q_pitch: int = 0):
    """The 8-bit linear: ``a`` int8 codes [M,K], ``Wq`` int8 codes [N,K].  ``config``: mkq_tuning_linear_int8.
    ``q_pitch``: codes per row of an int8 code output (0 = N; the padding columns are written as zeros)."""
    torch = _torch()
    M, K = a.shape
    N = Wq.shape[0]
    if out is None:
        cols = int(q_pitch) if (out_dtype == MKQ_I8 and q_pitch) else N
        out = torch.empty((M, cols), dtype=torch.int8 if out_dtype == MKQ_I8 else _torch_dtype(out_dtype),
                          device=a.device)
    acc = torch.empty((M, N), dtype=torch.int32, device=a.device) if want_acc else None
    epi = Epilogue(act=int(act), residual=residual.data_ptr() if residual is not None else None,
                   residual_dtype=_dtype_code(residual) if residual is not None else MKQ_F32,
                   s_next=float(s_next), q_out=None, acc_out=acc.data_ptr() if acc is not None else None,
                   q_pitch=int(q_pitch))
    if config is None:
        _check(load().mkq_linear_int8(_ptr(a), float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias), M, N, K, _ptr(out),
                                      int(out_dtype), C.byref(epi), _stream(stream)), "mkq_linear_int8")
    else:
        _check(load().mkq_tuning_linear_int8(_ptr(a), float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias), M, N, K, _ptr(out),
                                             int(out_dtype), C.byref(epi), _stream(stream), int(config)),
               "mkq_tuning_linear_int8")
    return {"out": out, "acc": acc}


def mkq_quantize_e3m2(x, s_x: float, stream=None):
    """x [M,K] float -> E3M2 containers uint8 [M, 3K/4] (experimental 6-bit float path)."""
    torch = _torch()
    M, K = x.shape
    q = torch.empty((M, K * 3 // 4), dtype=torch.uint8, device=x.device)
    _check(load().mkq_quantize_e3m2(_ptr(x), _dtype_code(x), M, K, x.stride(0), float(s_x), _ptr(q),
                                    _stream(stream)), "mkq_quantize_e3m2")
    return q


def mkq_pack_codes_e3m2(codes, stream=None):
    torch = _torch()
    rows, K = codes.shape
    q = torch.empty((rows, K * 3 // 4), dtype=torch.uint8, device=codes.device)
    _check(load().mkq_pack_codes_e3m2(_ptr(codes), rows, K, _ptr(q), _stream(stream)), "mkq_pack_codes_e3m2")
    return q


def mkq_pack_weights_e3m2(W, s_w_in=None, stream=None):
    torch = _torch()
    N, K = W.shape
    Wq = torch.empty((N, K * 3 // 4), dtype=torch.uint8, device=W.device)
    s_w = torch.empty(N, dtype=torch.float32, device=W.device)
    _check(load().mkq_pack_weights_e3m2(_ptr(W), N, K, _ptr(s_w_in), _ptr(s_w), _ptr(Wq), _stream(stream)),
           "mkq_pack_weights_e3m2")
    return Wq, s_w


def mkq_linear_int4_e3m2(a, s_x: float, Wq, s_w, bias, out_dtype: int = MKQ_F32, *, act: int = MKQ_ACT_NONE,
                         residual=None, s_next: float = 0.0, want_q: bool = False, want_acc: bool = False,
                         out=None, stream=None, config: int | None = None):
    """The 4-bit linear on E3M2 containers: a uint8 [M, 3K/4], Wq uint8 [N, 3K/4].
    ``config`` calls mkq_tuning_linear_int4_e3m2."""
    torch = _torch()
    M, K = a.shape[0], a.shape[1] * 4 // 3
    N = Wq.shape[0]
    dev = a.device
    if out is None:
        out = (torch.empty((M, N // 2), dtype=torch.uint8, device=dev) if out_dtype == MKQ_I4
               else torch.empty((M, N), dtype=_torch_dtype(out_dtype), device=dev))
    q = torch.empty((M, N // 2), dtype=torch.uint8, device=dev) if want_q else None
    acc = torch.empty((M, N), dtype=torch.int32, device=dev) if want_acc else None
    epi = Epilogue(act=int(act), residual=residual.data_ptr() if residual is not None else None,
                   residual_dtype=_dtype_code(residual) if residual is not None else MKQ_F32,
                   s_next=float(s_next), q_out=q.data_ptr() if q is not None else None,
                   acc_out=acc.data_ptr() if acc is not None else None)
    if config is None:
        _check(load().mkq_linear_int4_e3m2(_ptr(a), float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias), M, N, K, _ptr(out),
                                           int(out_dtype), C.byref(epi), _stream(stream)), "mkq_linear_int4_e3m2")
    else:
        _check(load().mkq_tuning_linear_int4_e3m2(_ptr(a), float(s_x), _ptr(Wq), _ptr(s_w), _ptr(bias), M, N, K,
                                                  _ptr(out), int(out_dtype), C.byref(epi), _stream(stream),
                                                  int(config)), "mkq_tuning_linear_int4_e3m2")
    return {"out": out, "q": q, "acc": acc}


def mkq_linear_fp16(a, W, bias, out_dtype: int = MKQ_F16, act: int = MKQ_ACT_NONE, residual=None,
                    out=None, stream=None):
    torch = _torch()
    M, K = a.shape
    N = W.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=_torch_dtype(out_dtype), device=a.device)
    _check(load().mkq_linear_fp16(_ptr(a), _ptr(W), _ptr(bias), M, N, K, _ptr(out), int(out_dtype),
                                  int(act), _ptr(residual), _stream(stream)), "mkq_linear_fp16")
    return out


def mkq_layernorm(x, gamma, beta, eps: float, s_next: float = 0.0, want_y: bool = True,
                  want_q: bool = False, stream=None):
    torch = _torch()
    M, D = x.shape
    y = torch.empty((M, D), dtype=torch.float16, device=x.device) if want_y else None
    q = torch.empty((M, D // 2), dtype=torch.uint8, device=x.device) if want_q else None
    _check(load().mkq_layernorm(_ptr(x), M, D, _ptr(gamma), _ptr(beta), float(eps), _ptr(y),
                                float(s_next), _ptr(q), _stream(stream)), "mkq_layernorm")
    return y, q


def mkq_attention(qkv, batch: int, seq: int, hidden: int, heads: int, s_next: float = 0.0,
                  want_ctx: bool = True, want_q: bool = False, stream=None):
    torch = _torch()
    M = batch * seq
    ctx = torch.empty((M, hidden), dtype=torch.float16, device=qkv.device) if want_ctx else None
    q = torch.empty((M, hidden // 2), dtype=torch.uint8, device=qkv.device) if want_q else None
    _check(load().mkq_attention(_ptr(qkv), batch, seq, hidden, heads, _ptr(ctx), float(s_next),
                                _ptr(q), _stream(stream)), "mkq_attention")
    return ctx, q


def mkq_layernorm_int8(x, gamma, beta, eps: float, s_next: float, want_y: bool = True, stream=None):
    torch = _torch()
    M, D = x.shape
    y = torch.empty((M, D), dtype=torch.float16, device=x.device) if want_y else None
    q = torch.empty((M, D), dtype=torch.int8, device=x.device)
    _check(load().mkq_layernorm_int8(_ptr(x), M, D, _ptr(gamma), _ptr(beta), float(eps), _ptr(y),
                                     float(s_next), _ptr(q), _stream(stream)), "mkq_layernorm_int8")
    return y, q


def mkq_attention_int8(qkv, batch: int, seq: int, hidden: int, heads: int, s_next: float,
                       want_ctx: bool = True, stream=None):
    torch = _torch()
    M = batch * seq
    ctx = torch.empty((M, hidden), dtype=torch.float16, device=qkv.device) if want_ctx else None
    q = torch.empty((M, hidden), dtype=torch.int8, device=qkv.device)
    _check(load().mkq_attention_int8(_ptr(qkv), batch, seq, hidden, heads, _ptr(ctx), float(s_next),
                                     _ptr(q), _stream(stream)), "mkq_attention_int8")
    return ctx, q


def mkq_attention_varlen(qkv, cu_seqlens, max_seq: int, hidden: int, heads: int, s_next: float = 0.0,
                         want_ctx: bool = True, q_bits: int = 0, stream=None):
    """Attention over a padding-free batch; cu_seqlens int32 device tensor [batch + 1]."""
    torch = _torch()
    total = qkv.shape[0]
    batch = cu_seqlens.numel() - 1
    ctx = torch.empty((total, hidden), dtype=torch.float16, device=qkv.device) if want_ctx else None
    q = None
    if q_bits == 4:
        q = torch.empty((total, hidden // 2), dtype=torch.uint8, device=qkv.device)
    elif q_bits == 8:
        q = torch.empty((total, hidden), dtype=torch.int8, device=qkv.device)
    _check(load().mkq_attention_varlen(_ptr(qkv), _ptr(cu_seqlens), batch, max_seq, hidden, heads, _ptr(ctx),
                                       float(s_next), _ptr(q), int(q_bits) if q_bits else 4, _stream(stream)),
           "mkq_attention_varlen")
    return ctx, q


# The two ends of an encoder and the training of its table.  These take tensors as programs have them, so what would be read
# wrongly is refused here: strides that the call cannot express, tensors of another device, sizes that do not agree.  Nothing is
# recorded by autograd, whatever requires a gradient: results have no graph, and what is written in place or into ``out`` keeps its
# version.  A training program joins lookup and gradient itself, in a torch.autograd.Function or a step of its own.

def _need(ok, what: str):
    if not ok:
        raise ValueError(what)


_FLOATS = "float32, float16 or bfloat16"


def _float_code(t, what: str) -> int:
    """_dtype_code of a tensor of floats."""
    _torch()
    code = _dtype_codes.get(t.dtype)
    if code is None:
        raise ValueError(f"{what}: {_FLOATS}")
    return code


def _float_dtype(code: int, what: str):
    """_torch_dtype of a code of floats."""
    if not _torch_dtypes:
        _torch_dtype(MKQ_F32)  # (fills the table)
    dtype = _torch_dtypes.get(code)
    if dtype is None:
        raise ValueError(f"{what}: {_FLOATS}")
    return dtype


def _rows(t, what: str):
    """Row stride of a matrix whose rows are contiguous."""
    if t.dim() == 2:
        rows, cols = t.shape
        ld, step = t.stride()
        if cols <= 1 or step == 1:
            return ld if rows > 1 else max(cols, 1)
    raise ValueError(f"{what}: a matrix with contiguous rows")


_current_device = None


def _same_device(*tensors) -> int:
    """The number of the current GPU, on which all tensors have to be.  (Numbers, -1 on the host: comparing device objects took 2 us
    of a call.)"""
    global _current_device
    if _current_device is None:
        torch = _torch()
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    dev = tensors[0].get_device()
    if dev < 0 or dev != _current_device():
        raise ValueError("tensors live on the current GPU")
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors live on one GPU")
    return dev


def _stream_on(dev: int, stream):
    """_stream where a tensor on the GPU has shown that it is set up."""
    if stream is None:
        try:
            return _torch_module._C._cuda_getCurrentRawStream(dev)
        except AttributeError:
            pass
    return _stream(stream)


def _workspace(workspace):
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace: contiguous")


def _new(shape, dtype, device, stream):
    """A tensor that belongs to the stream of the call, so that its memory is not handed on before the call is done."""
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _new_matrix(rows: int, cols: int, dtype, device, stream):
    if stream is None:  # (0.4 us less than empty)
        return _torch().empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)
    return _new((rows, cols), dtype, device, stream)


def mkq_group_weight_bytes(N: int, K: int) -> int:
    return int(load().mkq_group_weight_bytes(N, K))


def mkq_pack_weights_int4_group(W, group: int = 64, s_w_in=None, stream=None):
    """W [N,K] float32/float16/bfloat16 -> (Wq uint8 [N, ceil(K/32)*16], s_w float32 [N, ceil(K/group)])."""
    torch = _torch()
    ldw, w_dtype = _rows(W, "W"), _float_code(W, "W")
    N, K = W.shape
    dev = _same_device(W, s_w_in)
    groups = -(-K // group) if group > 0 else 0
    if s_w_in is not None:
        _need(s_w_in.dtype == torch.float32 and s_w_in.is_contiguous() and tuple(s_w_in.shape) == (N, groups),
              "s_w_in: contiguous float32 [N, ceil(K/group)]")
    Wq = _new((N, -(-K // 32) * 16), torch.uint8, W.device, stream)
    s_w = _new((N, groups), torch.float32, W.device, stream)
    _check(load().mkq_pack_weights_int4_group(_ptr(W), w_dtype, N, K, ldw, int(group), _ptr(s_w_in), _ptr(s_w),
                                              _ptr(Wq), _stream_on(dev, stream)), "mkq_pack_weights_int4_group")
    return Wq, s_w


def _group_table(Wq, s_w, N: int, K: int, group: int):
    torch = _torch()
    _need(Wq.dtype == torch.uint8 and Wq.is_contiguous() and Wq.numel() == N * (-(-K // 32) * 16),
          "Wq: contiguous uint8 [N, ceil(K/32)*16]")
    _need(s_w.dtype == torch.float32 and s_w.is_contiguous() and group > 0 and s_w.numel() == N * -(-K // group),
          "s_w: contiguous float32 [N, ceil(K/group)]")


def mkq_linear_int4_group(x, Wq, s_w, bias, N: int, K: int, group: int = 64, out_dtype: int | None = None, *,
                          act: int = MKQ_ACT_NONE, residual=None, out=None, stream=None):
    """x [M,K] float times group-scaled 4-bit weights (mkq_pack_weights_int4_group) -> [M,N] of out_dtype (None: x's)."""
    torch = _torch()
    ldx, x_dtype = _rows(x, "x"), _float_code(x, "x")
    M = x.size(0)
    _need(x.size(1) == K, "x: [M, K]")
    if out_dtype is None:
        out_dtype = x_dtype
    dtype = _float_dtype(out_dtype, "out_dtype")
    residual_dtype = _float_code(residual, "residual") if residual is not None else MKQ_F32
    dev = _same_device(x, Wq, s_w, bias, residual, out)
    _group_table(Wq, s_w, N, K, group)
    _need(bias is None or (bias.dtype == torch.float32 and bias.is_contiguous() and bias.numel() == N), "bias: float32 [N]")
    if out is None:
        out = _new_matrix(M, N, dtype, x.device, stream)
    else:
        _need(out.dtype == dtype and out.is_contiguous() and tuple(out.shape) == (M, N), "out: contiguous [M, N] of out_dtype")
    epi = None
    if act or residual is not None:
        _need(residual is None or (residual.is_contiguous() and tuple(residual.shape) == (M, N)), "residual: contiguous [M, N]")
        epi = C.byref(Epilogue(act=int(act), residual=_ptr(residual), residual_dtype=residual_dtype))
    _check(load().mkq_linear_int4_group(_ptr(x), x_dtype, ldx, _ptr(Wq), _ptr(s_w), int(group), _ptr(bias), M, N, K,
                                        _ptr(out), int(out_dtype), epi, _stream_on(dev, stream)), "mkq_linear_int4_group")
    return out


def _tokens(tokens):
    torch = _torch()
    _need(tokens.dtype in (torch.int32, torch.int64) and tokens.is_contiguous(), "tokens: contiguous int32 or int64")
    return 64 if tokens.dtype == torch.int64 else 32


def _token_rows(tokens, D: int, out, dtype, stream):
    """The caller's [M, D] rows, or new ones, and their stride."""
    M = tokens.numel()
    if out is None:
        return _new_matrix(M, D, dtype, tokens.device, stream), D
    ld = _rows(out, "out")
    _need(out.dtype == dtype and tuple(out.shape) == (M, D), "out: [M, D] of out_dtype")
    return out, ld


def mkq_embedding(tokens, table, scale: float = 1.0, out_dtype: int | None = None, *, out=None, stream=None):
    """Rows of table [V,D] for tokens (int32 / int64, any shape, M of them) times scale -> [M,D] of out_dtype (None: the table's).
    Autograd does not see it: the table's gradient is mkq_embedding_gradient."""
    bits = _tokens(tokens)
    ld_table, table_dtype = _rows(table, "table"), _float_code(table, "table")
    V, D = table.shape
    if out_dtype is None:
        out_dtype = table_dtype
    dtype = _float_dtype(out_dtype, "out_dtype")
    dev = _same_device(tokens, table, out)
    out, ld_out = _token_rows(tokens, D, out, dtype, stream)
    _check(load().mkq_embedding(_ptr(tokens), bits, tokens.numel(), _ptr(table), table_dtype, V, D, ld_table, float(scale),
                                _ptr(out), int(out_dtype), ld_out, _stream_on(dev, stream)), "mkq_embedding")
    return out


def mkq_embedding_int4_group(tokens, Wq, s_w, V: int, D: int, group: int = 64, scale: float = 1.0, out_dtype: int = MKQ_F32, *,
                             out=None, stream=None):
    """Rows of a group-scaled 4-bit table (mkq_pack_weights_int4_group with N = V, K = D) times scale -> [M,D] of out_dtype."""
    bits, dtype = _tokens(tokens), _float_dtype(out_dtype, "out_dtype")
    dev = _same_device(tokens, Wq, s_w, out)
    _group_table(Wq, s_w, V, D, group)
    out, ld_out = _token_rows(tokens, D, out, dtype, stream)
    _check(load().mkq_embedding_int4_group(_ptr(tokens), bits, tokens.numel(), _ptr(Wq), _ptr(s_w), int(group), V, D, float(scale),
                                           _ptr(out), int(out_dtype), ld_out, _stream_on(dev, stream)), "mkq_embedding_int4_group")
    return out


def mkq_embedding_gradient_workspace_bytes(M: int, D: int) -> int:
    return int(load().mkq_embedding_gradient_workspace_bytes(M, D))


def mkq_embedding_gradient(tokens, dy, V: int, scale: float = 1.0, grad_dtype: int = MKQ_F32, *, padding_token: int = -1,
                           grad=None, accumulate: bool = False, workspace=None, stream=None):
    """Gradient [V,D] of mkq_embedding's table from dy [M,D] (outside autograd).  ``accumulate``: added to the ``grad`` that is
    passed in."""
    torch = _torch()
    bits = _tokens(tokens)
    ld_dy, dy_dtype, dtype = _rows(dy, "dy"), _float_code(dy, "dy"), _float_dtype(grad_dtype, "grad_dtype")
    M, D = dy.shape
    _need(tokens.numel() == M, "dy: a row for every token")
    _workspace(workspace)
    dev = _same_device(tokens, dy, grad, workspace)
    _need(grad is not None or not accumulate, "accumulate: needs the gradient to add to")
    if grad is None:
        grad, ld_grad = _new_matrix(V, D, dtype, dy.device, stream), D
    else:
        ld_grad = _rows(grad, "grad")
        _need(grad.dtype == dtype and tuple(grad.shape) == (V, D), "grad: [V, D] of grad_dtype")
    if workspace is None:
        workspace = _new(mkq_embedding_gradient_workspace_bytes(M, D), torch.uint8, dy.device, stream)
    _check(load().mkq_embedding_gradient(_ptr(tokens), bits, M, _ptr(dy), dy_dtype, ld_dy, V, D, float(scale), int(padding_token),
                                         int(accumulate), _ptr(grad), int(grad_dtype), ld_grad, _ptr(workspace), workspace.nbytes,
                                         _stream_on(dev, stream)), "mkq_embedding_gradient")
    return grad


def mkq_gradient_norm_workspace_bytes(n: int) -> int:
    return int(load().mkq_gradient_norm_workspace_bytes(n))


def _float_codes(dtypes, what: str):
    """_dtype_code of every tensor of a list."""
    _torch()
    try:
        return array("i", map(_dtype_codes.__getitem__, dtypes))
    except KeyError:
        raise ValueError(f"{what}: {_FLOATS}") from None


def _tensor_list(tensors, what: str):
    """Numbers of values and addresses of contiguous tensors of the current GPU.  (One pass a question, in C: a loop over fifty
    tensors and their outputs took 50 us of a call.)"""
    torch = _torch()
    T = torch.Tensor
    if not tensors or not all(map(T.is_contiguous, tensors)):
        raise ValueError(f"{what}: contiguous tensors, one at least")
    _same_device(tensors[0])
    if len(set(map(T.get_device, tensors))) != 1:
        raise ValueError("tensors live on one GPU")
    return list(map(T.numel, tensors)), array("Q", map(T.data_ptr, tensors))


def _norm_buffers(n: int, device, norm_out, workspace, stream):
    torch = _torch()
    if norm_out is None:
        norm_out = _new(1, torch.float32, device, stream)
    _need(norm_out.dtype == torch.float32 and norm_out.numel() == 1, "norm_out: float32 [1]")
    if workspace is None:
        workspace = _new(mkq_gradient_norm_workspace_bytes(n), torch.uint8, device, stream)
    return norm_out, workspace


def mkq_gradient_norm(grads, norm_out=None, workspace=None, stream=None):
    """Norm over all values of a list of contiguous tensors (float32 / float16 / bfloat16, mixed) -> float32 tensor [1]."""
    grads = list(grads)
    _workspace(workspace)
    codes = _float_codes([t.dtype for t in grads], "grads")
    counts, at = _tensor_list(grads, "grads")
    dev = _same_device(grads[0], norm_out, workspace)
    norm_out, workspace = _norm_buffers(len(grads), grads[0].device, norm_out, workspace, stream)
    counts = array("q", counts)
    _check(load().mkq_gradient_norm(len(grads), at.buffer_info()[0], counts.buffer_info()[0], codes.buffer_info()[0], _ptr(norm_out),
                                    _ptr(workspace), workspace.nbytes, _stream_on(dev, stream)), "mkq_gradient_norm")
    return norm_out


def mkq_clip_gradients(grads, max_norm: float, *, outs=None, norm_out=None, workspace=None, stream=None):
    """Scales a list of gradients (float32 / float16 / bfloat16, mixed; the float64 sums of mkq_scale_gradients are to be cast) to a
    norm of at most max_norm, in place or into ``outs`` (same types and sizes); returns the norm before, float32 tensor [1]."""
    grads = list(grads)
    _workspace(workspace)
    dtypes = [t.dtype for t in grads]
    codes = _float_codes(dtypes, "grads")
    counts, at = _tensor_list(grads, "grads")
    dev = _same_device(grads[0], norm_out, workspace)
    out_at = at
    if outs is not None:
        outs = list(outs)
        out_counts, out_at = _tensor_list(outs, "outs")
        _same_device(grads[0], outs[0])
        _need(out_counts == counts and [t.dtype for t in outs] == dtypes, "outs: the gradients' types and sizes")
    norm_out, workspace = _norm_buffers(len(grads), grads[0].device, norm_out, workspace, stream)
    counts = array("q", counts)
    status = load().mkq_clip_gradients(len(grads), at.buffer_info()[0], out_at.buffer_info()[0], counts.buffer_info()[0],
                                       codes.buffer_info()[0], float(max_norm), _ptr(norm_out), _ptr(workspace), workspace.nbytes,
                                       _stream_on(dev, stream))
    if status == MKQ_ERR_UNSUPPORTED:
        raise ValueError("no result over another one or over another gradient: it would be scaled twice")
    _check(status, "mkq_clip_gradients")
    return norm_out


class TokenLogProbs:
    """What mkq_token_log_probs gives: float32 ``log_probs`` [M], ``entropies`` [M], ``normalizers`` [M,2] (largest score, logarithm of the sum
    of the exponentials relative to it), ``top_tokens`` int32 [M,top] with ``top_log_probs``."""
    __slots__ = ("log_probs", "entropies", "normalizers", "top_tokens", "top_log_probs")


@lru_cache(maxsize=4096)  # (they go by sizes alone, and the smallest calls are bound by their own calls)
def mkq_token_log_probs_workspace_bytes(M: int, V: int, top: int = 0) -> int:
    return int(load().mkq_token_log_probs_workspace_bytes(M, V, top))


def _vector(t, n: int, what: str):
    """A contiguous float32 vector of n values."""
    _need(t.dtype == _torch().float32 and t.is_contiguous() and t.numel() == n, f"{what}: contiguous float32 [{n}]")


def mkq_token_log_probs(logits, tokens, scale: float = 1.0, top: int = 0, *, workspace=None, stream=None) -> TokenLogProbs:
    """Log probabilities of tokens [M] (int32 / int64; outside the vocabulary: 0) under scale * logits [M,V], entropies, and the ``top`` most
    probable tokens of every row."""
    torch = _torch()
    ld, dtype, bits = _rows(logits, "logits"), _float_code(logits, "logits"), _tokens(tokens)
    M, V = logits.shape
    top = int(top)
    _need(tokens.numel() == M, "tokens: one for every row")
    _need(0 <= top <= V, "top: at most the vocabulary")
    _workspace(workspace)
    dev = _same_device(logits, tokens, workspace)
    r, device = TokenLogProbs(), logits.device
    r.log_probs, r.entropies = _new(M, torch.float32, device, stream), _new(M, torch.float32, device, stream)
    r.normalizers = _new((M, 2), torch.float32, device, stream)
    r.top_tokens, r.top_log_probs = _new((M, top), torch.int32, device, stream), _new((M, top), torch.float32, device, stream)
    if workspace is None:
        need = mkq_token_log_probs_workspace_bytes(M, V, top)
        workspace = _new(need, torch.uint8, device, stream) if need else None
    _check(load().mkq_token_log_probs(_ptr(logits), dtype, ld, M, V, float(scale), _ptr(tokens), bits, _ptr(r.normalizers), _ptr(r.log_probs),
                                      _ptr(r.entropies), top, _ptr(r.top_tokens), _ptr(r.top_log_probs), _ptr(workspace),
                                      0 if workspace is None else workspace.nbytes, _stream_on(dev, stream)), "mkq_token_log_probs")
    return r


def mkq_token_log_probs_gradient(logits, tokens, result: TokenLogProbs, d_log_probs, scale: float = 1.0, grad_dtype: int | None = None, *,
                                 d_entropies=None, grad=None, stream=None):
    """Gradient [M,V] of grad_dtype (None: the logits') of what mkq_token_log_probs gave for the same logits, tokens and scale, from the
    gradients of its log probabilities and, optionally, entropies.  ``grad``: where it goes, the logits themselves too."""
    ld, dtype, bits = _rows(logits, "logits"), _float_code(logits, "logits"), _tokens(tokens)
    M, V = logits.shape
    _need(tokens.numel() == M, "tokens: one for every row")
    normalizers, entropies = result.normalizers, result.entropies
    _vector(normalizers, 2 * M, "normalizers")
    _vector(entropies, M, "entropies")
    _vector(d_log_probs, M, "d_log_probs")
    if d_entropies is not None:
        _vector(d_entropies, M, "d_entropies")
    if grad_dtype is None:
        grad_dtype = dtype
    to = _float_dtype(grad_dtype, "grad_dtype")
    dev = _same_device(logits, tokens, normalizers, entropies, d_log_probs, d_entropies, grad)
    if grad is None:
        grad, ld_grad = _new_matrix(M, V, to, logits.device, stream), V
    else:
        ld_grad = _rows(grad, "grad")
        _need(grad.dtype == to and tuple(grad.shape) == (M, V), "grad: [M, V] of grad_dtype")
    _check(load().mkq_token_log_probs_gradient(_ptr(logits), dtype, ld, M, V, float(scale), _ptr(tokens), bits, _ptr(normalizers),
                                               _ptr(entropies), _ptr(d_log_probs), _ptr(d_entropies), _ptr(grad), int(grad_dtype),
                                               ld_grad, _stream_on(dev, stream)), "mkq_token_log_probs_gradient")
    return grad


def mkq_checkpoint_int8(x, group: int = 128, *, stream=None):
    """x [M,K] float32/float16/bfloat16 kept in 8 bits -> (codes int8 [M, ceil(K/32)*32], steps float32 [M, ceil(K/group)])."""
    torch = _torch()
    ldx, dtype = _rows(x, "x"), _float_code(x, "x")
    M, K = x.shape
    _need(group in (32, 64, 128), "group: 32, 64 or 128")
    dev = _same_device(x)
    codes = _new_matrix(M, -(-K // 32) * 32, torch.int8, x.device, stream)
    steps = _new_matrix(M, -(-K // group), torch.float32, x.device, stream)
    _check(load().mkq_checkpoint_int8(_ptr(x), dtype, M, K, ldx, group, _ptr(codes), _ptr(steps), _stream_on(dev, stream)),
           "mkq_checkpoint_int8")
    return codes, steps


def _checkpoint(codes, steps, K: int, group: int, what: str = "codes") -> int:
    """Rows of a checkpoint of K columns."""
    torch = _torch()
    _need(group in (32, 64, 128), "group: 32, 64 or 128")
    _need(codes.dtype == torch.int8 and codes.is_contiguous() and codes.dim() == 2 and codes.size(1) == -(-K // 32) * 32,
          f"{what}: contiguous int8 [M, ceil(K/32)*32]")
    M = codes.size(0)
    _need(steps.dtype == torch.float32 and steps.is_contiguous() and tuple(steps.shape) == (M, -(-K // group)),
          "steps: contiguous float32 [M, ceil(K/group)]")
    return M


def _out_rows(out, M: int, K: int, dtype, device, stream, what: str):
    """The caller's [M, K] rows, or new ones, and their stride."""
    if out is None:
        return _new_matrix(M, K, dtype, device, stream), K
    ld = _rows(out, what)
    _need(out.dtype == dtype and tuple(out.shape) == (M, K), f"{what}: [{M}, {K}] of its type")
    return out, ld


def mkq_checkpoint_restore(codes, steps, K: int, group: int = 128, out_dtype: int = MKQ_F32, *, act: int = MKQ_ACT_NONE, out=None,
                           stream=None):
    """The [M,K] activations of mkq_checkpoint_int8 again, or their GELU."""
    M, dtype = _checkpoint(codes, steps, K, group), _float_dtype(out_dtype, "out_dtype")
    dev = _same_device(codes, steps, out)
    out, ld_out = _out_rows(out, M, K, dtype, codes.device, stream, "out")
    _check(load().mkq_checkpoint_restore(_ptr(codes), _ptr(steps), group, M, K, int(act), _ptr(out), int(out_dtype), ld_out,
                                         _stream_on(dev, stream)), "mkq_checkpoint_restore")
    return out


def mkq_checkpoint_gelu_gradient(codes, steps, dy, group: int = 128, dx_dtype: int | None = None, *, dx=None, stream=None):
    """dy [M,K] times the GELU's derivative at the activations that mkq_checkpoint_int8 kept -> [M,K] of dx_dtype (None: dy's).  ``dx``: where it
    goes, dy itself too."""
    ld_dy, dy_dtype = _rows(dy, "dy"), _float_code(dy, "dy")
    M, K = dy.shape
    _need(_checkpoint(codes, steps, K, group) == M, "dy: a row for every row kept")
    if dx_dtype is None:
        dx_dtype = dy_dtype
    dtype = _float_dtype(dx_dtype, "dx_dtype")
    dev = _same_device(codes, steps, dy, dx)
    dx, ld_dx = _out_rows(dx, M, K, dtype, dy.device, stream, "dx")
    _check(load().mkq_checkpoint_gelu_gradient(_ptr(codes), _ptr(steps), group, M, K, _ptr(dy), dy_dtype, ld_dy, _ptr(dx), int(dx_dtype),
                                               ld_dx, _stream_on(dev, stream)), "mkq_checkpoint_gelu_gradient")
    return dx


@lru_cache(maxsize=4096)
def mkq_low_rank_adapters_workspace_bytes(M: int, K: int, N: int, rank: int, R: int) -> int:
    return int(load().mkq_low_rank_adapters_workspace_bytes(M, K, N, rank, R))


@lru_cache(maxsize=4096)
def mkq_low_rank_adapters_gradient_workspace_bytes(M: int, K: int, N: int, rank: int, R: int) -> int:
    return int(load().mkq_low_rank_adapters_gradient_workspace_bytes(M, K, N, rank, R))


def _adapters(adapter, down, up, scales, M: int):
    """R, rank, K, N and the type of the adapters' matrices."""
    torch = _torch()
    w_dtype = _float_code(down, "down")
    _need(adapter.dtype == torch.int32 and adapter.is_contiguous() and adapter.numel() == M, "adapter: contiguous int32, one for every row")
    _need(down.dim() == 3 and up.dim() == 3 and down.is_contiguous() and up.is_contiguous() and up.dtype == down.dtype
          and down.shape[:2] == up.shape[:2], "down, up: contiguous [R, rank, K] and [R, rank, N] of one type")
    R, rank, K = down.shape
    if scales is not None:
        _vector(scales, R, "scales")
    return R, rank, K, up.size(2), w_dtype


def mkq_low_rank_adapters(x, adapter, down, up, scales=None, out_dtype: int | None = None, *, base=None, out=None, hidden=None, workspace=None,
                          stream=None):
    """base + scales[a] * (x down_a^T) up_a for every row's adapter a (int32 [M]; outside: none) -> [M,N] of out_dtype (None: x's).  down [R,rank,K],
    up [R,rank,N]; ``base`` [M,N] of out_dtype, ``out`` too if need be, but never x; ``hidden`` float32 [M,rank]: x down_a^T for the gradient."""
    torch = _torch()
    ldx, x_dtype = _rows(x, "x"), _float_code(x, "x")
    M = x.size(0)
    R, rank, K, N, w_dtype = _adapters(adapter, down, up, scales, M)
    _need(x.size(1) == K, "x: [M, K]")
    if out_dtype is None:
        out_dtype = x_dtype
    dtype = _float_dtype(out_dtype, "out_dtype")
    _workspace(workspace)
    dev = _same_device(x, adapter, down, up, scales, base, out, hidden, workspace)
    ld_base = 0
    if base is not None:
        ld_base = _rows(base, "base")
        _need(base.dtype == dtype and tuple(base.shape) == (M, N), "base: [M, N] of out_dtype")
    if hidden is not None:
        _vector(hidden, M * rank, "hidden")
    out, ld_out = _out_rows(out, M, N, dtype, x.device, stream, "out")
    if workspace is None:
        need = mkq_low_rank_adapters_workspace_bytes(M, K, N, rank, R)
        workspace = _new(need, torch.uint8, x.device, stream) if need else None
    _check(load().mkq_low_rank_adapters(_ptr(x), x_dtype, ldx, _ptr(adapter), M, K, N, rank, R, _ptr(down), _ptr(up), w_dtype, _ptr(scales),
                                        _ptr(base), ld_base, _ptr(out), int(out_dtype), ld_out, _ptr(hidden), _ptr(workspace),
                                        0 if workspace is None else workspace.nbytes, _stream_on(dev, stream)), "mkq_low_rank_adapters")
    return out


def mkq_low_rank_adapters_gradient(dy, x, adapter, hidden, down, up, scales=None, dx_dtype: int | None = None, grad_dtype: int = MKQ_F32, *,
                                   steps=None, group: int = 0, base=None, dx=None, d_down=None, d_up=None, accumulate: bool = False,
                                   want_dx: bool = True, workspace=None, stream=None):
    """Gradients (dx [M,K] of dx_dtype (None: dy's), d_down [R,rank,K], d_up [R,rank,N] of grad_dtype) of mkq_low_rank_adapters from dy [M,N], its x and
    the ``hidden`` that it gave.  ``steps``, ``group``: x is the codes of mkq_checkpoint_int8.  ``base`` is added to dx; ``accumulate``: added to the
    ``d_down`` and ``d_up`` that are passed in; ``want_dx`` False: none."""
    torch = _torch()
    ld_dy, dy_dtype = _rows(dy, "dy"), _float_code(dy, "dy")
    M = dy.size(0)
    R, rank, K, N, w_dtype = _adapters(adapter, down, up, scales, M)
    _need(dy.size(1) == N, "dy: [M, N]")
    _vector(hidden, M * rank, "hidden")
    if steps is not None:
        _need(_checkpoint(x, steps, K, group, "x") == M, "x: a row for every row of dy")
        x_dtype, ldx = MKQ_I8, x.size(1)
    else:
        x_dtype, ldx = _float_code(x, "x"), _rows(x, "x")
        _need(tuple(x.shape) == (M, K), "x: [M, K]")
    if dx_dtype is None:
        dx_dtype = dy_dtype
    dtype, grad = _float_dtype(dx_dtype, "dx_dtype"), _float_dtype(grad_dtype, "grad_dtype")
    _workspace(workspace)
    dev = _same_device(dy, x, adapter, hidden, down, up, scales, steps, base, dx, d_down, d_up, workspace)
    ld_base = ld_dx = 0
    _need(want_dx or (dx is None and base is None), "dx: wanted")
    if want_dx:
        if base is not None:
            ld_base = _rows(base, "base")
            _need(base.dtype == dtype and tuple(base.shape) == (M, K), "base: [M, K] of dx_dtype")
        dx, ld_dx = _out_rows(dx, M, K, dtype, dy.device, stream, "dx")
    _need(not accumulate or (d_down is not None and d_up is not None), "accumulate: needs the gradients to add to")
    if d_down is None:
        d_down = _new((R, rank, K), grad, dy.device, stream)
    if d_up is None:
        d_up = _new((R, rank, N), grad, dy.device, stream)
    _need(d_down.dtype == d_up.dtype == grad and d_down.is_contiguous() and d_up.is_contiguous() and d_down.shape == down.shape
          and d_up.shape == up.shape, "d_down, d_up: contiguous, of the adapters' sizes and grad_dtype")
    if workspace is None:
        workspace = _new(mkq_low_rank_adapters_gradient_workspace_bytes(M, K, N, rank, R), torch.uint8, dy.device, stream)
    _check(load().mkq_low_rank_adapters_gradient(_ptr(dy), dy_dtype, ld_dy, _ptr(x), x_dtype, ldx, _ptr(steps), int(group), _ptr(adapter),
                                                 _ptr(hidden), M, K, N, rank, R, _ptr(down), _ptr(up), w_dtype, _ptr(scales), _ptr(base), ld_base,
                                                 _ptr(dx), int(dx_dtype), ld_dx, _ptr(d_down), _ptr(d_up), int(grad_dtype), int(accumulate),
                                                 _ptr(workspace), workspace.nbytes, _stream_on(dev, stream)),
           "mkq_low_rank_adapters_gradient")
    return dx, d_down, d_up


class BertLayerInt4:
    """Holds the device tensors of one W4A4 encoder layer and its parameter struct."""
    _workspace_fn = "mkq_bert_layer_workspace"
    _run_fn = "mkq_bert_layer_int4"

    def __init__(self, batch, seq, hidden, heads, ffn, packed: dict, sx: dict, ln: dict, ln_eps: float,
                 s_out_next: float = 0.0, next_bits: int = 0, cu_seqlens=None, total_tokens: int = 0):
        self._keep = (packed, ln, cu_seqlens)
        p = BertLayerParams()
        p.next_bits = int(next_bits)
        if cu_seqlens is not None:  # padding-free batch: seq is the upper bound of the lengths
            p.cu_seqlens, p.total_tokens = cu_seqlens.data_ptr(), int(total_tokens)
        p.batch, p.seq, p.hidden, p.heads, p.ffn = batch, seq, hidden, heads, ffn
        for nm in ("qkv", "ao", "up", "down"):
            Wq, s_w, b = packed[nm]
            setattr(p, "Wq_" + nm, Wq.data_ptr())
            setattr(p, "sw_" + nm, s_w.data_ptr())
            setattr(p, "b_" + nm, b.data_ptr())
            setattr(p, "sx_" + nm, float(sx[nm]))
        for nm in ("ln1_gamma", "ln1_beta", "ln2_gamma", "ln2_beta"):
            setattr(p, nm, ln[nm].data_ptr())
        p.ln_eps = float(ln_eps)
        p.s_out_next = float(s_out_next)
        self.params = p
        self.layout = BertLayerWorkspaceLayout()
        _check(getattr(load(), self._workspace_fn)(C.byref(p), C.byref(self.layout)), self._workspace_fn)
        self.M, self.hidden, self.ffn = (int(total_tokens) if cu_seqlens is not None else batch * seq), hidden, ffn

    def workspace_bytes(self) -> int:
        return int(self.layout.total)

    def __call__(self, h_in, workspace, h_out=None, q_in=None, q_out_next=None, stream=None):
        torch = _torch()
        if h_out is None:
            h_out = torch.empty((self.M, self.hidden), dtype=torch.float16, device=h_in.device)
        _check(getattr(load(), self._run_fn)(C.byref(self.params), _ptr(h_in), _dtype_code(h_in), _ptr(q_in),
                                             _ptr(h_out), _ptr(q_out_next), _ptr(workspace),
                                             workspace.numel() * workspace.element_size(), _stream(stream)),
               self._run_fn)
        return h_out


class BertLayerInt8(BertLayerInt4):
    """The same layer W8A8: ``packed`` holds int8 weights from mkq_pack_weights_int8, code buffers are int8."""
    _workspace_fn = "mkq_bert_layer_int8_workspace"
    _run_fn = "mkq_bert_layer_int8"


class BertLayerFp16:
    """The 16-bit float baseline layer."""

    def __init__(self, batch, seq, hidden, heads, ffn, weights: dict, ln: dict, ln_eps: float, cu_seqlens=None,
                 total_tokens: int = 0):
        self._keep = (weights, ln, cu_seqlens)
        p = BertLayerParamsFp16()
        if cu_seqlens is not None:
            p.cu_seqlens, p.total_tokens = cu_seqlens.data_ptr(), int(total_tokens)
        p.batch, p.seq, p.hidden, p.heads, p.ffn = batch, seq, hidden, heads, ffn
        for nm in ("qkv", "ao", "up", "down"):
            W, b = weights[nm]
            setattr(p, "W_" + nm, W.data_ptr())
            setattr(p, "b_" + nm, b.data_ptr())
        for nm in ("ln1_gamma", "ln1_beta", "ln2_gamma", "ln2_beta"):
            setattr(p, nm, ln[nm].data_ptr())
        p.ln_eps = float(ln_eps)
        self.params = p
        self.M, self.hidden = (int(total_tokens) if cu_seqlens is not None else batch * seq), hidden

    def workspace_bytes(self) -> int:
        return int(load().mkq_bert_layer_fp16_workspace_bytes(C.byref(self.params)))

    def __call__(self, h_in, workspace, h_out=None, stream=None):
        torch = _torch()
        if h_out is None:
            h_out = torch.empty((self.M, self.hidden), dtype=torch.float16, device=h_in.device)
        _check(load().mkq_bert_layer_fp16(C.byref(self.params), _ptr(h_in), _ptr(h_out), _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)),
               "mkq_bert_layer_fp16")
        return h_out
