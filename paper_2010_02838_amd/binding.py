"""Thin ctypes binding of libcodistill.so: argument marshalling only.

Every step of the training step runs in the library's HIP kernels; PyTorch is
used here for device memory (tensors) and the current stream, nothing else.
There is no fallback: if the shared library is missing, importing this module
raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcodistill.so")

CD_OK, CD_ERR_INVALID_ARG, CD_ERR_UNSUPPORTED, CD_ERR_WORKSPACE_TOO_SMALL, CD_ERR_HIP = 0, -1, -2, -3, -4
CD_F32, CD_BF16 = 0, 1
CD_DIST_MSE_LOGITS, CD_DIST_KL, CD_DIST_MSE_CENTERED = 0, 1, 2
CD_MEAN_ALL, CD_MEAN_ROWS = 0, 1
CD_BN_BATCH_STATS, CD_BN_RUNNING = 0, 1
CD_STREAMS_TWO, CD_STREAMS_AUTO = 0, 1
CD_ARCH_TINY_CNN, CD_ARCH_RESNET_BASIC, CD_ARCH_RESNET_BOTTLENECK, CD_ARCH_TRANSFORMER_HEAD = 0, 1, 2, 3
CD_ARCH_TRANSFORMER = 4
CD_ARCH_RESNET_BASIC_IMAGENET = 5
CD_ARCH_RESNEXT = 6
CD_ARCH_WIDE_RESNET_SPLIT = 7
CD_MAX_STAGES, CD_NAME_LEN, CD_LOSS_MAX_PEERS = 4, 48, 8
CD_ROPE_HALVES, CD_ROPE_PAIRS = 0, 1
CD_ROPE_MAX_PAIRS, CD_ROPE_MAX_TENSORS = 128, 4
CD_LAMBDA_HEAD, CD_LAMBDA_TOKEN = 0, 1
HEAD_NORM_MAX_WIDTH = 1024
ADAMW_BLOCK = 256   # elements that share an exponent in 8-bit moments
KERNEL_CLASSES = ["conv_fprop", "conv_dgrad", "conv_wgrad", "norm", "glue", "linear", "loss", "sgd", "conv_fprop_narrow",
                  "bn_apply", "conv_fprop_wide", "attention"]
PARAM_KINDS = ["conv_w", "bias", "bn_gamma", "bn_beta", "linear_w", "embed_w"]


class ArchDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("classes", ctypes.c_int32), ("in_h", ctypes.c_int32),
                ("in_w", ctypes.c_int32), ("n_stages", ctypes.c_int32),
                ("widths", ctypes.c_int32 * CD_MAX_STAGES), ("blocks", ctypes.c_int32 * CD_MAX_STAGES),
                ("stem_width", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("out_widths", ctypes.c_int32 * CD_MAX_STAGES), ("n_splits", ctypes.c_int32), ("split", ctypes.c_int32),
                ("max_sentences", ctypes.c_int32), ("max_sentence_len", ctypes.c_int32)]


class TensorInfo(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * CD_NAME_LEN), ("kind", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 4), ("offset", ctypes.c_int64), ("size", ctypes.c_int64),
                ("fan_in", ctypes.c_int64), ("frozen", ctypes.c_int32)]


class OpInfo(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("x", ctypes.c_int32), ("y", ctypes.c_int32), ("res", ctypes.c_int32),
                ("relu", ctypes.c_int32), ("param_w", ctypes.c_int32), ("param_b", ctypes.c_int32),
                ("k", ctypes.c_int32), ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("stats_offset", ctypes.c_int64), ("res_grad", ctypes.c_int32), ("k_col", ctypes.c_int32), ("v_col", ctypes.c_int32),
                ("fused_pool", ctypes.c_int32), ("key_tok0", ctypes.c_int32)]


class ActInfo(ctypes.Structure):
    _fields_ = [("h", ctypes.c_int32), ("w", ctypes.c_int32), ("c", ctypes.c_int32), ("is_f32", ctypes.c_int32),
                ("act_offset", ctypes.c_int64), ("grad_offset", ctypes.c_int64)]


class LossCfg(ctypes.Structure):
    _fields_ = [("alpha", ctypes.c_float), ("label_smoothing", ctypes.c_float), ("dist_kind", ctypes.c_int32),
                ("mse_reduction", ctypes.c_int32), ("ignore_index", ctypes.c_int32), ("n_peers", ctypes.c_int32),
                ("temperature", ctypes.c_float)]


class Rotary(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("dim", ctypes.c_int32), ("n_pairs", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("axis", ctypes.c_int32 * CD_ROPE_MAX_PAIRS), ("freq", ctypes.c_double * CD_ROPE_MAX_PAIRS)]


class RotaryTensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("heads", ctypes.c_int64), ("x_token", ctypes.c_int64),
                ("y_token", ctypes.c_int64)]


class DiffAttn(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "batch", "tq", "tk", "heads", "kv_heads", "head_dim", "causal", "lambda_kind")] + [
        ("scale", ctypes.c_float)] + [(n, ctypes.c_int64) for n in (
            "q_token", "q_batch", "k_token", "k_batch", "v_token", "v_batch", "o_token", "o_batch")] + [
        (n, ctypes.c_void_p) for n in ("q_lens", "k_lens", "q_starts", "k_starts")] + [("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64)]


class AdamwTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w", "grad", "lowp", "m", "v", "exps", "m_out", "v_out")] + [
        ("n", ctypes.c_int64), ("weight_decay", ctypes.c_float), ("lr_scale", ctypes.c_float)]


class AdamwPlan(ctypes.Structure):
    _fields_ = [("tensors", ctypes.c_int64), ("elements", ctypes.c_int64), ("workgroups", ctypes.c_int64), ("state_bits", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32), ("has_out", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class AdamwCfg(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("t", ctypes.c_int64), ("seed", ctypes.c_uint32)]


if not os.path.exists(LIB_PATH):
    raise ImportError("libcodistill.so is not built: run `python -m paper_2010_02838_amd.build` "
                      "(or __graft_entry__.build()) first; there is no fallback path")
lib = ctypes.CDLL(LIB_PATH)

_vp, _i64, _i32, _f32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_SIGS = {
    "codistill_arch_preset": [_i32, ctypes.POINTER(ArchDesc)],
    "codistill_model_create": [ctypes.POINTER(ArchDesc), _i32, ctypes.POINTER(_vp)],
    "codistill_param_count": [_vp, ctypes.POINTER(_i64), ctypes.POINTER(_i64)],
    "codistill_param_info": [_vp, _i64, ctypes.POINTER(TensorInfo)],
    "codistill_workspace_bytes": [_vp, _i64, _i32, ctypes.POINTER(_sz)],
    "codistill_bn_running_elements": [_vp, ctypes.POINTER(_i64)],
    "codistill_graph_size": [_vp, ctypes.POINTER(_i64), ctypes.POINTER(_i64)],
    "codistill_op_info": [_vp, _i64, _i64, ctypes.POINTER(OpInfo)],
    "codistill_tensor_info": [_vp, _i64, _i64, ctypes.POINTER(ActInfo)],
    "codistill_forward": [_vp, _vp, _vp, _i64, _i32, _i32, _vp, _vp, _sz, _vp, _vp],
    "codistill_loss_scratch_bytes": [_i64, _i64, ctypes.POINTER(_sz)],
    "codistill_loss_grad": [_vp, ctypes.POINTER(_vp), _vp, _i64, _i64, ctypes.POINTER(LossCfg), _vp, _vp, _vp, _sz, _vp],
    "codistill_loss_grad_static": [_vp, ctypes.POINTER(_vp), _vp, _i64, _i64, ctypes.POINTER(LossCfg), _vp, _vp, _vp],
    "codistill_backward": [_vp, _vp, _vp, _i64, _vp, _sz, _vp, _vp, _vp],
    "codistill_backward_streams": [_vp, _vp, _vp, _i64, _vp, _sz, _vp, _vp, _i32, _vp],
    "codistill_sgd_step": [_vp, _vp, _vp, _vp, _i64, _f32, _f32, _f32, _i32, _vp],
    "codistill_adam_step": [_vp, _vp, _vp, _vp, _vp, _i64, _f32, _f32, _f32, _f32, _f32, _i64, _vp],
    "codistill_rotary": [ctypes.POINTER(Rotary), _vp, _i64, ctypes.POINTER(RotaryTensor), _i64, _i32, _vp],
    "codistill_diff_attention_workspace_bytes": [ctypes.POINTER(DiffAttn), _i32, ctypes.POINTER(_sz)],
    "codistill_diff_attention": [ctypes.POINTER(DiffAttn)] + [_vp] * 8 + [_sz, _vp],
    "codistill_diff_attention_backward": [ctypes.POINTER(DiffAttn)] + [_vp] * 13 + [_sz, _vp],
    "codistill_head_norm": [_i32, _vp, _i64, _vp, _vp, _i64, _i64, _i64, _i64, _f32, _f32, _vp],
    "codistill_head_norm_workspace_bytes": [_i64, _i64, _i64, ctypes.POINTER(_sz)],
    "codistill_head_norm_backward": [_i32, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _f32, _f32, _vp, _sz, _vp],
    "codistill_adamw_table_bytes": [ctypes.POINTER(AdamwTensor), _i64, ctypes.POINTER(_sz)],
    "codistill_adamw_table": [ctypes.POINTER(AdamwTensor), _i64, _i32, _i32, _vp, _sz, ctypes.POINTER(AdamwPlan)],
    "codistill_adamw_step": [ctypes.POINTER(AdamwPlan), _vp, ctypes.POINTER(AdamwCfg), _vp, _vp],
    "codistill_adamw_unpack": [ctypes.POINTER(AdamwPlan), _vp, _vp],
    "codistill_profile_enable": [_i32],
    "codistill_profile_collect": [],
    "codistill_profile_get": [_i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_i64),
                              ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)],
    "codistill_profile_reset": [],
    "codistill_profile_event_overhead": [ctypes.POINTER(ctypes.c_double), _vp],
}
for _n, _a in _SIGS.items():
    getattr(lib, _n).argtypes = _a
    getattr(lib, _n).restype = ctypes.c_int
lib.codistill_model_destroy.argtypes = [_vp]
lib.codistill_model_destroy.restype = None
lib.codistill_last_error.restype = ctypes.c_char_p
lib.codistill_version.restype = ctypes.c_char_p
EXPORTED = list(_SIGS) + ["codistill_model_destroy", "codistill_last_error", "codistill_version"]


class CodistillError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("codistill error %d: %s" % (code, msg))
        self.code = code


def _check(rc):
    if rc != CD_OK:
        raise CodistillError(rc, lib.codistill_last_error().decode())


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def arch_preset(kind, **overrides):
    a = ArchDesc()
    _check(lib.codistill_arch_preset(kind, ctypes.byref(a)))
    for k, v in overrides.items():
        if k in ("widths", "blocks", "out_widths"):
            for i, x in enumerate(v):
                getattr(a, k)[i] = x
            if k == "widths" and a.kind != CD_ARCH_TINY_CNN:
                a.n_stages = len(v)
        else:
            setattr(a, k, v)
    return a


class Model:
    """Host-side model description (op list, parameter table)."""

    def __init__(self, arch, dtype):
        self.arch, self.dtype = arch, dtype
        self._h = _vp()
        _check(lib.codistill_model_create(ctypes.byref(arch), dtype, ctypes.byref(self._h)))
        nt, ne = _i64(), _i64()
        _check(lib.codistill_param_count(self._h, ctypes.byref(nt), ctypes.byref(ne)))
        self.n_tensors, self.n_elements = nt.value, ne.value
        self.params = []
        for i in range(self.n_tensors):
            ti = TensorInfo()
            _check(lib.codistill_param_info(self._h, i, ctypes.byref(ti)))
            self.params.append(dict(name=ti.name.decode(), kind=PARAM_KINDS[ti.kind], shape=tuple(ti.shape[:ti.ndim]),
                                    offset=ti.offset, size=ti.size, fan_in=ti.fan_in, frozen=bool(ti.frozen)))
        # frozen tensors (a frozen front end) come first: the update covers the flat buffers from here on
        self.trainable_offset = min([p["offset"] for p in self.params if not p["frozen"]] + [self.n_elements])
        self.classes = arch.classes
        # rows of logits per element of the batch: target tokens per sentence for the Transformer, else 1
        self.rows_per_sample = arch.in_w if arch.kind == CD_ARCH_TRANSFORMER else 1
        self.torch_dtype = torch.bfloat16 if dtype == CD_BF16 else torch.float32

    def __del__(self):
        if getattr(self, "_h", None) and lib is not None:   # module globals are gone at interpreter exit
            lib.codistill_model_destroy(self._h)
            self._h = None

    def param_table(self):
        """(name, shape, kind, fan_in) in declaration order, for the input generators."""
        return [(p["name"], p["shape"], p["kind"], p["fan_in"]) for p in self.params]

    def graph(self, batch):
        """(ops, tensors) as lists of dicts: the fused op list and the workspace layout for this batch."""
        no, nt = _i64(), _i64()
        _check(lib.codistill_graph_size(self._h, ctypes.byref(no), ctypes.byref(nt)))
        ops, tensors = [], []
        kinds = ["conv", "bn", "maxpool", "gap", "linear", "layernorm", "embed", "attn", "slice"]
        for i in range(no.value):
            o = OpInfo()
            _check(lib.codistill_op_info(self._h, batch, i, ctypes.byref(o)))
            d = {f: getattr(o, f) for f, _ in OpInfo._fields_}
            d["kind"] = kinds[o.kind]
            ops.append(d)
        for i in range(nt.value):
            t = ActInfo()
            _check(lib.codistill_tensor_info(self._h, batch, i, ctypes.byref(t)))
            tensors.append({f: getattr(t, f) for f, _ in ActInfo._fields_})
        return ops, tensors

    def bn_running_elements(self):
        n = _i64()
        _check(lib.codistill_bn_running_elements(self._h, ctypes.byref(n)))
        return n.value

    def workspace_bytes(self, batch, save_for_backward):
        b = _sz()
        _check(lib.codistill_workspace_bytes(self._h, batch, int(save_for_backward), ctypes.byref(b)))
        return b.value


def codistill_forward(model, params, x, workspace, logits_out, save_for_backward, bn_mode=CD_BN_BATCH_STATS,
                      bn_running=None):
    """z = f_params(x).  params: flat tensor in the model dtype; x: [B,H,W,3]; logits_out: [B,classes] fp32."""
    batch = x.shape[0]
    _check(lib.codistill_forward(model._h, _ptr(params), _ptr(x), batch, int(save_for_backward), bn_mode, _ptr(bn_running),
                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(logits_out),
                                 _stream()))


def loss_scratch_bytes(rows, cols):
    b = _sz()
    _check(lib.codistill_loss_scratch_bytes(rows, cols, ctypes.byref(b)))
    return b.value


def codistill_loss_grad(z_local, z_peers, targets, loss_out, dz_out, scratch, alpha, label_smoothing=0.0,
                        dist_kind=CD_DIST_MSE_LOGITS, mse_reduction=CD_MEAN_ALL, ignore_index=-1, temperature=1.0):
    """loss_out: float32[4] device tensor (total, task, distill, status bits)."""
    rows, cols = z_local.shape
    peers = list(z_peers) if z_peers is not None else []
    cfg = LossCfg(alpha, label_smoothing, dist_kind, mse_reduction, ignore_index, len(peers), temperature)
    arr = (_vp * max(len(peers), 1))(*[p.data_ptr() for p in peers])
    _check(lib.codistill_loss_grad(_ptr(z_local), arr if peers else None, _ptr(targets), rows, cols,
                                   ctypes.byref(cfg), _ptr(loss_out), _ptr(dz_out), _ptr(scratch),
                                   scratch.numel() * scratch.element_size(), _stream()))


def codistill_loss_grad_static(z_local, z_peers, targets, loss_out, dz_out, alpha, label_smoothing=0.0,
                               dist_kind=CD_DIST_MSE_LOGITS, mse_reduction=CD_MEAN_ALL, ignore_index=-1, temperature=1.0):
    """codistill_loss_grad without a scratch argument (the library's own fixed device array; rows <= 65536)."""
    rows, cols = z_local.shape
    peers = list(z_peers) if z_peers is not None else []
    cfg = LossCfg(alpha, label_smoothing, dist_kind, mse_reduction, ignore_index, len(peers), temperature)
    arr = (_vp * max(len(peers), 1))(*[p.data_ptr() for p in peers])
    _check(lib.codistill_loss_grad_static(_ptr(z_local), arr if peers else None, _ptr(targets), rows, cols,
                                          ctypes.byref(cfg), _ptr(loss_out), _ptr(dz_out), _stream()))


def codistill_backward(model, params, x, workspace, dlogits, grads_out, streams=CD_STREAMS_AUTO):
    _check(lib.codistill_backward_streams(model._h, _ptr(params), _ptr(x), x.shape[0], _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _ptr(dlogits), _ptr(grads_out),
                                          streams, _stream()))


def codistill_sgd_step(master_w, momentum_v, grad, lowp_w_out, lr, momentum, weight_decay=0.0, nesterov=False):
    _check(lib.codistill_sgd_step(_ptr(master_w), _ptr(momentum_v), _ptr(grad), _ptr(lowp_w_out), master_w.numel(),
                                  lr, momentum, weight_decay, int(nesterov), _stream()))


def codistill_adam_step(master_w, exp_avg, exp_avg_sq, grad, lowp_w_out, lr, t, beta1=0.9, beta2=0.98, eps=1e-8,
                        weight_decay=0.0):
    _check(lib.codistill_adam_step(_ptr(master_w), _ptr(exp_avg), _ptr(exp_avg_sq), _ptr(grad), _ptr(lowp_w_out),
                                   master_w.numel(), lr, beta1, beta2, eps, weight_decay, int(t), _stream()))


_raw_stream = getattr(getattr(torch, "_C", None), "_cuda_getCurrentRawStream", None)


def _stream_ptr():
    """The current stream's handle; without the stream object where torch lets one (5 of the 15 us of a small call were spent on it)."""
    return _raw_stream(torch.cuda.current_device()) if _raw_stream else torch.cuda.current_stream().cuda_stream


def _dtype(t):
    if t.dtype is torch.bfloat16:
        return CD_BF16
    if t.dtype is torch.float32:
        return CD_F32
    raise TypeError("bf16 or fp32 tensors only, got %s" % t.dtype)


def _inner(t, dims, what):
    """The last `dims` dimensions have to be contiguous; returns the strides of the others."""
    if t.is_contiguous():
        return t.stride()[:t.dim() - dims]
    run = 1
    for d in range(t.dim() - 1, t.dim() - 1 - dims, -1):
        if t.shape[d] != 1 and t.stride(d) != run:
            raise ValueError("%s: the channels of a token have to be contiguous" % what)
        run *= t.shape[d]
    return t.stride()[:t.dim() - dims]


def rotary_desc(dim, sections, theta, dtype, layout=CD_ROPE_HALVES, freq=None):
    """Rotary positions of heads of `dim` channels.  sections: pairs of each axis, in the order of `positions`' rows; pairs behind the last
    one are copied.  One ladder of frequencies over all pairs, theta^(-2p/dim), unless `freq` gives them (radians a position)."""
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    if len(axis) > min(dim // 2, CD_ROPE_MAX_PAIRS):
        raise ValueError("rotary: %d pairs in heads of %d channels" % (len(axis), dim))
    freq = [theta ** (-2.0 * p / dim) for p in range(len(axis))] if freq is None else list(freq)
    if len(freq) != len(axis):
        raise ValueError("rotary: %d frequencies for %d pairs" % (len(freq), len(axis)))
    d = Rotary(CD_BF16 if dtype is torch.bfloat16 else CD_F32, dim, len(axis), len(sections), layout)
    d.axis[:len(axis)] = axis
    d.freq[:len(freq)] = freq
    return d


_ROTARY_ARRAYS = {n: RotaryTensor * n for n in range(1, CD_ROPE_MAX_TENSORS + 1)}


def codistill_rotary(desc, positions, tensors, inverse=False):
    """positions: int32 [axes, tokens]; tensors: up to four pairs (x, y) of [tokens, heads, dim] (y may be x); inverse: the gradient."""
    n, tokens, dim = len(tensors), positions.shape[1], desc.dim
    arr = _ROTARY_ARRAYS[n]() if n in _ROTARY_ARRAYS else (RotaryTensor * n)()
    if positions.dtype is not torch.int32 or not positions.is_contiguous() or positions.shape[0] < desc.axes:
        raise ValueError("rotary: positions are contiguous int32 [axes, tokens]")
    dtype = torch.bfloat16 if desc.dtype == CD_BF16 else torch.float32
    for a, (x, y) in zip(arr, tensors):
        shape = x.shape
        if shape != y.shape or len(shape) != 3 or shape[0] != tokens or shape[2] != dim or x.dtype is not dtype or y.dtype is not dtype:
            raise ValueError("rotary: tensors are [tokens, heads, dim] of the descriptor's type")
        xs, ys = x.stride(), y.stride()
        if xs[1:] != (dim, 1) or ys[1:] != (dim, 1):
            _inner(x, 2, "rotary"), _inner(y, 2, "rotary")
        a.x, a.y, a.heads, a.x_token, a.y_token = x.data_ptr(), y.data_ptr(), shape[1], xs[0], ys[0]
    _check(lib.codistill_rotary(desc, positions.data_ptr(), tokens, arr, n, inverse, _stream_ptr()))


def diff_attention_desc(q, k, v, out, lam, causal=False, scale=0.0, q_lens=None, k_lens=None, q_starts=None, k_starts=None, max_q=0, max_k=0):
    """What differential attention of tensors laid out like these needs to know; kept by the caller and handed to every call.

    Padded: q [B, Tq, H, 2, D], k [B, Tk, Hk, 2, D], v [B, Tk, Hk, 2 D], out [B, Tq, H, 2 D], q_lens / k_lens int32 [B] or None.
    Packed (q_starts, k_starts int32 [B + 1] and the longest sequence's max_q, max_k, both): the same without the batch dimension.
    lam: fp32 [H], or [B, Tq, H] / [rows, H].  Tokens and sequences may be strided, the channels of a token are contiguous."""
    packed = q_starts is not None or k_starts is not None
    off = 0 if packed else 1
    if (q_starts is None) != (k_starts is None):
        raise ValueError("diff_attention: one of q_starts and k_starts without the other")
    if q.dim() != 4 + off or k.dim() != 4 + off or v.dim() != 3 + off or out.dim() != 3 + off or q.shape[-2] != 2 or k.shape[-2] != 2:
        raise ValueError("diff_attention: q, k are [.., heads, 2, head_dim], v and out [.., heads, 2 head_dim]")
    dim, heads, kv_heads = q.shape[-1], q.shape[off + 1], k.shape[off + 1]
    if (k.shape[-1] != dim or v.shape[-1] != 2 * dim or v.shape[off + 1] != kv_heads or out.shape != q.shape[:off + 2] + (2 * dim,)
            or k.shape[:off + 1] != v.shape[:off + 1] or (off and k.shape[0] != q.shape[0])):
        raise ValueError("diff_attention: the shapes of q, k, v and out do not fit")
    if any(t.dtype is not q.dtype for t in (k, v, out)) or lam.dtype is not torch.float32 or not lam.is_contiguous():
        raise TypeError("diff_attention: q, k, v and out have one type, lambda is contiguous fp32")
    if tuple(lam.shape) not in ((heads,), tuple(q.shape[:off + 2])):
        raise ValueError("diff_attention: lambda is [heads] or one for each query and head")
    batch = q_starts.numel() - 1 if packed else q.shape[0]
    for t, n in ((q_lens, batch), (k_lens, batch), (q_starts, batch + 1), (k_starts, batch + 1)):
        if t is not None and (t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or t.device != q.device):
            raise ValueError("diff_attention: lens are int32 [batch], starts int32 [batch + 1], on the queries' device")
    d = DiffAttn(dtype=_dtype(q), batch=batch, tq=max_q if packed else q.shape[1], tk=max_k if packed else k.shape[1], heads=heads, kv_heads=kv_heads,
                 head_dim=dim, causal=int(causal), lambda_kind=CD_LAMBDA_HEAD if lam.dim() == 1 else CD_LAMBDA_TOKEN, scale=scale,
                 q_rows=q.shape[0] if packed else 0, k_rows=k.shape[0] if packed else 0)
    for name, t, inner in (("q", q, 3), ("k", k, 3), ("v", v, 2), ("o", out, 2)):
        s = _inner(t, inner, "diff_attention")
        # (the stride of a dimension of one element says nothing)
        setattr(d, name + "_token", s[-1] if t.shape[off] > 1 else t.shape[off + 1] * 2 * dim)
        setattr(d, name + "_batch", s[0] if off and batch > 1 else 0)
    for name, t in (("q_lens", q_lens), ("k_lens", k_lens), ("q_starts", q_starts), ("k_starts", k_starts)):
        if t is not None:
            setattr(d, name, t.data_ptr())
    d.keep = (q_lens, k_lens, q_starts, k_starts)
    d.layout = tuple((t.shape, t.stride(), t.dtype) for t in (q, k, v, out, lam))
    d.lse_shape = (2, heads, q.shape[0] * (q.shape[1] if off else 1))
    return d


def _laid_out(desc, tensors):
    """The kernels go by the descriptor: a tensor of another shape, stride or type would be read beyond its end."""
    for t, want in zip(tensors, desc.layout):
        if (t.shape, t.stride(), t.dtype) != want and ((t.shape, t.dtype) != (want[0], want[2]) or any(
                n > 1 and x != y for n, x, y in zip(t.shape, t.stride(), want[1]))):
            raise ValueError("diff_attention: a tensor of shape %s, strides %s, %s where the descriptor has %s, %s, %s" % (
                tuple(t.shape), t.stride(), t.dtype, tuple(want[0]), want[1], want[2]))


def _kept(desc, o_second, lse):
    shape, _, dtype = desc.layout[3]
    if o_second.shape != shape or o_second.dtype is not dtype or not o_second.is_contiguous() or lse.shape != desc.lse_shape or (
            lse.dtype is not torch.float32 or not lse.is_contiguous()):
        raise ValueError("diff_attention: o_second is contiguous in out's shape, lse fp32 %s" % (desc.lse_shape,))


def diff_attention_workspace_bytes(desc, backward):
    b = _sz()
    _check(lib.codistill_diff_attention_workspace_bytes(ctypes.byref(desc), int(backward), ctypes.byref(b)))
    return b.value


def _room(t):
    return 0 if t is None else t.numel() * t.element_size()


def codistill_diff_attention(desc, q, k, v, lam, out, o_second=None, lse=None, workspace=None):
    """out = (softmax(q_1 k_1) - lam softmax(q_2 k_2)) v.  o_second (contiguous, out's shape) and lse (fp32 [2, heads, rows of q]) are kept for
    the backward pass; both or neither."""
    _laid_out(desc, (q, k, v, out, lam))
    if o_second is not None and lse is not None:
        _kept(desc, o_second, lse)
    _check(lib.codistill_diff_attention(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(lam), _ptr(out), _ptr(o_second), _ptr(lse), _ptr(workspace),
                                        _room(workspace), _stream_ptr()))


def codistill_diff_attention_backward(desc, q, k, v, lam, out, o_second, lse, dout, dq, dk, dv, dlam, workspace):
    """Gradients; dout is laid out like out, dq, dk, dv like q, k, v, dlam like lam."""
    _laid_out(desc, (q, k, v, out, lam))
    _laid_out(desc, (dq, dk, dv, dout, dlam))
    _kept(desc, o_second, lse)
    _check(lib.codistill_diff_attention_backward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(lam), _ptr(out), _ptr(o_second), _ptr(lse), _ptr(dout),
                                                 _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dlam), _ptr(workspace), _room(workspace), _stream_ptr()))


def head_norm_workspace_bytes(rows, heads, width):
    b = _sz()
    _check(lib.codistill_head_norm_workspace_bytes(rows, heads, width, ctypes.byref(b)))
    return b.value


def codistill_head_norm(x, gain, y, eps=1e-5, post=1.0):
    """y = post gain x / sqrt(mean(x^2) + eps) over the last dimension of x [rows, heads, width]."""
    if x.shape != y.shape or gain.shape != x.shape[2:] or y.dtype is not x.dtype or gain.dtype is not x.dtype or not gain.is_contiguous():
        raise ValueError("head_norm: x and y are [rows, heads, width], gain contiguous [width], all of one type")
    _check(lib.codistill_head_norm(_dtype(x), x.data_ptr(), _inner(x, 2, "head_norm")[0], gain.data_ptr(), y.data_ptr(), _inner(y, 2, "head_norm")[0], *x.shape, eps, post,
                                   _stream_ptr()))


def codistill_head_norm_backward(x, gain, dy, dx, dgain, workspace, eps=1e-5, post=1.0):
    """dx (may be dy) and dgain (fp32 [width]) of codistill_head_norm."""
    if x.shape != dy.shape or x.shape != dx.shape or gain.shape != x.shape[2:] or dgain.shape != gain.shape:
        raise ValueError("head_norm_backward: x, dy and dx are [rows, heads, width], gain and dgain [width]")
    if any(t.dtype is not x.dtype for t in (gain, dy, dx)) or dgain.dtype is not torch.float32 or not (gain.is_contiguous() and dgain.is_contiguous()):
        raise ValueError("head_norm_backward: one type, dgain fp32, gain and dgain contiguous")
    _check(lib.codistill_head_norm_backward(_dtype(x), _ptr(x), _inner(x, 2, "head_norm")[0], _ptr(gain), _ptr(dy), _inner(dy, 2, "head_norm")[0], _ptr(dx),
                                            _inner(dx, 2, "head_norm")[0], _ptr(dgain), x.shape[0], x.shape[1], x.shape[2], eps, post, _ptr(workspace),
                                            _room(workspace), _stream_ptr()))


def adamw_table(tensors, state_bits, grad_dtype):
    """(plan, host bytes) of a list of AdamwTensor: the bytes go to device memory, and both to every step."""
    arr = (AdamwTensor * len(tensors))(*tensors)
    n, plan = _sz(), AdamwPlan()
    _check(lib.codistill_adamw_table_bytes(arr, len(tensors), ctypes.byref(n)))
    host = torch.empty(n.value, dtype=torch.uint8)
    _check(lib.codistill_adamw_table(arr, len(tensors), state_bits, grad_dtype, _ptr(host), n.value, ctypes.byref(plan)))
    return plan, host


def codistill_adamw_step(plan, table, lr, t, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, grad_scale=None):
    """grad_scale: fp32 device tensor of one element, or None."""
    if grad_scale is not None and (grad_scale.dtype is not torch.float32 or grad_scale.numel() != 1):
        raise ValueError("adamw: grad_scale is an fp32 tensor of one element")
    cfg = AdamwCfg(lr, beta1, beta2, eps, int(t), seed & 0xffffffff)
    _check(lib.codistill_adamw_step(ctypes.byref(plan), _ptr(table), ctypes.byref(cfg), _ptr(grad_scale), _stream_ptr()))


def codistill_adamw_unpack(plan, table):
    _check(lib.codistill_adamw_unpack(ctypes.byref(plan), _ptr(table), _stream_ptr()))


def profile_enable(on):
    _check(lib.codistill_profile_enable(int(on)))


def profile_reset():
    _check(lib.codistill_profile_reset())


def profile_event_overhead():
    """Microseconds that the timer's event pair adds to a launch (measured on the current stream)."""
    us = ctypes.c_double()
    _check(lib.codistill_profile_event_overhead(ctypes.byref(us), _stream()))
    return us.value


def profile_collect():
    """Returns {class: dict(ms, launches, flops, bytes)} accumulated since the last reset."""
    _check(lib.codistill_profile_collect())
    out = {}
    for i, name in enumerate(KERNEL_CLASSES):
        ms, fl, by, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_double(), _i64()
        _check(lib.codistill_profile_get(i, ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl), ctypes.byref(by)))
        out[name] = dict(ms=ms.value, launches=n.value, flops=fl.value, bytes=by.value)
    return out
