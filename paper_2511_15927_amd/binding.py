"""ctypes binding of the C ABI in include/bimamba.h: argument marshalling only.

Tensors are torch tensors on the GPU (torch owns device memory and streams); every step of the path runs in the
HIP library.  There is no fallback: if libbimamba.so has not been built, loading raises.
"""
import ctypes as C
import os
import struct

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbimamba.so")

F32, BF16 = 0, 1
A_PER_HEAD_STATE, A_SCALAR_PER_HEAD = 0, 1
D_PER_CHANNEL, D_PER_HEAD = 0, 1
COMBINE_ADD, COMBINE_SEPARATE = 0, 1

STATUS = {0: "BIMAMBA_OK", -1: "BIMAMBA_ERR_NULL_POINTER", -2: "BIMAMBA_ERR_BAD_SHAPE", -3: "BIMAMBA_ERR_UNSUPPORTED",
          -4: "BIMAMBA_ERR_MISALIGNED", -5: "BIMAMBA_ERR_WORKSPACE_TOO_SMALL", -6: "BIMAMBA_ERR_HIP",
          -7: "BIMAMBA_ERR_SCRATCH_EXCEEDED", -8: "BIMAMBA_ERR_ALIAS"}
STATIC_SCRATCH_BYTES = 64 << 20

EXPORTS = ("bimamba_fwd", "bimamba_block_fwd", "bimamba_block_fwd_static", "bimamba_block_stack", "bimamba_block_stack_form",
           "bimamba_block_stack_side_by_side", "bimamba_copy_inputs", "bimamba_bwd", "bimamba_workspace_bytes",
           "bimamba_bwd_workspace_bytes", "bimamba_time_chunks", "bimamba_profile_next_call", "bimamba_status_string", "bimamba_version",
           "bimamba_embed", "bimamba_embed_bwd", "bimamba_embed_bwd_workspace_bytes", "bimamba_layer_norm", "bimamba_layer_norm_bwd",
           "bimamba_layer_norm_bwd_workspace_bytes", "bimamba_log_probs", "bimamba_log_probs_bwd", "bimamba_log_probs_workspace_bytes",
           "bimamba_clip_layout", "bimamba_clip_grads", "bimamba_clip_grads_workspace_bytes",
           "bimamba_recurrence", "bimamba_recurrence_workspace_bytes", "bimamba_recurrence_bwd", "bimamba_recurrence_bwd_workspace_bytes",
           "bimamba_group_norm", "bimamba_group_norm_bwd", "bimamba_group_norm_bwd_workspace_bytes",
           "bimamba_dropout_add", "bimamba_dropout_add_bwd", "bimamba_dropout_add_bwd_workspace_bytes")


class Desc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "batch", "seqlen", "d_inner", "d_state", "n_heads", "n_groups", "d_conv", "io_dtype", "a_kind", "d_kind",
        "dt_softplus", "conv_bc", "combine", "time_chunks", "state_split")]


class Params(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("conv_w", "conv_b", "A", "D", "dt_bias")]


class Tensor(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_batch", C.c_int64), ("stride_token", C.c_int64)]


class Inputs(C.Structure):
    _fields_ = [(n, Tensor) for n in ("x", "z", "dt", "B", "C")]


class StackLayer(C.Structure):
    _fields_ = [("f", Params), ("b", Params), ("h", C.c_void_p), ("tail", C.c_void_p)]


class InputGrads(C.Structure):
    _fields_ = [("dx", Tensor), ("dz", Tensor), ("ddt", Tensor), ("dB", C.c_void_p), ("dC", C.c_void_p)]


class ParamGrads(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dconv_w", "dconv_b", "dA", "dD", "ddt_bias")]


class Tokens(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("stride_batch", C.c_int64), ("stride_token", C.c_int64)]


class EmbedDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "batch", "seqlen", "d_model", "vocab", "table_dtype", "io_dtype")] + [("scale", C.c_float)]


class NormDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in ("batch", "seqlen", "d_model", "io_dtype")] + [("eps", C.c_float)]


class LogitsDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "batch", "seqlen", "vocab", "io_dtype", "top_k", "targets_only", "reserved")] + [("lse_rest", C.c_void_p)]


class Scores(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("logp", "lse", "entropy", "top_logp", "top_token")]


class Grad(C.Structure):
    _fields_ = [("from_", C.c_void_p), ("to", C.c_void_p), ("count", C.c_int64), ("first", C.c_int64), ("dtype", C.c_int32),
                ("reserved", C.c_int32)]


class RecurrenceDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in ("batch", "seqlen", "d_inner", "io_dtype", "gate", "reverse")]


class GroupNormDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "batch", "seqlen", "d_inner", "groups", "io_dtype", "act", "centred")] + [("eps", C.c_float)]


class DropoutDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in ("batch", "seqlen", "d_model", "io_dtype", "site")] + [("p", C.c_float)]


class BimambaError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = lib().bimamba_status_string(status).decode()
        super().__init__("%s failed: %s (%s)" % (where, STATUS.get(status, status), msg))


_lib = None


def lib():
    """Load libbimamba.so (built by paper_2511_15927_amd/build.py); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libbimamba.so is not built: run `python -m paper_2511_15927_amd.build` "
                               "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.bimamba_fwd.restype = C.c_int
        L.bimamba_fwd.argtypes = [C.POINTER(Desc), C.POINTER(Params), C.POINTER(Params), C.POINTER(Inputs),
                                  C.POINTER(Inputs), C.POINTER(Tensor), C.c_void_p, C.c_size_t, C.c_void_p]
        L.bimamba_block_fwd.restype = C.c_int
        L.bimamba_block_fwd.argtypes = [C.POINTER(Desc), C.POINTER(Params), C.POINTER(Params), C.POINTER(Inputs),
                                        C.POINTER(Inputs), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                        C.POINTER(Tensor), C.c_void_p, C.c_size_t, C.c_void_p]
        L.bimamba_block_fwd_static.restype = C.c_int
        L.bimamba_block_fwd_static.argtypes = [C.POINTER(Desc), C.POINTER(Params), C.POINTER(Params), C.POINTER(Inputs),
                                               C.POINTER(Inputs), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                               C.POINTER(Tensor), C.c_void_p]
        L.bimamba_block_stack.restype = C.c_int
        L.bimamba_block_stack.argtypes = [C.POINTER(Desc), C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.bimamba_block_stack_form.restype = C.c_int
        L.bimamba_block_stack_form.argtypes = [C.POINTER(Desc)]
        L.bimamba_block_stack_side_by_side.restype = C.c_int
        L.bimamba_block_stack_side_by_side.argtypes = [C.POINTER(Desc), C.c_int]
        L.bimamba_copy_inputs.restype = C.c_int
        L.bimamba_copy_inputs.argtypes = [C.POINTER(Desc), C.POINTER(Inputs), C.POINTER(Inputs), C.c_void_p]
        L.bimamba_bwd.restype = C.c_int
        L.bimamba_bwd.argtypes = [C.POINTER(Desc), C.POINTER(Params), C.POINTER(Params), C.POINTER(Inputs),
                                  C.POINTER(Inputs), C.POINTER(Tensor), C.POINTER(InputGrads), C.POINTER(InputGrads),
                                  C.POINTER(ParamGrads), C.POINTER(ParamGrads), C.c_void_p, C.c_size_t, C.c_void_p]
        L.bimamba_bwd_workspace_bytes.restype = C.c_size_t
        L.bimamba_bwd_workspace_bytes.argtypes = [C.POINTER(Desc)]
        L.bimamba_workspace_bytes.restype = C.c_size_t
        L.bimamba_workspace_bytes.argtypes = [C.POINTER(Desc), C.c_int]
        L.bimamba_time_chunks.restype = C.c_int
        L.bimamba_time_chunks.argtypes = [C.POINTER(Desc)]
        L.bimamba_status_string.restype = C.c_char_p
        L.bimamba_status_string.argtypes = [C.c_int]
        L.bimamba_version.restype = C.c_int
        L.bimamba_profile_next_call.restype = None
        L.bimamba_profile_next_call.argtypes = [C.c_void_p, C.c_void_p]
        P, V, Z, I = C.POINTER, C.c_void_p, C.c_size_t, C.c_int
        T, I64 = P(Tensor), C.c_int64
        for name, res, args in (
                ("bimamba_recurrence", I, [P(RecurrenceDesc), T, T, V, T, V, V, T, V, V, V, Z, V]),
                ("bimamba_recurrence_workspace_bytes", Z, [P(RecurrenceDesc)]),
                ("bimamba_recurrence_bwd", I, [P(RecurrenceDesc), T, T, V, V, V, T, V, T, T, V, V, V, Z, V]),
                ("bimamba_recurrence_bwd_workspace_bytes", Z, [P(RecurrenceDesc)]),
                ("bimamba_group_norm", I, [P(GroupNormDesc), T, T, V, V, T, V, V, V]),
                ("bimamba_group_norm_bwd", I, [P(GroupNormDesc), T, T, V, V, V, V, T, T, T, V, V, V, Z, V]),
                ("bimamba_group_norm_bwd_workspace_bytes", Z, [P(GroupNormDesc)]),
                ("bimamba_dropout_add", I, [P(DropoutDesc), V, T, V, I64, T, T, V]),
                ("bimamba_dropout_add_bwd", I, [P(DropoutDesc), V, T, V, I64, T, T, V, V, Z, V]),
                ("bimamba_dropout_add_bwd_workspace_bytes", Z, [P(DropoutDesc), I]),
                ("bimamba_embed", I, [P(EmbedDesc), P(Tokens), V, P(Tensor), V]),
                ("bimamba_embed_bwd", I, [P(EmbedDesc), P(Tokens), P(Tensor), V, V, Z, V]),
                ("bimamba_embed_bwd_workspace_bytes", Z, [P(EmbedDesc)]),
                ("bimamba_layer_norm", I, [P(NormDesc), P(Tensor), V, V, C.c_int64, P(Tensor), V, V, V]),
                ("bimamba_layer_norm_bwd", I, [P(NormDesc), P(Tensor), V, C.c_int64, V, V, P(Tensor), P(Tensor), V, V, V, Z, V]),
                ("bimamba_layer_norm_bwd_workspace_bytes", Z, [P(NormDesc), I]),
                ("bimamba_log_probs", I, [P(LogitsDesc), P(Tensor), P(Tokens), P(Scores), V, Z, V]),
                ("bimamba_log_probs_bwd", I, [P(LogitsDesc), P(Tensor), P(Tokens), V, V, V, V, P(Tensor), V]),
                ("bimamba_log_probs_workspace_bytes", Z, [P(LogitsDesc)]),
                ("bimamba_clip_layout", I, [P(Grad), I]),
                ("bimamba_clip_grads", I, [P(Grad), I, V, C.c_float, V, V, Z, V]),
                ("bimamba_clip_grads_workspace_bytes", Z, [P(Grad), I])):
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def make_desc(cfg, seqlen=None, **override):
    """C descriptor from a config dict (keys as in synth.mixer_cfg)."""
    c = dict(cfg)
    c.update(override)
    return Desc(C.sizeof(Desc), c["batch"], c["seqlen"] if seqlen is None else seqlen, c["d_inner"], c["d_state"],
                c["n_heads"], c["n_groups"], c["d_conv"], BF16 if c["io"] == "bf16" else F32, c["a_kind"], c["d_kind"],
                c["dt_softplus"], c["conv_bc"], c["combine"], c.get("time_chunks", 0), c.get("state_split", 0))


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def make_params(p):
    """p: dict of float32 device tensors conv_w, conv_b, A, D, dt_bias (conv_b / dt_bias may be None)."""
    for k in ("conv_w", "conv_b", "A", "D", "dt_bias"):
        t = p.get(k)
        if t is not None:
            assert t.dtype == torch.float32 and t.is_contiguous(), k
    return Params(_ptr(p["conv_w"]), _ptr(p.get("conv_b")), _ptr(p["A"]), _ptr(p["D"]), _ptr(p.get("dt_bias")))


def make_tensor(t):
    """[batch, L, channels] view with unit channel stride (batch/token strides are passed through)."""
    assert t.dim() == 3 and (t.numel() == 0 or t.shape[2] == 1 or t.stride(2) == 1), "channel dimension must be contiguous"
    return Tensor(t.data_ptr(), t.stride(0), t.stride(1))


_INPUT_WORDS = struct.Struct("=" + "Qqq" * 5)
assert _INPUT_WORDS.size == C.sizeof(Inputs)


def input_words(words):
    """Inputs from pointer, batch stride and token stride of x, z, dt, B and C, in that order."""
    return Inputs.from_buffer_copy(_INPUT_WORDS.pack(*words))


def make_inputs(i):
    """i: dict of device tensors x, z [Bt,L,Dn]; dt [Bt,L,H]; B, C [Bt,L,G,N] or [Bt,L,G*N]."""
    # (the host's share of a call counts: 256 tokens of 512 channels run in 9.7 us and took 12.6 with a struct a tensor and a stream object)
    words = []
    for k in ("x", "z", "dt", "B", "C"):
        t = i[k]
        strides = t.stride()
        if len(strides) == 4:
            assert t.shape[2] == 1 or strides[2] == t.shape[3] * strides[3], "B/C groups must be adjacent"
        else:
            assert len(strides) == 3, "channel dimension must be contiguous"
        assert strides[-1] == 1 or t.numel() == 0 or t.shape[2:].numel() == 1, "channel dimension must be contiguous"
        words += (t.data_ptr(), strides[0], strides[1])
    return input_words(words)


def _stream_ptr(stream):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return C.c_void_p(stream.cuda_stream)


def bimamba_workspace_bytes(desc, block_variant=0):
    return int(lib().bimamba_workspace_bytes(C.byref(desc), int(block_variant)))


def bimamba_time_chunks(desc):
    return int(lib().bimamba_time_chunks(C.byref(desc)))


def bimamba_version():
    return int(lib().bimamba_version())


def bimamba_profile_next_call(ev_start, ev_stop):
    """ev_start/ev_stop: torch.cuda.Event(enable_timing=True) that have been recorded once (so the HIP event
    exists), or None to disarm."""
    h0 = None if ev_start is None else C.c_void_p(ev_start.cuda_event)
    h1 = None if ev_stop is None else C.c_void_p(ev_stop.cuda_event)
    lib().bimamba_profile_next_call(h0, h1)


def bimamba_fwd(desc, pf, pb, in_f, in_b, out, workspace, stream=None, check=True):
    """Enqueue the full-sequence path.  pf/pb: Params; in_f/in_b: Inputs (in_b None = shared); out: Tensor struct;
    workspace: uint8 device tensor or None.  Returns the status code (raises on error when check)."""
    ws_ptr = None if workspace is None else C.c_void_p(workspace.data_ptr())
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().bimamba_fwd(C.byref(desc), C.byref(pf), C.byref(pb), C.byref(in_f),
                           None if in_b is None else C.byref(in_b), C.byref(out), ws_ptr, ws_bytes, _stream_ptr(stream))
    if check and rc != 0:
        raise BimambaError(rc, "bimamba_fwd")
    return rc


def make_input_grads(g):
    """g: dict of device tensors dx, dz [Bt,L,Dn], ddt [Bt,L,H] (io dtype, unit channel stride) and dB, dC
    [Bt,L,G,N] float32 contiguous."""
    for k in ("dB", "dC"):
        assert g[k].dtype == torch.float32 and g[k].is_contiguous(), k
    return InputGrads(make_tensor(g["dx"]), make_tensor(g["dz"]), make_tensor(g["ddt"]), g["dB"].data_ptr(), g["dC"].data_ptr())


def make_param_grads(g):
    """g: dict of float32 contiguous device tensors dconv_w, dA, dD and optionally dconv_b, ddt_bias."""
    for k in ("dconv_w", "dconv_b", "dA", "dD", "ddt_bias"):
        t = g.get(k)
        if t is not None:
            assert t.dtype == torch.float32 and t.is_contiguous(), k
    return ParamGrads(_ptr(g["dconv_w"]), _ptr(g.get("dconv_b")), _ptr(g["dA"]), _ptr(g["dD"]), _ptr(g.get("ddt_bias")))


def bimamba_bwd_workspace_bytes(desc):
    return int(lib().bimamba_bwd_workspace_bytes(C.byref(desc)))


def bimamba_bwd(desc, pf, pb, in_f, in_b, dout, din_f, din_b, dpf, dpb, workspace, stream=None, check=True):
    """Enqueue the gradients of bimamba_fwd.  dout: Tensor; din_f/din_b: InputGrads (din_b None with shared
    activations); dpf/dpb: ParamGrads; workspace: uint8 device tensor of bimamba_bwd_workspace_bytes(desc)."""
    ws_ptr = None if workspace is None else C.c_void_p(workspace.data_ptr())
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().bimamba_bwd(C.byref(desc), C.byref(pf), C.byref(pb), C.byref(in_f), None if in_b is None else C.byref(in_b),
                           C.byref(dout), C.byref(din_f), None if din_b is None else C.byref(din_b), C.byref(dpf),
                           C.byref(dpb), ws_ptr, ws_bytes, _stream_ptr(stream))
    if check and rc != 0:
        raise BimambaError(rc, "bimamba_bwd")
    return rc


def bimamba_block_fwd(desc, pf, pb, in_f, in_b, h_in, tail_in, h_out, tail_out, out, workspace, stream=None, check=True):
    """Enqueue the block variant.  h_in/h_out: float32 device tensors or None; tail_in/tail_out: io-dtype device
    tensors or None."""
    ws_ptr = None if workspace is None else C.c_void_p(workspace.data_ptr())
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = lib().bimamba_block_fwd(C.byref(desc), C.byref(pf), C.byref(pb), C.byref(in_f),
                                 None if in_b is None else C.byref(in_b), _ptr(h_in), _ptr(tail_in), _ptr(h_out),
                                 _ptr(tail_out), C.byref(out), ws_ptr, ws_bytes, _stream_ptr(stream))
    if check and rc != 0:
        raise BimambaError(rc, "bimamba_block_fwd")
    return rc


def bimamba_block_fwd_static(desc, pf, pb, in_f, in_b, h_in, tail_in, h_out, tail_out, out, stream=None, check=True):
    """bimamba_block_fwd on the library's own fixed scratch buffer: no workspace argument, nothing allocated."""
    rc = lib().bimamba_block_fwd_static(C.byref(desc), C.byref(pf), C.byref(pb), C.byref(in_f),
                                        None if in_b is None else C.byref(in_b), _ptr(h_in), _ptr(tail_in), _ptr(h_out),
                                        _ptr(tail_out), C.byref(out), _stream_ptr(stream))
    if check and rc != 0:
        raise BimambaError(rc, "bimamba_block_fwd_static")
    return rc


def bimamba_block_stack_form(desc):
    return int(lib().bimamba_block_stack_form(C.byref(desc)))


def bimamba_block_stack_side_by_side(desc, n_steps):
    return int(lib().bimamba_block_stack_side_by_side(C.byref(desc), n_steps))


def make_stack_table(layers, steps, outs):
    """layers: StackLayer structs; steps: Inputs structs; outs: one output tensor or None per (step, layer), layers fastest.
    Returns the table's bytes."""
    assert len(outs) == len(layers) * len(steps)
    return b"".join(bytes(s) for s in list(layers) + list(steps)) + bytes((C.c_void_p * len(outs))(*[0 if o is None else o.data_ptr() for o in outs]))


def bimamba_block_stack(desc, n_layers, n_steps, table, table_dev, stream=None, check=True):
    """Enqueue all steps of a block through the stack.  table: make_stack_table's bytes; table_dev: a uint8 device tensor
    holding the same."""
    rc = lib().bimamba_block_stack(C.byref(desc), n_layers, n_steps, table, C.c_void_p(table_dev.data_ptr()), _stream_ptr(stream))
    if check and rc != 0:
        raise BimambaError(rc, "bimamba_block_stack")
    return rc


def bimamba_copy_inputs(desc, src, dst, stream=None, check=True):
    """Enqueue the copy of a call's inputs into buffers of the caller.  src, dst: Inputs structs."""
    rc = lib().bimamba_copy_inputs(C.byref(desc), C.byref(src), C.byref(dst), _stream_ptr(stream))
    if check and rc != 0:
        raise BimambaError(rc, "bimamba_copy_inputs")
    return rc


# ---- what stands around the mixers: token table, layer norm, log probabilities, clipped gradients ----
#
# These take the tensors themselves.  csrc/torch_calls.cpp checks them against the descriptor (shape, type, unit stride along a row, on the
# GPU: an AssertionError) and makes the call.  Tensors of a call are on the current device, and the stream is the current one unless
# another is given.

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_NAMES = {"f32": F32, "bf16": BF16}
_calls_module = None


def _calls():
    """The extension module built beside libbimamba.so; raises if it is missing."""
    global _calls_module
    if _calls_module is None:
        lib()   # (which it is linked to)
        try:
            from . import _calls as module
        except ImportError as e:
            raise RuntimeError("_calls.so is not built: run `python -m paper_2511_15927_amd.build` (there is no CPU fallback): %s" % e) from e
        _calls_module = module
    return _calls_module


def _stream(stream):
    # (a call's tensors are on the GPU, so torch has been initialised; if they are not, the call ends before the stream is used)
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) if torch.cuda.is_initialized() else 0


def _checked(rc, name, check):
    if check and rc != 0:
        raise BimambaError(rc, name)
    return rc


def make_embed_desc(batch, seqlen, d_model, vocab, table="f32", io="bf16", scale=1.0):
    return EmbedDesc(C.sizeof(EmbedDesc), batch, seqlen, d_model, vocab, _NAMES[table], _NAMES[io], scale)


def bimamba_embed(desc, tokens, table, out, stream=None, check=True):
    """Enqueue out[b, t] = scale * table[tokens[b, t]].  tokens: int64 [batch, L]; table [vocab, d_model] contiguous; out
    [batch, L, d_model]."""
    return _checked((_calls_module or _calls()).embed(desc, tokens, table, out, _stream(stream)), "bimamba_embed", check)


def bimamba_embed_bwd_workspace_bytes(desc):
    return int(lib().bimamba_embed_bwd_workspace_bytes(C.byref(desc)))


def bimamba_embed_bwd(desc, tokens, dout, dtable, workspace, stream=None, check=True):
    """Enqueue the gradient of the table: dtable float32 [vocab, d_model] contiguous, overwritten."""
    return _checked((_calls_module or _calls()).embed_bwd(desc, tokens, dout, dtable, workspace, _stream(stream)), "bimamba_embed_bwd", check)


def make_norm_desc(batch, seqlen, d_model, io="bf16", eps=1e-5):
    return NormDesc(C.sizeof(NormDesc), batch, seqlen, d_model, _NAMES[io], eps)


def bimamba_layer_norm(desc, x, weight, bias, y, mean=None, rstd=None, stream=None, check=True):
    """Enqueue the layer norm of every row.  weight, bias: float32 [d_model], or [batch, d_model] with a vector for each batch
    element, or None; both of the same kind and row stride.  mean, rstd: float32 [batch, L] or None (bimamba_layer_norm_bwd takes them)."""
    return _checked((_calls_module or _calls()).layer_norm(desc, x, weight, bias, y, mean, rstd, _stream(stream)), "bimamba_layer_norm", check)


def bimamba_layer_norm_bwd_workspace_bytes(desc, per_batch):
    return int(lib().bimamba_layer_norm_bwd_workspace_bytes(C.byref(desc), int(per_batch)))


def bimamba_layer_norm_bwd(desc, x, weight, mean, rstd, dy, dx, dweight, dbias, workspace, stream=None, check=True):
    """Enqueue the gradients of bimamba_layer_norm.  dweight, dbias: float32 [d_model], or [batch, d_model] where each batch element
    has a vector of its own (weight None: their shape says which), or None; overwritten."""
    return _checked((_calls_module or _calls()).layer_norm_bwd(desc, x, weight, mean, rstd, dy, dx, dweight, dbias, workspace, _stream(stream)),
                    "bimamba_layer_norm_bwd", check)


def make_logits_desc(batch, seqlen, vocab, io="bf16", top_k=0, targets_only=0):
    return LogitsDesc(C.sizeof(LogitsDesc), batch, seqlen, vocab, _NAMES[io], top_k, targets_only)


def bimamba_log_probs_workspace_bytes(desc):
    return int(lib().bimamba_log_probs_workspace_bytes(C.byref(desc)))


def bimamba_log_probs(desc, logits, targets, out, workspace=None, stream=None, check=True):
    """Enqueue the log probabilities of targets (int64 [batch, L], or None) under softmax(logits).  out: dict of what is wanted:
    logp, lse, entropy float32 [batch, L]; lse_rest, of the same kind, is what rounding left of lse (bimamba_log_probs_bwd takes it);
    top_logp float32 and top_token int64 [batch, L, top_k]."""
    get = out.get
    rc = (_calls_module or _calls()).log_probs(desc, logits, targets, get("logp"), get("lse"), get("entropy"), get("top_logp"), get("top_token"),
                                               get("lse_rest"), workspace, _stream(stream))
    return _checked(rc, "bimamba_log_probs", check)


def bimamba_log_probs_bwd(desc, logits, targets, lse, entropy, dlogp, dentropy, dlogits, stream=None, check=True, lse_rest=None):
    """Enqueue the gradient for the logits, given those of logp and of the entropy (float32 [batch, L]; either None).  dlogits may be
    logits itself.  A descriptor with targets_only: rows without a target get zeros.  Without lse_rest the
    probabilities are off by up to 2^-24 |lse|, relatively."""
    return _checked((_calls_module or _calls()).log_probs_bwd(desc, logits, targets, lse, lse_rest, entropy, dlogp, dentropy, dlogits, _stream(stream)),
                    "bimamba_log_probs_bwd", check)


class GradTable:
    """The tensors of a clipping call, made once: where each gradient lies and where the scaled one goes (to None: in place).  Holds the
    tensors and the table's copy on the device.  It is of these tensors: gradients that a program frees and makes anew (a parameter's .grad
    after an optimizer's zero_grad()) are others, and want another table."""

    def __init__(self, grads, to=None):
        self.grads, self.to = list(grads), list(grads if to is None else to)
        assert len(self.grads) == len(self.to)
        for g, t in zip(self.grads, self.to):
            assert g.dtype in _DTYPES and t.dtype is g.dtype and t.shape == g.shape, "a gradient and where it goes: one shape and type"
            assert g.is_contiguous() and t.is_contiguous() and g.is_cuda and t.device == g.device, "gradients: contiguous, on one GPU"
        self.n = len(self.grads)
        self.host = (Grad * self.n)(*[Grad(g.data_ptr(), t.data_ptr(), g.numel(), 0, _DTYPES[g.dtype], 0) for g, t in zip(self.grads, self.to)])
        rc = lib().bimamba_clip_layout(self.host, self.n)
        if rc != 0:
            raise BimambaError(rc, "bimamba_clip_layout")
        self.dev = torch.frombuffer(bytearray(self.host), dtype=torch.uint8).to(self.grads[0].device) if self.n else None


def bimamba_clip_grads_workspace_bytes(table):
    return int(lib().bimamba_clip_grads_workspace_bytes(table.host, table.n))


def bimamba_clip_grads(table, max_norm, norm, workspace, stream=None, check=True):
    """Enqueue the norm of a GradTable's gradients (norm: float32 [1], or None) and their scaling to at most max_norm."""
    return _checked((_calls_module or _calls()).clip_grads(table.host, table.dev, max_norm, norm, workspace, _stream(stream)), "bimamba_clip_grads", check)


# ---- the block of a gated linear recurrence: the recurrence, the norm of its gated output, dropout into the residual stream ----

RECURRENCE_KEEP = 64   # steps between two kept states
_GATES = {"log": 0, "sigmoid": 1}
_ACTS = {"none": 0, "silu": 1, "gate_before": 2, "gate_after": 3}


def make_recurrence_desc(batch, seqlen, d_inner, io="bf16", gate="sigmoid", reverse=0):
    """gate: "log" (a = exp(min(g, 0)), u = x) or "sigmoid" (a = sigmoid(g + bias), u = (1 - a) x); reverse: from the last token to the first."""
    return RecurrenceDesc(C.sizeof(RecurrenceDesc), batch, seqlen, d_inner, _NAMES[io], _GATES[gate], int(reverse))


def bimamba_recurrence_workspace_bytes(desc):
    return int(lib().bimamba_recurrence_workspace_bytes(C.byref(desc)))


def bimamba_recurrence(desc, x, g, bias, y, add=None, lengths=None, h_in=None, h_out=None, states=None, workspace=None, stream=None, check=True):
    """Enqueue h = a h + u along the sequence, y = h + add (add may be y).  x, g, add, y [batch, L, d]; bias float32 [d] or None; lengths int64
    [batch] or None; h_in, h_out float32 [batch, d] or None, the state before the first and after the last step; states float32
    [batch, ceil(L / 64), d] or None, that before every 64th (bimamba_recurrence_bwd takes them)."""
    return _checked((_calls_module or _calls()).recurrence(desc, x, g, bias, add, lengths, h_in, y, h_out, states, workspace, _stream(stream)),
                    "bimamba_recurrence", check)


def bimamba_recurrence_bwd_workspace_bytes(desc):
    return int(lib().bimamba_recurrence_bwd_workspace_bytes(C.byref(desc)))


def bimamba_recurrence_bwd(desc, x, g, bias, states, dy, dx, dg, dbias=None, lengths=None, dh_out=None, dh_in=None, workspace=None, stream=None,
                           check=True):
    """Enqueue the gradients of bimamba_recurrence (add's is dy).  dbias float32 [d] or None; dh_out, dh_in float32 [batch, d] or None."""
    return _checked((_calls_module or _calls()).recurrence_bwd(desc, x, g, bias, lengths, states, dy, dh_out, dx, dg, dbias, dh_in, workspace,
                                                               _stream(stream)), "bimamba_recurrence_bwd", check)


def make_group_norm_desc(batch, seqlen, d_inner, groups, io="bf16", act="none", centred=0, eps=1e-5):
    """act: "none", "silu", "gate_before" (the norm of x * SiLU(z)) or "gate_after" (times SiLU(z)); centred: the mean is taken off."""
    return GroupNormDesc(C.sizeof(GroupNormDesc), batch, seqlen, d_inner, groups, _NAMES[io], _ACTS[act], int(centred), eps)


def bimamba_group_norm(desc, x, z, weight, bias, y, mean=None, rstd=None, stream=None, check=True):
    """Enqueue the norm of every token's groups of channels.  z: the gate's input, or None without one; weight, bias float32 [d] or None;
    mean (centred only), rstd float32 [batch, L, groups] or None (bimamba_group_norm_bwd takes them)."""
    return _checked((_calls_module or _calls()).group_norm(desc, x, z, weight, bias, y, mean, rstd, _stream(stream)), "bimamba_group_norm", check)


def bimamba_group_norm_bwd_workspace_bytes(desc):
    return int(lib().bimamba_group_norm_bwd_workspace_bytes(C.byref(desc)))


def bimamba_group_norm_bwd(desc, x, z, weight, bias, mean, rstd, dy, dx, dz, dweight, dbias, workspace, stream=None, check=True):
    """Enqueue the gradients of bimamba_group_norm.  dz: None without a gate; dweight, dbias float32 [d] or None; overwritten."""
    return _checked((_calls_module or _calls()).group_norm_bwd(desc, x, z, weight, bias, mean, rstd, dy, dx, dz, dweight, dbias, workspace,
                                                               _stream(stream)), "bimamba_group_norm_bwd", check)


def make_dropout_desc(batch, seqlen, d_model, io="bf16", p=0.1, site=0):
    return DropoutDesc(C.sizeof(DropoutDesc), batch, seqlen, d_model, _NAMES[io], site, p)


def bimamba_dropout_add(desc, key, x, gate, residual, out, stream=None, check=True):
    """Enqueue out = residual + gate * dropout(x).  key: int64 [2], seed and offset; gate: float32 [d], or [batch, d] with a vector for each
    batch element, or None; residual: None, or like x; it may be out."""
    return _checked((_calls_module or _calls()).dropout_add(desc, key, x, gate, residual, out, _stream(stream)), "bimamba_dropout_add", check)


def bimamba_dropout_add_bwd_workspace_bytes(desc, per_batch):
    return int(lib().bimamba_dropout_add_bwd_workspace_bytes(C.byref(desc), int(per_batch)))


def bimamba_dropout_add_bwd(desc, key, x, gate, dout, dx, dgate=None, workspace=None, stream=None, check=True):
    """Enqueue the gradients of bimamba_dropout_add (the residual's is dout; dx may be dout).  dgate: float32 like gate, contiguous, or None
    (x may then be None); without a gate its shape says whether each batch element has a vector of its own."""
    return _checked((_calls_module or _calls()).dropout_add_bwd(desc, key, x, gate, dout, dx, dgate, workspace, _stream(stream)),
                    "bimamba_dropout_add_bwd", check)


# ---- conveniences used by tests and the benchmark (allocation through torch, no arithmetic) ----

def io_dtype(cfg):
    return torch.bfloat16 if cfg["io"] == "bf16" else torch.float32


def to_device(tensors, cfg=None, device="cuda"):
    """Upload a dict of CPU float32 tensors; activations are cast to the config's I/O dtype (exact: values were
    rounded to it by the generator), parameters stay float32."""
    out = {}
    for k, v in tensors.items():
        if v is None:
            out[k] = None
        elif cfg is not None and k in ("x", "z", "dt", "B", "C"):
            out[k] = v.to(device=device, dtype=io_dtype(cfg)).contiguous()
        else:
            out[k] = v.to(device=device, dtype=torch.float32).contiguous()
    return out


def alloc_out(cfg, device="cuda", seqlen=None):
    L = cfg["seqlen"] if seqlen is None else seqlen
    width = cfg["d_inner"] * (2 if cfg["combine"] == COMBINE_SEPARATE else 1)
    return torch.empty(cfg["batch"], L, width, dtype=io_dtype(cfg), device=device)


def alloc_workspace(desc, block_variant=0, device="cuda"):
    n = bimamba_workspace_bytes(desc, block_variant)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=device)
