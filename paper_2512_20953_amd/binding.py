"""ctypes binding of include/ah_stage.h, ah_cost.h and ah_ops.h: argument marshalling only.

Device memory and streams come from PyTorch (ROCm); tensors are passed as raw
device pointers.  The library must have been built (paper_2512_20953_amd/build.py
or __graft_entry__.build()); a missing library is an ImportError-level failure,
there is no fallback path.
"""
import ctypes as C
import itertools
import os

HERE = os.path.dirname(os.path.abspath(__file__))
AH_ARCH_GPT, AH_ARCH_LLAMA, AH_ARCH_BERT = 0, 1, 2
_ARCH = {"gpt": AH_ARCH_GPT, "llama": AH_ARCH_LLAMA, "bert": AH_ARCH_BERT}
PARAM_INDEX = {"ln1_g": 0, "ln1_b": 1, "wqkv": 2, "bqkv": 3, "wo": 4, "bo": 5,
               "ln2_g": 6, "ln2_b": 7, "w1": 8, "b1": 9, "w2": 10, "b2": 11, "qn_g": 12, "kn_g": 13}
# names the layer's tensors go by elsewhere (LLaMA: fused gate|up and down)
PARAM_ALIASES = {"wgu": "w1", "wd": "w2"}


def _clamped(n):
    """A number for an int32 field, which would keep the lowest 32 bits of a larger one: a window, say, above that stands for all positions, what is negative is refused."""
    return max(-1, min(n, (1 << 31) - 1))


class AhError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("ah status %d: %s" % (status, msg))
        self.status = status


class StageConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("arch", C.c_int32), ("n_layers", C.c_int32), ("hidden", C.c_int32),
                ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn_hidden", C.c_int32), ("tp_degree", C.c_int32),
                ("tp_rank", C.c_int32), ("seq_len", C.c_int32), ("microbatch_size", C.c_int32),
                ("n_microbatches", C.c_int32), ("max_in_flight", C.c_int32), ("recompute", C.c_int32),
                ("wgrad_group", C.c_int32), ("norm_eps", C.c_float), ("rope_base", C.c_float), ("residual_fp32", C.c_int32),
                ("attn_window", C.c_int32), ("attn_sinks", C.c_int32), ("qk_norm", C.c_int32)]

    @classmethod
    def make(cls, arch="gpt", n_layers=1, hidden=256, n_heads=4, head_dim=64, ffn=1024, tp=1, tp_rank=0, seq=128, mb=1,
             n_mb=1, max_in_flight=1, recompute=0, wgrad_group=0, norm_eps=0.0, rope_base=0.0, residual_fp32=0,
             attn_window=0, attn_sinks=0, qk_norm=0):
        return cls(C.sizeof(cls), _ARCH[arch], n_layers, hidden, n_heads, head_dim,
                   ffn, tp, tp_rank, seq, mb, n_mb, max_in_flight, recompute, wgrad_group, norm_eps, rope_base, residual_fp32,
                   _clamped(attn_window), _clamped(attn_sinks), qk_norm)


class _Sizes(C.Structure):
    _fields_ = [("param_elems", C.c_uint64), ("param_bytes", C.c_uint64), ("grad_bytes", C.c_uint64),
                ("activation_bytes_per_slot", C.c_uint64), ("activation_bytes_per_layer_per_slot", C.c_uint64),
                ("workspace_bytes", C.c_uint64)]


class _Buffers(C.Structure):
    _fields_ = [("params", C.c_void_p), ("grads", C.c_void_p), ("activations", C.c_void_p), ("workspace", C.c_void_p)]


class _Profile(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_layers", C.c_int32), ("fwd_ms", C.POINTER(C.c_float)),
                ("bwd_ms", C.POINTER(C.c_float)), ("stage_fwd_ms", C.c_float), ("stage_bwd_ms", C.c_float),
                ("iteration_ms", C.c_float), ("peak_activation_bytes", C.c_uint64),
                ("activation_bytes_per_layer_per_slot", C.c_uint64), ("param_bytes", C.c_uint64), ("grad_bytes", C.c_uint64)]


class _TraceEntry(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("launches", C.c_int64), ("total_ms", C.c_double),
                ("flops_per_launch", C.c_double), ("bytes_per_launch", C.c_double)]


class _AdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("m_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("master", C.c_void_p), ("n", C.c_uint64), ("weight_decay", C.c_float), ("reserved", C.c_uint32)]


class _AdamWConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("param_type", C.c_int32), ("grad_type", C.c_int32), ("state_bits", C.c_int32),
                ("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64),
                ("lr_dev", C.c_void_p), ("step_dev", C.c_void_p), ("grad_norm", C.c_void_p), ("seed", C.c_uint32), ("reserved", C.c_uint32)]


class _WindowConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_seq", C.c_int32), ("seq_len", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("sinks", C.c_int32), ("rows", C.c_int64), ("offsets", C.c_void_p)] + [
                (n, C.c_int64) for n in ("ld_q", "ld_k", "ld_v", "ld_o", "ld_do", "ld_dq", "ld_dk", "ld_dv")]


class _QkNormConfig(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("rows", C.c_int32), ("seq_len", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("n_pos", C.c_int32), ("eps", C.c_float), ("ld_x", C.c_int64), ("ld_y", C.c_int64), ("ld_dx", C.c_int64),
                ("gain_q", C.c_void_p), ("gain_k", C.c_void_p), ("cos_sin", C.c_void_p), ("positions", C.c_void_p)]


def library_path():
    return os.path.join(HERE, "libahstage.so")


def _load():
    path = library_path()
    if not os.path.exists(path):
        raise ImportError("libahstage.so is not built: run `python -m paper_2512_20953_amd.build` "
                          "(or __graft_entry__.build()); there is no fallback implementation")
    # PyTorch ships its own copy of the HIP runtime and must be loaded first: the dynamic linker
    # then resolves this library's runtime dependency to that same copy.  Loaded the other way
    # round the process ends up with two runtimes, and the second one finds no device.
    import torch  # noqa: F401
    L = C.CDLL(path)
    L.ah_last_error.restype = C.c_char_p
    vp, i = C.c_void_p, C.c_int
    L.ah_stage_query_sizes.argtypes = [C.POINTER(StageConfig), C.POINTER(_Sizes)]
    L.ah_stage_create.argtypes = [C.POINTER(StageConfig), C.POINTER(_Buffers), C.POINTER(vp)]
    L.ah_stage_destroy.argtypes = [vp]
    L.ah_stage_param_layout.argtypes = [vp, i, i, C.POINTER(C.c_uint64), C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
    L.ah_stage_forward.argtypes = [vp, i, vp, vp, vp]
    L.ah_stage_backward.argtypes = [vp, i, vp, vp, vp]
    L.ah_stage_backward_streams.argtypes = [vp, C.POINTER(i)]
    L.ah_stage_grads.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_uint64)]
    L.ah_stage_zero_grads.argtypes = [vp, vp]
    L.ah_stage_flush_grads.argtypes = [vp, vp]
    L.ah_stage_profile.argtypes = [vp, i, i, C.POINTER(_Profile)]
    L.ah_stage_trace_begin.argtypes = [vp]
    L.ah_stage_trace_end.argtypes = [vp, C.POINTER(_TraceEntry), i, C.POINTER(i)]
    dp, ip = C.POINTER(C.c_double), C.POINTER(C.c_int)
    L.ah_cost_layers_time.argtypes = [i, dp, i, dp]
    L.ah_cost_pipeline_time.argtypes = [dp, i, i, dp]
    L.ah_cost_iteration_time.argtypes = [dp, ip, i, i, C.c_double, dp]
    L.ah_cost_idle_fractions.argtypes = [dp, i, i, dp, dp]
    L.ah_cost_partition_layers.argtypes = [i, i, dp, dp, C.c_double, C.c_double, ip, ip, dp]
    L.ah_gemm_nn.argtypes = [vp, vp, vp, vp, i, i, i, vp]
    L.ah_gemm_nt.argtypes = [vp, vp, vp, i, i, i, vp]
    L.ah_gemm_nn_swiglu.argtypes = [vp, vp, vp, vp, i, i, i, vp]
    L.ah_gemm_tn.argtypes = [vp, vp, vp, i, i, i, i, vp]
    L.ah_gemm_tn_segmented.argtypes = [C.POINTER(vp), C.POINTER(vp), i, vp, i, i, i, i, vp]
    L.ah_gemm_plan.argtypes = [i, i, i, i, i, C.c_uint64, C.POINTER(C.c_int32)]
    L.ah_attention_fwd.argtypes = [vp, vp, vp, i, i, i, i, i, vp]
    L.ah_attention_bwd.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp]
    L.ah_attention_bwd_static.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, vp]
    L.ah_stage_layer_input.argtypes = [vp, i, i, C.POINTER(vp)]
    tp = C.POINTER(_AdamWTensor)
    L.ah_adamw_step.argtypes = [C.POINTER(_AdamWConfig), tp, i, vp]
    L.ah_grad_norm.argtypes = [tp, i, i, C.c_double, vp, vp, vp]
    L.ah_grad_norm_workspace.argtypes = [i, C.POINTER(C.c_uint64)]
    wc, qc = C.POINTER(_WindowConfig), C.POINTER(_QkNormConfig)
    L.ah_attention_window_fwd.argtypes = [wc] + [vp] * 6
    L.ah_attention_window_bwd.argtypes = [wc] + [vp] * 11
    L.ah_attention_window_bwd_workspace.argtypes = [wc, C.POINTER(C.c_uint64)]
    L.ah_qk_norm_rope_fwd.argtypes = [qc, vp, vp, vp]
    L.ah_qk_norm_rope_bwd.argtypes = [qc, vp, vp, vp, vp, vp, i, vp, vp]
    L.ah_qk_norm_rope_bwd_workspace.argtypes = [qc, C.POINTER(C.c_uint64)]
    L.ah_rope_table.argtypes = [vp, i, i, C.c_double, vp]
    L.ah_adamw_state_values.argtypes = [tp, i, C.POINTER(vp), C.POINTER(vp), vp]
    return L


lib = _load()


def _check(rc):
    if rc != 0:
        raise AhError(rc, lib.ah_last_error().decode())


# The smallest calls last as long as the host needs for them (three products of 256 x 256 x 1024: 13.4 us in a graph; one
# call 11 us, of which 3.9 in the library and 2.9 for an object of the current stream): addresses go over as plain integers,
# which the argument types above make pointers, and the current stream as its handle.  The three products 31.7 -> 22.5 us.
def _ptr(t):
    return t.data_ptr() if t is not None else None


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    if not torch.cuda.is_initialized():
        torch.cuda.current_stream()      # initialises the device state, or raises as it does without a GPU
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def query_sizes(cfg):
    s = _Sizes()
    _check(lib.ah_stage_query_sizes(C.byref(cfg), C.byref(s)))
    return {k: int(getattr(s, k)) for k, _ in _Sizes._fields_}


class Stage:
    """A stage over torch-allocated device buffers."""

    def __init__(self, cfg, device="cuda:0"):
        import torch
        self.cfg = cfg
        self.sizes = query_sizes(cfg)
        self.device = torch.device(device)
        self.params = torch.zeros(self.sizes["param_elems"], dtype=torch.bfloat16, device=self.device)
        self.grads = torch.zeros(self.sizes["param_elems"], dtype=torch.float32, device=self.device)
        self.activations = torch.empty(self.sizes["activation_bytes_per_slot"] * cfg.max_in_flight, dtype=torch.uint8,
                                       device=self.device)
        self.workspace = torch.empty(self.sizes["workspace_bytes"], dtype=torch.uint8, device=self.device)
        bufs = _Buffers(self.params.data_ptr(), self.grads.data_ptr(), self.activations.data_ptr(), self.workspace.data_ptr())
        h = C.c_void_p()
        _check(lib.ah_stage_create(C.byref(cfg), C.byref(bufs), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None) and lib is not None:   # at interpreter shutdown the module globals may be gone already
            lib.ah_stage_destroy(self._h)
            self._h = None

    __del__ = close

    def param_layout(self, layer, name):
        which = PARAM_INDEX[PARAM_ALIASES.get(name, name)]
        off, r, c = C.c_uint64(), C.c_int32(), C.c_int32()
        _check(lib.ah_stage_param_layout(self._h, layer, which, C.byref(off), C.byref(r), C.byref(c)))
        return off.value, r.value, c.value

    def param_view(self, layer, name):
        off, r, c = self.param_layout(layer, name)
        v = self.params[off:off + r * c]
        return v.view(r, c) if r > 1 else v

    def grad_view(self, layer, name):
        off, r, c = self.param_layout(layer, name)
        v = self.grads[off:off + r * c]
        return v.view(r, c) if r > 1 else v

    def layer_input(self, slot, layer):
        """[T, hidden] view (bf16, or fp32 with residual_fp32) of the input the stage keeps for `layer` of the micro-batch in `slot`."""
        import torch
        p = C.c_void_p()
        _check(lib.ah_stage_layer_input(self._h, slot, layer, C.byref(p)))
        T, h = self.cfg.microbatch_size * self.cfg.seq_len, self.cfg.hidden
        dt, nb = (torch.float32, 4) if self.cfg.residual_fp32 else (torch.bfloat16, 2)
        off = p.value - self.activations.data_ptr()
        assert 0 <= off and off + nb * T * h <= self.activations.numel()
        return self.activations[off:off + nb * T * h].view(dt).view(T, h)

    def forward(self, slot, x, y, stream=None):
        _check(lib.ah_stage_forward(self._h, slot, _ptr(x), _ptr(y), _stream(stream)))

    def backward(self, slot, dy, dx, stream=None):
        _check(lib.ah_stage_backward(self._h, slot, _ptr(dy), _ptr(dx), _stream(stream)))

    def zero_grads(self, stream=None):
        _check(lib.ah_stage_zero_grads(self._h, _stream(stream)))

    def flush_grads(self, stream=None):
        _check(lib.ah_stage_flush_grads(self._h, _stream(stream)))

    def backward_streams(self):
        n = C.c_int()
        _check(lib.ah_stage_backward_streams(self._h, C.byref(n)))
        return n.value

    def adamw(self, weight_decay=0.1, **options):
        """An AdamW over the stage's parameters and gradients (state_bits, master, betas, eps as there); weight_decay acts on the matrices, not on
        biases, gains and offsets.  Its step goes behind the last backward (or flush_grads) of an iteration, on the same stream."""
        params, grads, decay = [], [], []
        for layer in range(self.cfg.n_layers):
            for which in PARAM_INDEX.values():
                off, r, c = C.c_uint64(), C.c_int32(), C.c_int32()
                if lib.ah_stage_param_layout(self._h, layer, which, C.byref(off), C.byref(r), C.byref(c)) == 0:    # (not every architecture has each)
                    at = slice(off.value, off.value + r.value * c.value)
                    params.append(self.params[at])
                    grads.append(self.grads[at])
                    decay.append(weight_decay if r.value > 1 else 0.0)
        return AdamW(params, grads, weight_decay=decay, **options)

    def grads_ptr(self):
        p, n = C.c_void_p(), C.c_uint64()
        _check(lib.ah_stage_grads(self._h, C.byref(p), C.byref(n)))
        return p.value, n.value

    def trace_begin(self):
        _check(lib.ah_stage_trace_begin(self._h))

    def trace_end(self):
        arr = (_TraceEntry * 32)()
        n = C.c_int()
        _check(lib.ah_stage_trace_end(self._h, arr, 32, C.byref(n)))
        return [{"name": arr[k].name.decode(), "launches": int(arr[k].launches), "total_ms": arr[k].total_ms,
                 "flops_per_launch": arr[k].flops_per_launch, "bytes_per_launch": arr[k].bytes_per_launch}
                for k in range(n.value)]

    def profile(self, warmup=2, iters=5):
        L = self.cfg.n_layers
        f, b = (C.c_float * L)(), (C.c_float * L)()
        p = _Profile(C.sizeof(_Profile), L, f, b)
        _check(lib.ah_stage_profile(self._h, warmup, iters, C.byref(p)))
        return {"fwd_ms": list(f), "bwd_ms": list(b), "stage_fwd_ms": p.stage_fwd_ms, "stage_bwd_ms": p.stage_bwd_ms,
                "iteration_ms": p.iteration_ms, "peak_activation_bytes": int(p.peak_activation_bytes),
                "activation_bytes_per_layer_per_slot": int(p.activation_bytes_per_layer_per_slot),
                "param_bytes": int(p.param_bytes), "grad_bytes": int(p.grad_bytes)}


def gemm_nn(A, B, bias, Cout, stream=None):
    M, K = A.shape
    _check(lib.ah_gemm_nn(_ptr(A), _ptr(B), _ptr(bias), _ptr(Cout), M, B.shape[1], K, _stream(stream)))


def gemm_nn_swiglu(A, B, U, Mout, stream=None):
    M, K = A.shape
    _check(lib.ah_gemm_nn_swiglu(_ptr(A), _ptr(B), _ptr(U), _ptr(Mout), M, B.shape[1] // 2, K, _stream(stream)))


def gemm_nt(A, B, Cout, stream=None):
    M, K = A.shape
    _check(lib.ah_gemm_nt(_ptr(A), _ptr(B), _ptr(Cout), M, B.shape[0], K, _stream(stream)))


def gemm_tn(A, B, Cout, beta, stream=None):
    K, M = A.shape
    _check(lib.ah_gemm_tn(_ptr(A), _ptr(B), _ptr(Cout), M, B.shape[1], K, int(beta), _stream(stream)))


def gemm_tn_segmented(A_list, B_list, Cout, beta, stream=None):
    n = len(A_list)
    seg_k, M = A_list[0].shape
    pa = (C.c_void_p * n)(*[a.data_ptr() for a in A_list])
    pb = (C.c_void_p * n)(*[b.data_ptr() for b in B_list])
    _check(lib.ah_gemm_tn_segmented(pa, pb, n, _ptr(Cout), M, B_list[0].shape[1], seg_k, int(beta), _stream(stream)))


def gemm_plan(layout, M, N, K, n_seg=1, part_floats=0):
    """How the library covers a product ("nn", "nt", "tn"): (parts of the k axis between blocks,
    [(columns, rows of a tile, columns of a tile, waves along k, tile rows walked together) per launch])."""
    o = (C.c_int32 * 12)()
    _check(lib.ah_gemm_plan(("nn", "nt", "tn").index(layout), M, N, K, n_seg, part_floats, o))
    return o[1], [tuple(o[2 + 5 * l:7 + 5 * l]) for l in range(o[0])]


def attention_fwd(qkv, o, lse, B, S, nh, d, causal=True, stream=None):
    _check(lib.ah_attention_fwd(_ptr(qkv), _ptr(o), _ptr(lse), B, S, nh, d, int(bool(causal)), _stream(stream)))


def attention_bwd(qkv, o, lse, d_o, dqkv, delta, B, S, nh, d, causal=True, stream=None):
    _check(lib.ah_attention_bwd(_ptr(qkv), _ptr(o), _ptr(lse), _ptr(d_o), _ptr(dqkv), _ptr(delta), B, S, nh, d, int(bool(causal)), _stream(stream)))


ATTENTION_STATIC_MAX_ROWS = 262144


def attention_bwd_static(qkv, o, lse, d_o, dqkv, B, S, nh, d, causal=True, stream=None):
    _check(lib.ah_attention_bwd_static(_ptr(qkv), _ptr(o), _ptr(lse), _ptr(d_o), _ptr(dqkv), B, S, nh, d, int(bool(causal)), _stream(stream)))


# ---- cost model (include/ah_cost.h): host arrays in, numbers out
def _darr(v):
    return (C.c_double * len(v))(*[float(x) for x in v])


def cost_layers_time(n, t_pow2):
    out = C.c_double()
    _check(lib.ah_cost_layers_time(int(n), _darr(t_pow2), len(t_pow2), C.byref(out)))
    return out.value


def cost_pipeline_time(t_stage, K):
    out = C.c_double()
    _check(lib.ah_cost_pipeline_time(_darr(t_stage), len(t_stage), int(K), C.byref(out)))
    return out.value


def cost_iteration_time(groups, K, t_sync):
    flat = [t for g in groups for t in g]
    stages = (C.c_int * len(groups))(*[len(g) for g in groups])
    out = C.c_double()
    _check(lib.ah_cost_iteration_time(_darr(flat), stages, len(groups), int(K), float(t_sync), C.byref(out)))
    return out.value


def cost_idle_fractions(t_stage, K):
    idle = (C.c_double * len(t_stage))()
    mean = C.c_double()
    _check(lib.ah_cost_idle_fractions(_darr(t_stage), len(t_stage), int(K), idle, C.byref(mean)))
    return list(idle), mean.value


def cost_partition_layers(n_layers, t_layer, mem_bytes, fixed_per_layer, act_per_layer, in_flight):
    P = len(t_layer)
    l = (C.c_int * P)()
    worst = C.c_double()
    _check(lib.ah_cost_partition_layers(P, int(n_layers), _darr(t_layer), _darr(mem_bytes), float(fixed_per_layer),
                                        float(act_per_layer), (C.c_int * P)(*[int(f) for f in in_flight]), l, C.byref(worst)))
    return list(l), worst.value


# ---- operators beside the stage (include/ah_ops.h).  What the library cannot see is checked here: that a tensor lies on the current device, its
# type, its size, and that its rows are as the call takes them.  The smallest calls last as long as these checks: each looks at a tensor's
# attributes once.
import torch  # noqa: E402  (loaded above, before the library)

_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_WINDOW_SIZE, _QK_SIZE = C.sizeof(_WindowConfig), C.sizeof(_QkNormConfig)


def _refuse(msg, *args):
    raise AhError(1, msg % args)


_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else lambda: -1   # (-1 without a GPU, as a host tensor's)


def _on_device(what, t):
    at = t.get_device()
    if at < 0 or at != _current_device():
        _refuse("%s is not in device memory" if at < 0 else "%s lies on device " + str(at) + ", which is not the current one", what)


def _dense(what, t, dtype, n=None):
    """Address of a contiguous tensor of n elements."""
    device = t.get_device()
    if device < 0 or device != _current_device():
        _on_device(what, t)
    if t.dtype is not dtype or not t.is_contiguous() or (n is not None and t.numel() != n):
        _refuse("%s: %s of shape %s (contiguous: %s), wanted a contiguous tensor of %s%s", what, t.dtype, tuple(t.shape), t.is_contiguous(), dtype,
                "" if n is None else " with %d elements" % n)
    return t.data_ptr()


def _rows(what, t, rows, cols):
    """(address, columns from row to row) of a bf16 matrix whose rows are dense and 16-byte aligned, at any distance from each other."""
    device = t.get_device()
    if device < 0 or device != _current_device():
        _on_device(what, t)
    shape, stride, at = t.shape, t.stride(), t.data_ptr()
    if t.dtype is not _BF16 or len(shape) != 2 or shape[1] != cols or shape[0] != rows:
        _refuse("%s: %s of shape %s, wanted bf16 [%d, %d]", what, t.dtype, tuple(shape), rows, cols)
    ld = stride[0] if rows > 1 else cols
    if stride[1] != 1 or ld < cols or ld & 7 or at & 15:
        _refuse("%s: rows must be dense, 16-byte aligned and a multiple of 8 columns apart (strides %s)", what, stride)
    return at, ld


def _window_config(n_seq, seq_len, nh, nh_kv, d, window, sinks):
    sizes = n_seq, seq_len, nh, nh_kv, d, window, sinks
    if (n_seq | seq_len | nh | nh_kv | d | window | sinks) >> 31:    # one of them does not fit
        sizes = map(_clamped, sizes)
    return _WindowConfig(_WINDOW_SIZE, *sizes)


def _window_args(c, q, k, v, o, lse, offsets):
    wq, wk = c.n_heads * c.head_dim, c.n_kv_heads * c.head_dim
    c.rows = T = q.shape[0]
    pq, c.ld_q = _rows("q", q, T, wq)
    pk, c.ld_k = _rows("k", k, T, wk)
    pv, c.ld_v = _rows("v", v, T, wk)
    po, c.ld_o = _rows("o", o, T, wq)
    if offsets is not None:
        c.offsets = _dense("offsets", offsets, _I32, c.n_seq + 1)
    elif T != c.n_seq * c.seq_len:
        _refuse("attention_window: %d rows for %d sequences of %d", T, c.n_seq, c.seq_len)
    return pq, pk, pv, po, _dense("lse", lse, _F32, c.n_seq * c.n_heads * c.seq_len)


def attention_window_fwd(q, k, v, o, lse, n_seq, seq_len, nh, nh_kv, d, window, sinks=0, offsets=None, stream=None):
    """Causal attention of which a query sees the last `window` positions and the first `sinks` (ah_attention_window_fwd).  q, o: [T, nh * d],
    k, v: [T, nh_kv * d], rows at any distance (columns of a packed projection, for one); lse: fp32 [n_seq, nh, seq_len].
    offsets: int32 [n_seq + 1], where packed sequences of at most seq_len rows begin and the last one ends."""
    c = _window_config(n_seq, seq_len, nh, nh_kv, d, window, sinks)
    at = _window_args(c, q, k, v, o, lse, offsets)
    _check(lib.ah_attention_window_fwd(c, *at, _stream(stream)))


def attention_window_bwd_workspace(n_seq, seq_len, nh, nh_kv, d, window, sinks=0):
    """Bytes of scratch memory that attention_window_bwd takes."""
    n = C.c_uint64()
    _check(lib.ah_attention_window_bwd_workspace(_window_config(n_seq, seq_len, nh, nh_kv, d, window, sinks), n))
    return n.value


def attention_window_bwd(q, k, v, o, lse, d_o, dq, dk, dv, workspace, n_seq, seq_len, nh, nh_kv, d, window, sinks=0, offsets=None, stream=None):
    """dq, dk, dv of attention_window_fwd from its inputs, its results and d_o.  workspace: uint8, attention_window_bwd_workspace(...) bytes."""
    c = _window_config(n_seq, seq_len, nh, nh_kv, d, window, sinks)
    at = _window_args(c, q, k, v, o, lse, offsets)
    wq, wk, T = nh * d, nh_kv * d, c.rows
    pdo, c.ld_do = _rows("d_o", d_o, T, wq)
    pdq, c.ld_dq = _rows("dq", dq, T, wq)
    pdk, c.ld_dk = _rows("dk", dk, T, wk)
    pdv, c.ld_dv = _rows("dv", dv, T, wk)
    work, need = _dense("workspace", workspace, _U8), C.c_uint64()
    _check(lib.ah_attention_window_bwd_workspace(c, need))
    if workspace.numel() < need.value:
        _refuse("attention_window_bwd: the workspace holds %d bytes, too few", workspace.numel())
    _check(lib.ah_attention_window_bwd(c, *at, pdo, pdq, pdk, pdv, work, _stream(stream)))


def rope_table(cos_sin, d, base=10000.0, stream=None):
    """Fills cos_sin, fp32 [n_pos, d / 2, 2], with the angles of the stage's rotary embedding."""
    if cos_sin.dim() != 3 or cos_sin.shape[1:] != (d // 2, 2):
        _refuse("rope_table: cos_sin is %s, wanted [n_pos, %d, 2]", tuple(cos_sin.shape), d // 2)
    _check(lib.ah_rope_table(_dense("cos_sin", cos_sin, _F32), cos_sin.shape[0], d, float(base), _stream(stream)))


def _qk_args(x, other, gain_q, gain_k, cos_sin, seq_len, nh, nh_kv, d, eps, positions):
    w, T = (nh + nh_kv) * d, x.shape[0]
    px, ld_x = _rows("x", x, T, w)
    po, ld_o = _rows("y or dy", other, T, w)
    pq = _dense("gain_q", gain_q, _BF16, d) if nh else None
    pk = _dense("gain_k", gain_k, _BF16, d) if nh_kv else None
    table = pos = None
    n_pos = 0
    if cos_sin is not None:
        n_pos = cos_sin.shape[0]
        table = _dense("cos_sin", cos_sin, _F32, n_pos * d)
        if cos_sin.shape != (n_pos, d // 2, 2):
            _refuse("cos_sin is %s, wanted [n_pos, %d, 2]", tuple(cos_sin.shape), d // 2)
        if positions is not None:
            pos = _dense("positions", positions, _I32, T)
    if (seq_len | nh | nh_kv | d) >> 31:
        seq_len, nh, nh_kv, d = map(_clamped, (seq_len, nh, nh_kv, d))
    return _QkNormConfig(_QK_SIZE, T, seq_len, nh, nh_kv, d, n_pos, eps, ld_x, ld_o, 0, pq, pk, table, pos), px, po


def qk_norm_rope_fwd(x, gain_q, gain_k, cos_sin, y, seq_len, nh, nh_kv, d, eps=1e-6, positions=None, stream=None):
    """RMS norm of every head with its gain, then the rotation (ah_qk_norm_rope_fwd).  x, y: [T, (nh + nh_kv) * d], query heads then key heads, rows at
    any distance (the first columns of a packed projection); y may be x, its rows as far apart.  cos_sin: see rope_table; None: no rotation.  positions: int32 [T], without them
    row t has position t % seq_len."""
    c, px, py = _qk_args(x, y, gain_q, gain_k, cos_sin, seq_len, nh, nh_kv, d, eps, positions)
    _check(lib.ah_qk_norm_rope_fwd(c, px, py, _stream(stream)))


def qk_norm_rope_bwd_workspace(rows, nh, nh_kv, d):
    """Bytes of scratch memory that qk_norm_rope_bwd takes."""
    n = C.c_uint64()
    _check(lib.ah_qk_norm_rope_bwd_workspace(_QkNormConfig(_QK_SIZE, *map(_clamped, (rows, 0, nh, nh_kv, d))), n))
    return n.value


def qk_norm_rope_bwd(x, gain_q, gain_k, cos_sin, dy, dx, d_gain_q, d_gain_k, workspace, seq_len, nh, nh_kv, d, eps=1e-6, positions=None, beta=0,
                     stream=None):
    """dx from x and dy (dx may be either, row for row), and d_gain = beta * d_gain + the gain's gradient (fp32 [d]).  workspace: uint8, qk_norm_rope_bwd_workspace(...) bytes."""
    if beta not in (0, 1):
        _refuse("qk_norm_rope_bwd: beta %s: 0 or 1", beta)
    c, px, pdy = _qk_args(x, dy, gain_q, gain_k, cos_sin, seq_len, nh, nh_kv, d, eps, positions)
    pdx, c.ld_dx = _rows("dx", dx, c.rows, (nh + nh_kv) * d)
    pgq = _dense("d_gain_q", d_gain_q, _F32, d) if nh else None
    pgk = _dense("d_gain_k", d_gain_k, _F32, d) if nh_kv else None
    work, need = _dense("workspace", workspace, _U8), C.c_uint64()
    _check(lib.ah_qk_norm_rope_bwd_workspace(c, need))
    if workspace.numel() < need.value:
        _refuse("qk_norm_rope_bwd: the workspace holds %d bytes, too few", workspace.numel())
    _check(lib.ah_qk_norm_rope_bwd(c, px, pdy, pdx, pgq, pgk, int(beta), work, _stream(stream)))


def _apart(written, read):
    """Whether no two of the (begin, end) spans in `written` overlap, nor one of them and one of `read`."""
    last_written = last = 0                    # where those that begin before end
    for begin, end, writes in sorted([(b, e, True) for b, e in written if b < e] + [(b, e, False) for b, e in read if b < e]):
        if begin < (last if writes else last_written):
            return False
        last = max(last, end)
        if writes:
            last_written = max(last_written, end)
    return True


class AdamW:
    """AdamW over a list of tensors (ah_adamw_step): bf16 or fp32 parameters with fp32 or bf16 gradients.

    state_bits 32: moments in fp32.  8: one byte an element and a scale for each 32.
    master: True keeps bf16 parameters in fp32 too (the step updates those and rounds them into the parameters), starting from
    the parameters' values; or a list of such tensors.
    weight_decay: one number, or one for each tensor.
    m, v (m_scale, v_scale): lists of state tensors to go on from; without them zeroed ones are made.
    Tensors that a step writes overlap no other.  The object keeps the tensors that it was given, and its scratch memory serves one grad_norm at a time.
    It makes its own on the stream that is torch's current one at its construction: steps on other streams come behind that."""

    def __init__(self, params, grads, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.0, state_bits=32, master=None, m=None, v=None,
                 m_scale=None, v_scale=None):
        params, grads = list(params), list(grads)
        n = len(params)
        if n == 0 or len(grads) != n:
            _refuse("AdamW: %d parameters and %d gradients", n, len(grads))
        if state_bits not in (8, 32):
            raise AhError(5, "AdamW: state_bits %s: 32 or 8" % state_bits)
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        if len(decay) != n:
            _refuse("AdamW: %d weight decays for %d parameters", len(decay), n)
        if state_bits == 8 and ((m is None) != (m_scale is None) or (v is None) != (v_scale is None)):
            _refuse("AdamW: states in 8 bits are nothing without their scales: m goes with m_scale, v with v_scale")
        p_type, g_type = params[0].dtype, grads[0].dtype
        if p_type not in (_BF16, _F32) or g_type not in (_BF16, _F32):
            _refuse("AdamW: parameters of %s and gradients of %s, wanted bf16 or fp32", p_type, g_type)
        self._device = params[0].device
        sizes = [p.numel() for p in params]
        for k in range(n):
            _dense("AdamW: parameter %d" % k, params[k], p_type)
            _dense("AdamW: gradient %d" % k, grads[k], g_type, sizes[k])
        wide = _F32 if state_bits == 32 else _U8

        def state(what, given, dtype, per):
            counts = [(x + per - 1) // per for x in sizes]
            if given is None:                # one buffer, each tensor's part from a multiple of 64 elements on
                step = 64 // per
                room = [(c + step - 1) // step * step for c in counts]
                flat = torch.zeros(sum(room), dtype=dtype, device=self._device)
                ends = list(itertools.accumulate(room))
                return [flat[e - r:e - r + c] for e, r, c in zip(ends, room, counts)]
            given = list(given)
            if len(given) != n:
                _refuse("AdamW: %d tensors of %s for %d parameters", len(given), what, n)
            for k in range(n):
                _dense("AdamW: %s %d" % (what, k), given[k], dtype, counts[k])
            return given

        self.params, self.grads, self._sizes = params, grads, sizes
        self.m, self.v = state("m", m, wide, 1), state("v", v, wide, 1)
        self.m_scale = state("m_scale", m_scale, _U8, 32) if state_bits == 8 else None
        self.v_scale = state("v_scale", v_scale, _U8, 32) if state_bits == 8 else None
        self.master = None
        if master is not None and master is not False:
            if p_type != _BF16:
                _refuse("AdamW: master copies go with bf16 parameters")
            self.master = state("master", None if master is True else master, _F32, 1)
            if master is True:
                for a, b in zip(self.master, params):
                    a.copy_(b.detach().reshape(-1))    # (the copies are no part of a graph of b's)
        spans = lambda tensors: [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in tensors]  # noqa: E731
        if not _apart(spans([*params, *self.m, *self.v, *(self.m_scale or ()), *(self.v_scale or ()), *(self.master or ())]), spans(grads)):
            _refuse("AdamW: parameters, states, copies and gradients overlap (gradients alone may)")
        self._list = (_AdamWTensor * n)()
        for k in range(n):
            e = self._list[k]
            e.param, e.grad, e.m, e.v, e.n = params[k].data_ptr(), grads[k].data_ptr(), self.m[k].data_ptr(), self.v[k].data_ptr(), sizes[k]
            if state_bits == 8:
                e.m_scale, e.v_scale = self.m_scale[k].data_ptr(), self.v_scale[k].data_ptr()
            if self.master is not None:
                e.master = self.master[k].data_ptr()
            e.weight_decay = float(decay[k])
        self._cfg = _AdamWConfig(struct_size=C.sizeof(_AdamWConfig), param_type=int(p_type == _F32), grad_type=int(g_type == _F32),
                                 state_bits=state_bits, beta1=float(betas[0]), beta2=float(betas[1]), eps=float(eps))
        need = C.c_uint64()
        _check(lib.ah_grad_norm_workspace(n, C.byref(need)))
        self._norm_work = torch.empty(need.value, dtype=_U8, device=self._device)
        self._norm = torch.zeros(2, device=self._device)

    def grad_norm(self, max_norm=0.0, stream=None):
        """Device tensor [norm of all gradients, factor that brings it down to max_norm] (the object's own: the next call rewrites it).  0: no limit."""
        _on_device("AdamW: parameters", self._norm)
        _check(lib.ah_grad_norm(self._list, len(self._list), self._cfg.grad_type, float(max_norm), self._norm.data_ptr(), self._norm_work.data_ptr(), _stream(stream)))
        return self._norm

    def step(self, lr, step, grad_norm=None, seed=None, stream=None):
        """One step, number `step` (from 1 on).  lr: a number, or an fp32 tensor of one element on the device; step: likewise, int32 (a captured
        step reads them anew when it is replayed; one with 8-bit states needs the step's number there).  grad_norm: what grad_norm() gave: gradients are
        multiplied by its factor, and where that is NaN nothing changes.  seed: of the random rounding of 8-bit states, which has to differ from step to step.
        None: it goes by the step's number.  A number beside a `step` on the device: by their sum.  A number beside a number: by that seed alone, and
        the caller gives another one for every step."""
        c = self._cfg
        _on_device("AdamW: parameters", self._norm)
        c.lr_dev = c.step_dev = c.grad_norm = None
        if isinstance(lr, torch.Tensor):
            c.lr, c.lr_dev = 0.0, _dense("AdamW.step: lr", lr, _F32, 1)
        else:
            c.lr = lr
        if isinstance(step, torch.Tensor):
            c.step, c.step_dev = 1, _dense("AdamW.step: step", step, _I32, 1)
        else:
            c.step = step
        if grad_norm is not None:
            c.grad_norm = _dense("AdamW.step: grad_norm", grad_norm, _F32, 2)
        # (the library adds the step's number)
        c.seed = 0 if seed is None else (seed if c.step_dev else seed - step) & 0xFFFFFFFF
        _check(lib.ah_adamw_step(c, self._list, len(self._list), _stream(stream)))

    def state_values(self, m_out, v_out, stream=None):
        """What 8-bit states stand for, into two lists of bf16 tensors (which hold them exactly, and do not overlap)."""
        if self.m_scale is None:
            _refuse("AdamW.state_values: the states are in fp32 (m, v)")
        n, device = len(self._list), self._norm.get_device()
        _on_device("AdamW: parameters", self._norm)
        both = [*m_out, *v_out]
        if len(m_out) != n or [t.numel() for t in both] != self._sizes * 2:
            _refuse("AdamW.state_values: the outputs are not of the parameters' sizes")
        for t in both:
            if t.dtype is not _BF16 or t.get_device() != device or not t.is_contiguous():
                _refuse("AdamW.state_values: outputs are contiguous bf16 tensors on the parameters' device")
        at = [t.data_ptr() for t in both]
        _check(lib.ah_adamw_state_values(self._list, n, (C.c_void_p * n)(*at[:n]), (C.c_void_p * n)(*at[n:]), _stream(stream)))
