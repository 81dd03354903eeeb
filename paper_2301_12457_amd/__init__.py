"""Python binding of the gfx950 EvoX hot path (libevox.so, C ABI in include/evox.h).

Argument marshalling only: torch supplies device memory and the HIP stream,
every step of the path runs in the library's kernels.  Importing this module
does not touch the GPU; the first call that needs the library loads it and
raises if it has not been built (python paper_2301_12457_amd/build.py).
"""
import ctypes
import math
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libevox.so")

SPHERE, ACKLEY, RASTRIGIN, GRIEWANK, ROSENBROCK, SCHWEFEL = range(6)
FN_IDS = {"sphere": SPHERE, "ackley": ACKLEY, "rastrigin": RASTRIGIN, "griewank": GRIEWANK,
          "rosenbrock": ROSENBROCK, "schwefel": SCHWEFEL}
PSO, CSO, DE, ES, PGPE, MAES, NSGA2 = 0, 1, 2, 3, 4, 5, 6
OK, EINVAL, EHIP, ENOSPC, EALIGN = 0, -1, -2, -3, -4
MAX_D = 32768
F32, BF16, F16 = range(3)
ACT_NONE, ACT_RELU, ACT_TANH, ACT_GELU, ACT_SILU = range(5)
GATE_CHOSEN, GATE_ALL = range(2)
GATE_MAX_K, ADAM_BLOCK, ADAM_CLOCK = 32, 256, 528
KERNEL_ROWS, KERNEL_NARROW, KERNEL_FEW_INPUTS, KERNEL_SHORT, KERNEL_SHARES, KERNEL_TILES = 0, 1, 2, 3, 8, 16

# every symbol include/evox.h declares
EXPORTS = (
    "evox_scratch_bytes", "evox_state_create", "evox_state_destroy", "evox_eval", "evox_eval_ld",
    "evox_eval_argmin_scratch_bytes", "evox_eval_argmin", "evox_eval_argmin_noalloc", "evox_pso_step",
    "evox_pso_wait",
    "evox_cso_step",
    "evox_de_step", "evox_es_step", "evox_pgpe_step", "evox_maes_step", "evox_nsga2_step",
    "evox_nsga2_sort_scratch_bytes", "evox_nsga2_sort",
    "evox_cso_refresh", "evox_best", "evox_generation", "evox_set_generation", "evox_row_layout",
    "evox_default_ldx",
    "evox_fill_normal", "evox_sgemm", "evox_copy", "evox_pso_stream", "evox_pair_move", "evox_philox_fill",
    "evox_permutation_scratch_bytes",
    "evox_permutation", "evox_argsort_u32",
    "evox_profile", "evox_profile_read", "evox_strerror", "evox_last_error",
    "evox_layer_kernels", "evox_linear", "evox_linear_grad_scratch_bytes", "evox_linear_grad",
    "evox_layernorm", "evox_layernorm_grad_scratch_bytes", "evox_layernorm_grad",
    "evox_xent_scratch_bytes", "evox_xent",
    "evox_gate", "evox_gate_grad", "evox_route_scratch_bytes", "evox_route", "evox_dispatch", "evox_combine",
    "evox_combine_grad", "evox_adamw_table_bytes", "evox_adamw_plan", "evox_adamw",
)


class EvoxError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"evox error {code}: {msg}")
        self.code = code


class Params(ctypes.Structure):
    _fields_ = [
        ("algo", ctypes.c_int32), ("fn_id", ctypes.c_int32),
        ("N", ctypes.c_int64), ("D", ctypes.c_int64), ("ldx", ctypes.c_int64),
        ("lb", ctypes.c_float), ("ub", ctypes.c_float),
        ("v_lo", ctypes.c_float), ("v_hi", ctypes.c_float),
        ("w", ctypes.c_float), ("c1", ctypes.c_float), ("c2", ctypes.c_float),
        ("phi", ctypes.c_float), ("vmax", ctypes.c_float),
        ("clamp_x", ctypes.c_int32),
        ("x_init", ctypes.c_int32), ("x_mu", ctypes.c_float), ("x_sigma", ctypes.c_float),
        ("de_f", ctypes.c_float), ("de_cr", ctypes.c_float),
        ("es_sigma", ctypes.c_float), ("es_lr", ctypes.c_float),
        ("pgpe_sigma_lr", ctypes.c_float), ("pgpe_max_change", ctypes.c_float),
        ("seed", ctypes.c_uint64),
        ("n_obj", ctypes.c_int32), ("sbx_eta", ctypes.c_float), ("pm_eta", ctypes.c_float),
        ("cso_local", ctypes.c_int32),
    ]


class Buffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "v", "pbest", "pfit", "fit", "gbest", "xbar", "mat",
                                                "sigma", "obj", "front", "crowd")] + [
        ("scratch", ctypes.c_void_p), ("scratch_bytes", ctypes.c_size_t)]


class Layer(ctypes.Structure):
    """evox_layer: one layer of G networks."""
    _fields_ = [("dtype", ctypes.c_int32), ("act", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("G", "M", "n_in", "n_out")] + [
        ("off", ctypes.c_void_p), ("x_shared", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("ldx", "ldw", "w_stride", "b_stride", "ldr", "ldz", "ldy", "lddx", "lddw",
                                      "dw_stride", "db_stride")]


class Norm(ctypes.Structure):
    """evox_norm: a norm over rows with a gain and a shift per network."""
    _fields_ = [("dtype", ctypes.c_int32)] + [(n, ctypes.c_int64) for n in ("G", "M", "D")] + [
        ("off", ctypes.c_void_p)] + [
        (n, ctypes.c_int64) for n in ("ldx", "ldy", "lddx", "p_stride", "dp_stride")] + [("eps", ctypes.c_float)]


class Classes(ctypes.Structure):
    """evox_classes: rows of logits."""
    _fields_ = [("dtype", ctypes.c_int32)] + [(n, ctypes.c_int64) for n in ("G", "M", "C")] + [
        ("off", ctypes.c_void_p), ("labels_shared", ctypes.c_int32), ("ldz", ctypes.c_int64),
        ("lddz", ctypes.c_int64)]


class Choice(ctypes.Structure):
    """evox_choice: rows of logits of which a gate takes the largest."""
    _fields_ = [("dtype", ctypes.c_int32), ("over", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("T", "G", "k", "ldz", "lddz")]


class Slots(ctypes.Structure):
    """evox_slots: rows with k choices each, and the networks' rows that they become."""
    _fields_ = [("dtype", ctypes.c_int32)] + [
        (n, ctypes.c_int64) for n in ("T", "k", "G", "M", "D", "ldx", "ldy", "lds", "ldds")]


class Parameter(ctypes.Structure):
    """evox_parameter: a tensor that an optimizer updates, as rows."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("p", "g", "m", "v", "m_scale", "v_scale", "master")] + [
        (n, ctypes.c_int64) for n in ("rows", "n", "ldp", "ldg", "lds")]


class AdamPlan(ctypes.Structure):
    """evox_adam_plan: the tensors of a step, as a table in device memory."""
    _fields_ = [("table", ctypes.c_void_p)] + [(n, ctypes.c_int64) for n in ("count", "tiles")] + [
        (n, ctypes.c_int32) for n in ("dtype", "bits", "master")]


class Adam(ctypes.Structure):
    """evox_adam: an optimizer's constants."""
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("lr_dev", ctypes.c_void_p)]


_lib = None


def lib():
    """The loaded libevox.so (raises if it is not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python paper_2301_12457_amd/build.py` (no fallback exists)")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, u32, u64, sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64,
                                     ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t)
        sig = {
            "evox_scratch_bytes": ([P], sz),
            "evox_state_create": ([P, P, P, P], i32),
            "evox_state_destroy": ([P], i32),
            "evox_eval": ([i32, P, i64, i64, P, P], i32),
            "evox_eval_ld": ([i32, P, i64, i64, i64, P, P], i32),
            "evox_eval_argmin_scratch_bytes": ([i64], sz),
            "evox_eval_argmin": ([i32, P, i64, i64, i64, P, P, P, P, sz, P], i32),
            "evox_eval_argmin_noalloc": ([i32, P, i64, i64, i64, P, P, P, P], i32),
            "evox_pso_step": ([P, i64], i32),
            "evox_pso_wait": ([P, ctypes.c_double, P], i32),
            "evox_cso_step": ([P, i64], i32),
            "evox_de_step": ([P, i64], i32),
            "evox_es_step": ([P, i64], i32),
            "evox_pgpe_step": ([P, i64], i32),
            "evox_maes_step": ([P, i64], i32),
            "evox_nsga2_step": ([P, i64], i32),
            "evox_nsga2_sort_scratch_bytes": ([i64, i32], ctypes.c_size_t),
            "evox_nsga2_sort": ([P, i64, i32, P, P, P, ctypes.c_size_t, P], i32),
            "evox_cso_refresh": ([P, i32], i32),
            "evox_best": ([P, P, P, P], i32),
            "evox_generation": ([P], i64),
            "evox_set_generation": ([P, i64], i32),
            "evox_row_layout": ([i32, i64, P, P], i32),
            "evox_default_ldx": ([i32, i64], i64),
            "evox_fill_normal": ([u64, i64, i64, i64, ctypes.c_float, ctypes.c_float, P, P], i32),
            "evox_copy": ([P, P, i64, P], i32),
            "evox_pair_move": ([P, P, i64, i64, i64, P, P], i32),
            "evox_pso_stream": ([P, P, P, i64, P], i32),
            "evox_sgemm": ([i32, i32, i64, i64, i64, ctypes.c_float, P, i64, P, i64, ctypes.c_float, P, i64, P],
                           i32),
            "evox_permutation_scratch_bytes": ([i64, i64], sz),
            "evox_permutation": ([u64, i64, i64, i64, P, P, sz, P], i32),
            "evox_argsort_u32": ([P, i64, P, P, sz, P], i32),
            "evox_philox_fill": ([u64, u32, u32, u32, i64, P, P], i32),
            "evox_profile": ([P, i32], i32),
            "evox_profile_read": ([P, P, P, P], i32),
            "evox_layer_kernels": ([P] * 4, i32),
            "evox_linear": ([P] * 8, i32),
            "evox_linear_grad_scratch_bytes": ([P], sz),
            "evox_linear_grad": ([P] * 9 + [sz, P], i32),
            "evox_layernorm": ([P] * 8, i32),
            "evox_layernorm_grad_scratch_bytes": ([P], sz),
            "evox_layernorm_grad": ([P] * 10 + [sz, P], i32),
            "evox_xent_scratch_bytes": ([P], sz),
            "evox_xent": ([P] * 6 + [sz, P], i32),
            "evox_gate": ([P] * 5, i32),
            "evox_gate_grad": ([P] * 7, i32),
            "evox_route_scratch_bytes": ([P], sz),
            "evox_route": ([P] * 6 + [sz, P], i32),
            "evox_dispatch": ([P] * 6, i32),
            "evox_combine": ([P] * 7, i32),
            "evox_combine_grad": ([P] * 8, i32),
            "evox_adamw_table_bytes": ([i64], sz),
            "evox_adamw_plan": ([i32, i32, P, i64, P, sz, P, P], i32),
            "evox_adamw": ([P] * 4, i32),
            "evox_strerror": ([i32], ctypes.c_char_p),
            "evox_last_error": ([], ctypes.c_char_p),
        }
        for name, (args, res) in sig.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = res
        _lib = L
    return _lib


def _check(rc):
    if rc != OK:
        raise EvoxError(rc, lib().evox_last_error().decode())
    return rc


def _stream(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


LAYOUT_PSO, LAYOUT_CSO, LAYOUT_EVAL = 0, 1, 2


def row_layout(D, kernels=LAYOUT_PSO):
    """(threads per row, float4 chunks per thread) of a kernel family at dimension D."""
    g, n = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().evox_row_layout(kernels, D, ctypes.byref(g), ctypes.byref(n)))
    return g.value, n.value


def evox_eval(fn_id, X, out, stream=None):
    """out[i] = F(X[i]) on the GPU (X: contiguous [N, D] float32 device tensor)."""
    assert X.dim() == 2 and X.is_contiguous()
    _check(lib().evox_eval(fn_id, _ptr(X), X.shape[0], X.shape[1], _ptr(out), _stream(stream)))
    return out


def evox_eval_ld(fn_id, X, N, D, ldx, out, stream=None):
    _check(lib().evox_eval_ld(fn_id, _ptr(X), N, D, ldx, _ptr(out), _stream(stream)))
    return out


def evox_eval_argmin(fn_id, X, N, D, ldx, out, best_fit, best_idx, scratch, stream=None):
    """Fitness of every row plus (best_fit[0], best_idx[0]) = argmin, on the GPU."""
    _check(lib().evox_eval_argmin(fn_id, _ptr(X), N, D, ldx, _ptr(out), _ptr(best_fit),
                                  _ptr(best_idx), _ptr(scratch), scratch.numel() * scratch.element_size(),
                                  _stream(stream)))
    return out


def evox_eval_argmin_noalloc(fn_id, X, N, D, ldx, out, best_fit, best_idx, stream=None):
    """evox_eval_argmin with the library's static per-device scratch (no allocation)."""
    _check(lib().evox_eval_argmin_noalloc(fn_id, _ptr(X), N, D, ldx, _ptr(out), _ptr(best_fit),
                                          _ptr(best_idx), _stream(stream)))
    return out


def evox_eval_argmin_scratch_bytes(N):
    return int(lib().evox_eval_argmin_scratch_bytes(N))


def evox_philox_fill(seed, c1, c2, c3, n_ctr, out, stream=None):
    _check(lib().evox_philox_fill(seed, c1, c2, c3, n_ctr, _ptr(out), _stream(stream)))
    return out


def evox_fill_normal(seed, N, D, ldx, mu, sigma, X, stream=None):
    """X[:N, :D] = mu + sigma z (Philox stream 5, Box-Muller); padding set to 0."""
    _check(lib().evox_fill_normal(seed, N, D, ldx, mu, sigma, _ptr(X), _stream(stream)))
    return X


def evox_sgemm(A, B, C, trans_a=False, trans_b=False, alpha=1.0, beta=0.0, stream=None):
    """C = alpha op(A) op(B) + beta C on the matrix cores (2-D fp32 tensors,
    row strides multiples of 4)."""
    M = A.shape[1] if trans_a else A.shape[0]
    K = A.shape[0] if trans_a else A.shape[1]
    N = B.shape[0] if trans_b else B.shape[1]
    _check(lib().evox_sgemm(int(trans_a), int(trans_b), M, N, K, alpha, _ptr(A), A.stride(0), _ptr(B),
                            B.stride(0), beta, _ptr(C), C.stride(0), _stream(stream)))
    return C


# ---------------------------------------------------------------------------
# Populations of networks.  Weights and vectors are views of the parameter
# rows ([G, n_out, n_in] and [G, n] tensors whose last dimension is dense);
# activations are [M, n] tensors with dense rows.  A control step is one row per
# network and a few microseconds of GPU time, so the checks are one comparison per
# tensor and name what is wrong only once something is.
# ---------------------------------------------------------------------------
_DTYPES = {}
_FLOAT, _INT = "float32", "int32"  # vectors' types, by name: torch is imported with the first call


def _look_at_torch():
    """Fills _DTYPES, whole or not at all for whoever reads it meanwhile."""
    global _DTYPES
    import torch
    # a device's current stream's handle without its object (3 us), where torch has it
    raw, device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
    _DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16, _FLOAT: torch.float32, _INT: torch.int32,
               "stream": raw or (lambda d: torch.cuda.current_stream(d).cuda_stream),
               "device": device or torch.cuda.current_device}


def _dtype(t):
    """The element type's id of a tensor on the GPU."""
    if not _DTYPES:
        _look_at_torch()
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise EvoxError(EINVAL, f"element type {t.dtype}: float32, bfloat16 or float16")
    if t.get_device() < 0:
        raise EvoxError(EINVAL, f"a tensor on {t.device}: the kernels read the GPU's memory")
    return d


def _view(what, t, like, shape):
    """Checks a tensor (or None): this shape, like's type and device, dense rows.  Its address."""
    if t is None:
        return None
    if (t.dtype is like.dtype and t.shape == shape and (t.stride(-1) == 1 or shape[-1] == 1)
            and t.get_device() == like.get_device()):
        return t.data_ptr()
    if t.dtype != like.dtype or t.device != like.device:
        raise EvoxError(EINVAL, f"{what}: {t.dtype} on {t.device}, needs {like.dtype} on {like.device}")
    if tuple(t.shape) != tuple(shape):
        raise EvoxError(EINVAL, f"{what} has shape {tuple(t.shape)}, needs {tuple(shape)}")
    if t.numel():
        raise EvoxError(EINVAL, f"{what}: rows are not dense")
    return t.data_ptr()


def _vector(what, t, dtype, n, like):
    """Checks a dense vector (or None) of n elements on like's device.  Its address."""
    if t is None:
        return None
    if t.dtype is not _DTYPES[dtype] or t.shape != (n,) or t.get_device() != like.get_device() or not t.is_contiguous():
        raise EvoxError(EINVAL, f"{what}: a dense {dtype} tensor of {n} on {like.device}")
    return t.data_ptr()


def _pitch(t):
    """The row pitch of an [M, n] tensor (of one row, or none: n)."""
    return t.stride(-2) if t.size(-2) > 1 else t.size(-1)


def _dense(what, t):
    """The row pitch of an [M, n] tensor, whose rows have to be dense."""
    (M, n), s = t.shape, t.stride()
    if s[1] != 1:
        _view(what, t, t, t.shape)
    return s[0] if M > 1 else n


def _net_stride(t):
    return t.stride(0) if t.shape[0] > 1 else 0


def _offsets(off, like, G):
    return _vector("off", off, _INT, G + 1, like)


def _raw_stream(stream, like):
    """The HIP stream of a call, the given one or the current one: of like's device, which
    has to be the current one too (the handle of any device's default stream is 0)."""
    d, current = like.get_device(), _DTYPES["device"]()
    own = getattr(stream, "device", None)  # (a bare handle has none)
    if current != d or own is not None and own.index != d:
        raise EvoxError(EINVAL, f"tensors on device {d}: the current device is {current}"
                                + ("" if own is None else f", the stream's {own.index}"))
    return _DTYPES["stream"](d) if stream is None else stream.cuda_stream


def _empty(nbytes, device, stream):
    """Bytes of the memory pool of a stream (None: the current one)."""
    import torch
    if stream is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _scratch(nbytes, like, scratch, stream):
    """The caller's scratch, or one of this size from the memory of the call's stream (a
    block of the current stream's may be in use there, which nothing orders another
    stream behind, and its next user would not wait for this one)."""
    if nbytes == 0:
        _check(EINVAL)
    if scratch is None:
        scratch = _empty(nbytes, like.device, stream)
    elif scratch.get_device() != like.get_device() or not scratch.is_contiguous():
        raise EvoxError(EINVAL, f"scratch: a dense tensor on {like.device}")
    return scratch, scratch.numel() * scratch.element_size()


def _layer(x, w, y, act, off):
    """The layer of weights w [G, n_out, n_in] between x and y (or dy)."""
    # one pass for what most calls are; anything else is checked and named below
    d, dev = _dtype(w), w.get_device()
    ws, xs, ys, wt, xt, yt = w.shape, x.shape, y.shape, w.stride(), x.stride(), y.stride()
    if (len(ws) == 3 and len(xs) == 2 and len(ys) == 2 and x.dtype is w.dtype and y.dtype is w.dtype
            and x.get_device() == dev and y.get_device() == dev and wt[2] == 1 and xt[1] == 1 and yt[1] == 1):
        (G, n_out, n_in), (R, k), (M, n) = ws, xs, ys
        shared = off is None and G > 1 and R != M
        if G > 1 and n_out > 1 and R > 1 and M > 1 and k == n_in and n == n_out and (R * G if shared else R) == M:
            return Layer(d, act, G, M, n_in, n_out, _offsets(off, w, G), shared, xt[0], wt[1], wt[0], 0, 0, 0, yt[0])
    if w.dim() != 3 or x.dim() != 2 or y.dim() != 2:
        raise EvoxError(EINVAL, "w must be [G, n_out, n_in], x and y [rows, n]")
    (G, n_out, n_in), M = w.shape, y.shape[0]
    shared = off is None and G > 1 and x.shape[0] != M
    if shared and M % G:
        raise EvoxError(EINVAL, f"{M} rows for {G} networks")
    _view("w", w, w, w.shape)
    _view("x", x, w, (M // G if shared else M, n_in))
    _view("y", y, w, (M, n_out))
    return Layer(_dtype(w), act, G, M, n_in, n_out, _offsets(off, w, G), shared, _pitch(x), _pitch(w), _net_stride(w),
                 0, 0, 0, _pitch(y))


def layer_kernels(dtype, G, M, n_in, n_out, ragged=False, act=ACT_NONE):
    """(forward, dx, dw): the kernels of a layer of this type and these sizes, with
    offsets or as many rows for each network (host arithmetic)."""
    p = Layer(dtype, act, G, M, n_in, n_out, 4 if ragged else None)  # (the offsets are not read)
    out = [ctypes.c_int32(0) for _ in range(3)]
    _check(lib().evox_layer_kernels(ctypes.byref(p), *(ctypes.byref(o) for o in out)))
    return tuple(o.value for o in out)


def evox_linear(x, w, y, b=None, r=None, z=None, off=None, act=ACT_NONE, stream=None):
    """y = act(x W_g^T + b_g) + r for the rows of every network g.

    x [M, n_in] (or [M / G, n_in]: every network on the same rows), w [G, n_out,
    n_in], b [G, n_out], r, z, y [M, n_out]; off int32 [G + 1]: network g has
    rows off[g] .. off[g + 1), by default M / G each.  z receives the
    pre-activations (for evox_linear_grad)."""
    p = _layer(x, w, y, act, off)
    rows = y.shape
    if b is not None:
        _view("b", b, w, (p.G, p.n_out))
        p.b_stride = _net_stride(b)
    if r is not None:
        _view("r", r, w, rows)
        p.ldr = _pitch(r)
    if z is not None:
        _view("z", z, w, rows)
        p.ldz = _pitch(z)
    rc = lib().evox_linear(ctypes.byref(p), x.data_ptr(), w.data_ptr(), None if b is None else b.data_ptr(),
                           None if r is None else r.data_ptr(), None if z is None else z.data_ptr(), y.data_ptr(),
                           _raw_stream(stream, w))
    if rc != OK:
        _check(rc)
    return y


def evox_linear_grad_scratch(x, w, dy):
    """Scratch for evox_linear_grad calls of these shapes (any activation and offsets)."""
    import torch
    G, M = w.shape[0], dy.shape[0]
    off = torch.zeros(G + 1, dtype=torch.int32, device=w.device) if x.shape[0] == M and M % G else None
    p = _layer(x, w, dy, ACT_NONE, off)
    return _scratch(lib().evox_linear_grad_scratch_bytes(ctypes.byref(p)), w, None, None)[0]


def evox_linear_grad(x, w, dy, z=None, dx=None, dw=None, db=None, off=None, act=ACT_NONE, scratch=None, stream=None):
    """The gradient of evox_linear from dy and the stored z: dx [M, n_in], dw [G,
    n_out, n_in], db [G, n_out], each where given (the residual's is dy)."""
    p = _layer(x, w, dy, act, off)
    z_at = _view("z", z, w, dy.shape)
    dx_at = _view("dx", dx, w, (p.M, p.n_in))
    dw_at = _view("dw", dw, w, w.shape)
    db_at = _view("db", db, w, (p.G, p.n_out))
    if z is not None:
        p.ldz = _pitch(z)
    if dx is not None:
        p.lddx = _pitch(dx)
    if dw is not None:
        p.lddw, p.dw_stride = _pitch(dw), _net_stride(dw)
    if db is not None:
        p.db_stride = _net_stride(db)
    scratch, nbytes = _scratch(lib().evox_linear_grad_scratch_bytes(ctypes.byref(p)), w, scratch, stream)
    _check(lib().evox_linear_grad(ctypes.byref(p), x.data_ptr(), w.data_ptr(), z_at, dy.data_ptr(), dx_at, dw_at,
                                  db_at, scratch.data_ptr(), nbytes, _raw_stream(stream, w)))
    return dx, dw, db


def _norm(x, gamma, off, eps):
    if x.dim() != 2 or gamma.dim() != 2:
        raise EvoxError(EINVAL, "x must be [M, D], gamma [G, D]")
    (M, D), G, d = x.shape, gamma.shape[0], _dtype(x)
    _view("gamma", gamma, x, (G, D))
    return Norm(d, G, M, D, _offsets(off, x, G), _dense("x", x), 0, 0, _net_stride(gamma), 0, eps)


def evox_layernorm(x, gamma, beta, y, mean=None, rstd=None, off=None, eps=1e-5, stream=None):
    """y = (x - mean) rstd gamma_g + beta_g over the rows of x [M, D], with gamma and
    beta [G, D]; mean and rstd (float32 [M]) receive the rows' statistics."""
    p = _norm(x, gamma, off, eps)
    _view("beta", beta, x, gamma.shape)
    _view("y", y, x, x.shape)
    if _net_stride(beta) != p.p_stride:
        raise EvoxError(EINVAL, "gamma and beta have different strides")
    p.ldy = _pitch(y)
    _check(lib().evox_layernorm(ctypes.byref(p), x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.data_ptr(),
                                _vector("mean", mean, _FLOAT, p.M, x), _vector("rstd", rstd, _FLOAT, p.M, x),
                                _raw_stream(stream, x)))
    return y


def evox_layernorm_grad_scratch(x, gamma):
    """Scratch for evox_layernorm_grad calls of these shapes (any offsets)."""
    import torch
    G = gamma.shape[0]
    off = torch.zeros(G + 1, dtype=torch.int32, device=x.device) if x.shape[0] % G else None
    return _scratch(lib().evox_layernorm_grad_scratch_bytes(ctypes.byref(_norm(x, gamma, off, 1.0))), x, None, None)[0]


def evox_layernorm_grad(x, gamma, mean, rstd, dy, dx=None, dgamma=None, dbeta=None, off=None, scratch=None,
                        stream=None):
    """The gradient of evox_layernorm: dx [M, D], dgamma and dbeta [G, D], where given."""
    p = _norm(x, gamma, off, 1.0)
    dy_at = _view("dy", dy, x, x.shape)
    dx_at = _view("dx", dx, x, x.shape)
    dg_at = _view("dgamma", dgamma, x, gamma.shape)
    db_at = _view("dbeta", dbeta, x, gamma.shape)
    p.ldy = _pitch(dy)
    if dx is not None:
        p.lddx = _pitch(dx)
    if dgamma is not None and dbeta is not None:
        p.dp_stride = _net_stride(dgamma)
        if p.dp_stride != _net_stride(dbeta):
            raise EvoxError(EINVAL, "dgamma and dbeta have different strides")
    scratch, nbytes = _scratch(lib().evox_layernorm_grad_scratch_bytes(ctypes.byref(p)), x, scratch, stream)
    _check(lib().evox_layernorm_grad(ctypes.byref(p), x.data_ptr(), gamma.data_ptr(),
                                     _vector("mean", mean, _FLOAT, p.M, x),
                                     _vector("rstd", rstd, _FLOAT, p.M, x), dy_at, dx_at, dg_at, db_at,
                                     scratch.data_ptr(), nbytes, _raw_stream(stream, x)))
    return dx, dgamma, dbeta


def _classes(logits, G, off, shared):
    if logits.dim() != 2:
        raise EvoxError(EINVAL, "logits must be [M, C]")
    (M, C), d = logits.shape, _dtype(logits)
    return Classes(d, G, M, C, _offsets(off, logits, G), shared, _dense("logits", logits), 0)


def evox_xent_scratch(logits, fit):
    """Scratch for evox_xent calls of these shapes (any offsets)."""
    import torch
    G = fit.shape[0]
    off = torch.zeros(G + 1, dtype=torch.int32, device=fit.device) if logits.shape[0] % G else None
    return _scratch(lib().evox_xent_scratch_bytes(ctypes.byref(_classes(logits, G, off, False))), logits, None, None)[0]


def evox_xent(logits, labels, fit, dz=None, off=None, scratch=None, stream=None):
    """fit[g] = mean cross-entropy of network g's rows of logits [M, C] against labels
    (int32 [M], or [M / G]: the same for every network; rows whose label is outside
    0 .. C-1 do not count), and its gradient dz [M, C] where given."""
    if fit.dim() != 1 or labels.dim() != 1:
        raise EvoxError(EINVAL, "fit and labels are vectors")
    G, M = fit.shape[0], logits.shape[0]
    shared = off is None and G > 1 and labels.shape[0] != M
    p = _classes(logits, G, off, shared)
    fit_at = _vector("fit", fit, _FLOAT, G, logits)
    labels_at = _vector("labels", labels, _INT, M // G if shared else M, logits)
    dz_at = _view("dz", dz, logits, logits.shape)
    if dz is not None:
        p.lddz = _pitch(dz)
    scratch, nbytes = _scratch(lib().evox_xent_scratch_bytes(ctypes.byref(p)), logits, scratch, stream)
    _check(lib().evox_xent(ctypes.byref(p), logits.data_ptr(), labels_at, fit_at, dz_at, scratch.data_ptr(), nbytes,
                           _raw_stream(stream, logits)))
    return fit


# ---------------------------------------------------------------------------
# Mixtures of networks: T rows of data, each with k of G networks.  Tables by slot
# ([T, k]: ids, w, pos, dw) are dense; rows are [T, D] and [M, D] tensors with dense rows.
# ---------------------------------------------------------------------------
def _table(what, t, dtype, shape, like):
    """Checks a dense table (or None) of this type and shape on like's device.  Its address."""
    if t is None:
        return None
    if t.dtype is not _DTYPES[dtype] or t.shape != shape or t.get_device() != like.get_device() or not t.is_contiguous():
        raise EvoxError(EINVAL, f"{what}: a dense {dtype} tensor of {tuple(shape)} on {like.device}")
    return t.data_ptr()


def _given(**tensors):
    """Refuses None for what a call cannot do without."""
    for what, t in tensors.items():
        if t is None:
            raise EvoxError(EINVAL, f"{what} is required")


def _is_table(t, dtype, shape, dev):
    return t.dtype is _DTYPES[dtype] and t.shape == shape and t.get_device() == dev and t.is_contiguous()


def _choice(logits, ids, over):
    if logits.dim() != 2 or ids.dim() != 2:
        raise EvoxError(EINVAL, "logits must be [T, G], ids [T, k]")
    (T, G), d = logits.shape, _dtype(logits)
    return Choice(d, over, T, G, ids.shape[1], _dense("logits", logits), 0)


def evox_gate(logits, ids, w, over=GATE_CHOSEN, stream=None):
    """ids (int32 [T, k]) and weights w (float32 [T, k]) of the k largest of every row of
    logits [T, G], in descending order: a softmax over the chosen, or over all (GATE_ALL)."""
    if logits is None or ids is None or w is None:
        _given(logits=logits, ids=ids, w=w)
    p = _choice(logits, ids, over)
    shape = (p.T, p.k)
    rc = lib().evox_gate(ctypes.byref(p), logits.data_ptr(), _table("ids", ids, _INT, shape, logits),
                         _table("w", w, _FLOAT, shape, logits), _raw_stream(stream, logits))
    if rc != OK:
        _check(rc)
    return ids, w


def evox_gate_grad(logits, ids, w, dw, dz, over=GATE_CHOSEN, stream=None):
    """The gradient dz [T, G] of evox_gate's logits from dw (float32 [T, k]), with the
    ids and w that it gave."""
    if logits is None or ids is None or w is None or dw is None or dz is None:
        _given(logits=logits, ids=ids, w=w, dw=dw, dz=dz)
    p = _choice(logits, ids, over)
    dz_at = _view("dz", dz, logits, logits.shape)
    p.lddz = _pitch(dz)
    shape = (p.T, p.k)
    rc = lib().evox_gate_grad(ctypes.byref(p), logits.data_ptr(), _table("ids", ids, _INT, shape, logits),
                              _table("w", w, _FLOAT, shape, logits), _table("dw", dw, _FLOAT, shape, logits), dz_at,
                              _raw_stream(stream, logits))
    if rc != OK:
        _check(rc)
    return dz


def _route(ids, off):
    if ids.dim() != 2 or off.dim() != 1 or off.shape[0] < 2:
        raise EvoxError(EINVAL, "ids must be [T, k], off [G + 1]")
    if not _DTYPES:
        _look_at_torch()
    if ids.get_device() < 0:
        raise EvoxError(EINVAL, f"a tensor on {ids.device}: the kernels read the GPU's memory")
    T, k = ids.shape
    return Slots(F32, T, k, off.shape[0] - 1)


def evox_route_scratch(ids, off):
    """Scratch for evox_route calls of these shapes."""
    p = _route(ids, off)
    return _scratch(lib().evox_route_scratch_bytes(ctypes.byref(p)), ids, None, None)[0]


def evox_route(ids, off, pos, src=None, scratch=None, stream=None):
    """The slots (row, choice) of ids (int32 [T, k]) sorted by network: network g has the
    rows off[g] .. off[g + 1) (int32 [G + 1]); pos (int32 [T, k]) receives every slot's
    row, -1 for ids outside 0 .. G - 1, src (int32 [T k]) every row's slot t k + j."""
    if ids is None or off is None or pos is None:
        _given(ids=ids, off=off, pos=pos)
    p = _route(ids, off)
    # one pass for what most calls are; anything else is checked and named below
    shape, dev, n = ids.shape, ids.get_device(), p.T * p.k
    if (_is_table(ids, _INT, shape, dev) and _is_table(pos, _INT, shape, dev) and _is_table(off, _INT, (p.G + 1,), dev)
            and (src is None or _is_table(src, _INT, (n,), dev)) and scratch is not None and scratch.get_device() == dev
            and scratch.is_contiguous()):
        ids_at, off_at, pos_at = ids.data_ptr(), off.data_ptr(), pos.data_ptr()
        src_at, nbytes = None if src is None else src.data_ptr(), scratch.numel() * scratch.element_size()
    else:
        ids_at, off_at = _table("ids", ids, _INT, shape, ids), _vector("off", off, _INT, p.G + 1, ids)
        pos_at, src_at = _table("pos", pos, _INT, shape, ids), _vector("src", src, _INT, n, ids)
        # (the size of a scratch that the caller has is the call's own to check)
        scratch, nbytes = _scratch(1 if scratch is not None else lib().evox_route_scratch_bytes(ctypes.byref(p)), ids,
                                   scratch, stream)
    rc = lib().evox_route(ctypes.byref(p), ids_at, off_at, pos_at, src_at, scratch.data_ptr(), nbytes,
                          _raw_stream(stream, ids))
    if rc != OK:
        _check(rc)
    return off, pos, src


def _slots(what, rows, xs, pos, w):
    """Slots of pos [T, k] between rows [T, D] and xs [M, D] (or None), with the pitch of the
    rows as ldx, and pos' and w's addresses."""
    # one pass for what most calls are; anything else is checked and named below
    d, dev = _dtype(rows), rows.get_device()
    if xs is not None and rows.dim() == 2 and xs.dim() == 2 and pos.dim() == 2:
        (T, D), (M, n), (t, k), rt, st = rows.shape, xs.shape, pos.shape, rows.stride(), xs.stride()
        if (n == D and t == T and rt[1] == 1 and st[1] == 1 and xs.dtype is rows.dtype and xs.get_device() == dev
                and _is_table(pos, _INT, (T, k), dev) and (w is None or _is_table(w, _FLOAT, (T, k), dev))):
            return (Slots(d, T, k, 0, M, D, rt[0] if T > 1 else D, 0, st[0] if M > 1 else D, 0), pos.data_ptr(),
                    None if w is None else w.data_ptr())
    if rows.dim() != 2 or pos.dim() != 2 or xs is not None and xs.dim() != 2:
        raise EvoxError(EINVAL, "rows must be [T, D], xs [M, D], pos [T, k]")
    (T, D), shape = rows.shape, (rows.shape[0], pos.shape[1])
    if xs is not None:
        _view("xs", xs, rows, (xs.shape[0], D))
    pitch = _pitch(xs) if xs is not None else 0
    return (Slots(d, T, pos.shape[1], 0, 0 if xs is None else xs.shape[0], D, _dense(what, rows), 0, pitch, 0),
            _table("pos", pos, _INT, shape, rows), _table("w", w, _FLOAT, shape, rows))


def evox_dispatch(x, pos, xs, w=None, stream=None):
    """xs[pos[t, j]] = w[t, j] x[t] (x[t] itself without w) for the rows of x [T, D]: the
    rows xs [M, D] in the networks' grouping."""
    if x is None or pos is None or xs is None:
        _given(x=x, pos=pos, xs=xs)
    p, pos_at, w_at = _slots("x", x, xs, pos, w)
    rc = lib().evox_dispatch(ctypes.byref(p), x.data_ptr(), pos_at, w_at, xs.data_ptr(), _raw_stream(stream, x))
    if rc != OK:
        _check(rc)
    return xs


def evox_combine(xs, pos, y, w=None, r=None, stream=None):
    """y[t] = sum_j w[t, j] xs[pos[t, j]] + r[t] for the rows of y [T, D] (w None: 1; r may
    be y)."""
    if xs is None or pos is None or y is None:
        _given(xs=xs, pos=pos, y=y)
    p, pos_at, w_at = _slots("y", y, xs, pos, w)
    p.ldy, r_at = p.ldx, None
    if r is not None:
        r_at = _view("r", r, y, y.shape)
        p.ldx = _pitch(r)
    rc = lib().evox_combine(ctypes.byref(p), xs.data_ptr(), pos_at, w_at, r_at, y.data_ptr(), _raw_stream(stream, y))
    if rc != OK:
        _check(rc)
    return y


def evox_combine_grad(xs, pos, dy, w=None, dxs=None, dw=None, stream=None):
    """The gradient of evox_combine from dy [T, D], each where given: dxs[pos[t, j]] =
    w[t, j] dy[t] [M, D] and dw (float32 [T, k]), for which alone xs is read."""
    if pos is None or dy is None or dw is not None and xs is None:
        _given(pos=pos, dy=dy, xs=xs)
    p, pos_at, w_at = _slots("dy", dy, xs, pos, w)
    dxs_at = dw_at = None
    if dxs is not None:
        if dxs.dim() != 2:
            raise EvoxError(EINVAL, "dxs must be [M, D]")
        (M, n), st = dxs.shape, dxs.stride()
        if (xs is None or M == p.M) and n == p.D and st[1] == 1 and dxs.dtype is dy.dtype and dxs.get_device() == dy.get_device():
            dxs_at = dxs.data_ptr()
        else:
            dxs_at = _view("dxs", dxs, dy, (M if xs is None else p.M, p.D))
        p.M, p.ldds = M, st[0] if M > 1 else p.D
    if dw is not None:
        dw_at = _table("dw", dw, _FLOAT, (p.T, p.k), dy)
    rc = lib().evox_combine_grad(ctypes.byref(p), None if xs is None else xs.data_ptr(), pos_at, w_at, dy.data_ptr(),
                                 dxs_at, dw_at, _raw_stream(stream, dy))
    if rc != OK:
        _check(rc)
    return dxs, dw


class AdamW:
    """AdamW over a list of tensors at once (evox_adamw).

    params and grads are tensors of one type on one device, [n], [G, n] or [G, n_out,
    n_in], each dense or a view of the rows of a wider matrix (of a population's
    parameters: Networks' views), a gradient of its parameter's shape.  Every step()
    reads the gradients from the memory that they have now and updates the parameters in
    theirs, which the optimizer keeps: a tensor that is given other memory (p.data = ..., a new
    gradient in each backward pass) needs a new optimizer, which load() gives the states of
    the one before.

    lr is a number (the attribute may change from step to step) or a float32 tensor [1]
    on the device, which a captured step reads when it is replayed.  master: an fp32 copy of
    16-bit parameters, which the steps update in their place.

    bits: of the moments, 32, or 8 (e4m3 numbers and a scale per 256).  A scale is for
    elements of one row of its parameter's first dimension (of one network, of [G, n]),
    dense or not (but of up to 256 elements in dense rows of fewer than 8 all have one).
    Where rows are short and need none of their own, p.view(-1) has fewer.

    state holds what a checkpoint saves, each for all tensors one behind the other:
    "t" (steps done, int64 [1]), "m", "v" (float32, or float8_e4m3fn: of v the root), with
    8 bits "m_scale" and "v_scale" (ceil(n / 256) for each row of n), and "master".
    """

    def __init__(self, params, grads, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, bits=32, master=False):
        import torch
        self.params, self.grads = list(params), list(grads)
        if not self.params or len(self.params) != len(self.grads):
            raise EvoxError(EINVAL, f"{len(self.params)} parameters and {len(self.grads)} gradients")
        like = self.params[0]
        d = _dtype(like)
        if master and d == F32:
            raise EvoxError(EINVAL, "fp32 parameters are their own master")
        if bits not in (8, 32):
            raise EvoxError(EINVAL, f"bits = {bits}: states of 32 or 8")
        # (what the table's addresses are of, whatever becomes of the tensors)
        self._memory = [t.detach() for t in self.params + self.grads]
        shapes = [self._rows(i, p, g, like, bits) for i, (p, g) in enumerate(zip(self.params, self.grads))]
        sizes = [rows * n for rows, n, *_ in shapes]
        blocks = [rows * -(-n // ADAM_BLOCK) for rows, n, *_ in shapes]
        device, N = like.device, sum(sizes)
        zeros = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype, device=device)
        self._clock = zeros(ADAM_CLOCK, torch.int64)
        self.state = {"t": self._clock[:1]}
        for name in ("m", "v"):
            if bits == 32:
                self.state[name] = zeros(N)
            else:
                self.state[name] = zeros(N, torch.uint8).view(torch.float8_e4m3fn)
                self.state[name + "_scale"] = zeros(sum(blocks))
        if master:
            self.state["master"] = torch.cat([p.detach().reshape(-1) for p in self.params]).float()
        width = {"m": bits // 8, "v": bits // 8, "m_scale": 4, "v_scale": 4, "master": 4}
        at = {name: t.data_ptr() for name, t in self.state.items()}
        tensors = (Parameter * len(shapes))()
        for i, (rows, n, ldp, ldg) in enumerate(shapes):
            tensors[i] = Parameter(self.params[i].data_ptr(), self.grads[i].data_ptr(), at["m"], at["v"],
                                   at.get("m_scale"), at.get("v_scale"), at.get("master"), rows, n, ldp, ldg, n)
            for name, t in self.state.items():
                if name != "t":
                    at[name] += width[name] * (blocks[i] if name.endswith("_scale") else sizes[i])
        self._table, nbytes = _scratch(lib().evox_adamw_table_bytes(len(shapes)), like, None, None)
        self._plan, self._adam = AdamPlan(), Adam(0.0, betas[0], betas[1], eps, weight_decay, None)
        # (waits for the current stream: a step on another one finds the states there too)
        own = _raw_stream(None, like)
        _check(lib().evox_adamw_plan(d, bits, tensors, len(shapes), self._table.data_ptr(), nbytes, ctypes.byref(self._plan), own))
        self.lr, self._like, self._seen, self._shapes = lr, like, {own}, shapes

    def _used_on(self, stream, raw):
        """The memory that the optimizer keeps is not given to others while this stream, the given or the current
        one, works on it (a bare handle's caller sees to that)."""
        import torch
        if stream is None:
            stream = torch.cuda.current_stream(self._like.device)
        elif not isinstance(stream, torch.cuda.Stream):
            return
        self._seen.add(raw)
        for t in (self._clock, self._table, *self.state.values(), *self._memory):
            t.record_stream(stream)

    @staticmethod
    def _rows(i, p, g, like, bits):
        """(rows, n, pitch of p, pitch of g) of a parameter and its gradient."""
        for what, t in ((f"params[{i}]", p), (f"grads[{i}]", g)):
            if t.dtype != like.dtype or t.get_device() != like.get_device():
                raise EvoxError(EINVAL, f"{what}: {t.dtype} on {t.device}, needs {like.dtype} on {like.device}")
            if t.dim() > 1 and t.numel() and not t[0].is_contiguous() or t.dim() == 1 and not t.is_contiguous():
                raise EvoxError(EINVAL, f"{what}: rows are not dense")
        if p.shape != g.shape or p.dim() == 0:
            raise EvoxError(EINVAL, f"params[{i}] has shape {tuple(p.shape)}, its gradient {tuple(g.shape)}")
        dense, N = p.is_contiguous() and g.is_contiguous(), p.numel()
        if not N:
            return 1, 0, 0, 0
        rows, n = p.shape[0], N // p.shape[0]
        # (all elements as one row, but where scales would go from one row into the next)
        if dense and (bits == 32 or p.dim() == 1 or n % ADAM_BLOCK == 0 or N <= ADAM_BLOCK and n < 8):
            return 1, N, N, N
        pitch = lambda t: t.stride(0) if rows > 1 else n
        return rows, n, pitch(p), pitch(g)

    def step(self, stream=None):
        """One step of all parameters along their gradients."""
        lr, a = self.lr, self._adam
        if hasattr(lr, "data_ptr"):
            a.lr_dev = _vector("lr", lr, _FLOAT, 1, self._like)
        else:
            a.lr, a.lr_dev = lr, None
        raw = _raw_stream(stream, self._like)
        if raw not in self._seen:
            self._used_on(stream, raw)
        rc = lib().evox_adamw(ctypes.byref(a), ctypes.byref(self._plan), self._clock.data_ptr(), raw)
        if rc != OK:
            _check(rc)

    def load(self, state):
        """The states (and the count of steps) of a checkpoint, by the names of `state`."""
        if set(state) != set(self.state):
            raise EvoxError(EINVAL, f"states {sorted(state)}, needs {sorted(self.state)}")
        for name, t in state.items():
            if t.shape != self.state[name].shape or t.dtype != self.state[name].dtype:
                raise EvoxError(EINVAL, f"{name}: {t.dtype} {tuple(t.shape)}, needs {self.state[name].dtype} "
                                        f"{tuple(self.state[name].shape)}")
        raw = _DTYPES["stream"](self._like.get_device())
        if raw not in self._seen:
            self._used_on(None, raw)
        for name, t in state.items():
            self.state[name].copy_(t)


def evox_nsga2_sort(F, front, crowd, scratch=None, stream=None):
    """Fronts (int32) and crowding distances (float64) of the rows of F
    [n, M] (fp32 device tensor), through the library's sort."""
    n, M = F.shape
    nbytes = int(lib().evox_nsga2_sort_scratch_bytes(n, M))
    if nbytes == 0:
        _check(EINVAL)
    if scratch is None:
        scratch = _empty(nbytes, F.device, stream)
    _check(lib().evox_nsga2_sort(_ptr(F), n, M, _ptr(front), _ptr(crowd), _ptr(scratch),
                                 scratch.numel() * scratch.element_size(), _stream(stream)))
    return front, crowd


def evox_copy(src, dst, n, stream=None):
    """dst[:n] = src[:n] by the library's streaming copy (bandwidth reference)."""
    _check(lib().evox_copy(_ptr(src), _ptr(dst), n, _stream(stream)))
    return dst


def evox_pso_stream(x, v, p, n, stream=None):
    """v[:n] += p[:n] - x[:n]; x[:n] += v[:n]: the 20 B per element stream of
    a PSO generation (diagnostic)."""
    _check(lib().evox_pso_stream(_ptr(x), _ptr(v), _ptr(p), n, _stream(stream)))


def evox_pair_move(x, v, N, D, ldx, winner_of, stream=None):
    """The data movement of one swarm-mean CSO generation (diagnostic)."""
    _check(lib().evox_pair_move(_ptr(x), _ptr(v), N, D, ldx, _ptr(winner_of), _stream(stream)))


def evox_permutation(seed, t0, n_gens, N, perm_out, scratch, stream=None):
    """perm_out[g] = the CSO pairing permutation of generation t0 + g."""
    _check(lib().evox_permutation(seed, t0, n_gens, N, _ptr(perm_out), _ptr(scratch),
                                  scratch.numel() * scratch.element_size(), _stream(stream)))
    return perm_out


def evox_argsort_u32(keys, N, perm_out, scratch, stream=None):
    """perm_out[:N] = stable argsort of the uint32 keys[:N] (as int32 tensors)."""
    _check(lib().evox_argsort_u32(_ptr(keys), N, _ptr(perm_out), _ptr(scratch),
                                  scratch.numel() * scratch.element_size(), _stream(stream)))
    return perm_out


def pitch(D, algo=PSO):
    """Recommended row pitch in floats for an algo's state (evox_default_ldx:
    128-byte-aligned rows where that pays, else 16-byte)."""
    ldx = lib().evox_default_ldx(algo, D)
    if ldx <= 0:
        raise EvoxError(EINVAL, f"no row pitch for algo {algo}, D = {D}")
    return ldx


def make_params(algo, fn_id, N, D, lb, ub, v_lo=0.0, v_hi=0.0, w=0.6, c1=1.5, c2=1.5, phi=0.1,
                vmax=0.0, clamp_x=0, seed=0, ldx=None, x_init=0, x_mu=0.0, x_sigma=1.0, de_f=0.5,
                de_cr=0.9, es_sigma=0.1, es_lr=0.01, pgpe_sigma_lr=0.01, pgpe_max_change=0.2, n_obj=3,
                sbx_eta=20.0, pm_eta=20.0, cso_local=0):
    return Params(algo=algo, fn_id=fn_id, N=N, D=D, ldx=pitch(D, algo) if ldx is None else ldx,
                  lb=lb, ub=ub, v_lo=v_lo, v_hi=v_hi, w=w, c1=c1, c2=c2, phi=phi, vmax=vmax,
                  clamp_x=clamp_x, x_init=x_init, x_mu=x_mu, x_sigma=x_sigma, de_f=de_f,
                  de_cr=de_cr, es_sigma=es_sigma, es_lr=es_lr, pgpe_sigma_lr=pgpe_sigma_lr,
                  pgpe_max_change=pgpe_max_change, seed=seed, n_obj=n_obj, sbx_eta=sbx_eta, pm_eta=pm_eta,
                  cso_local=cso_local)


def evox_scratch_bytes(params):
    return int(lib().evox_scratch_bytes(ctypes.byref(params)))


class Swarm:
    """A PSO, CSO, DE, OpenES, PGPE, MA-ES or NSGA-II state over torch-allocated device buffers.

    x, v (and pbest) are [N, ldx] float32 tensors whose first D columns are the
    population; pfit / fit are [N]; gbest / xbar are [ldx].  DE has x and fit
    only (its second population buffer lives in the scratch); ES has x = the
    center theta [ldx] and fit = the last generation's sample fitness [N];
    PGPE also v = the per-dimension deviations [ldx].  MA-ES has x = the center
    y [ldx], v = the path s [ldx], mat = M [D, ldx], sigma [1] and fit [N].
    NSGA-II has x [N, ldx], obj [N, n_obj] (DTLZ1), front [N] (int32) and
    crowd [N] (float64).
    """

    def __init__(self, params: Params, device="cuda", stream=None):
        import torch
        self.P = params
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        N, ldx = params.N, params.ldx
        f32 = dict(dtype=torch.float32, device=device)
        # ES / PGPE: x is the center (one row); PGPE: v the deviations (one row)
        one_row = params.algo in (ES, PGPE, MAES)
        self.x = torch.empty((ldx,) if one_row else (N, ldx), **f32)
        self.v = (torch.empty((N, ldx), **f32) if params.algo in (PSO, CSO)
                  else torch.empty((ldx,), **f32) if params.algo in (PGPE, MAES) else None)
        self.mat = torch.empty((params.D, ldx), **f32) if params.algo == MAES else None
        self.sigma = torch.empty((1,), **f32) if params.algo == MAES else None
        nsga = params.algo == NSGA2
        self.obj = torch.empty((N, params.n_obj), **f32) if nsga else None
        self.front = torch.empty((N,), dtype=torch.int32, device=device) if nsga else None
        self.crowd = torch.empty((N,), dtype=torch.float64, device=device) if nsga else None
        if nsga:
            self.pbest = self.pfit = self.gbest = self.xbar = self.fit = None
        elif params.algo in (DE, ES, PGPE, MAES):
            self.pbest = self.pfit = self.gbest = self.xbar = None
            self.fit = torch.empty((N,), **f32)
        elif params.algo == PSO:
            self.pbest = torch.empty((N, ldx), **f32)
            self.pfit = torch.empty((N,), **f32)
            self.gbest = torch.empty((ldx,), **f32)
            self.fit = torch.empty((N,), **f32)
            self.xbar = None
        else:
            self.pbest = self.pfit = self.gbest = None
            self.fit = torch.empty((N,), **f32)
            self.xbar = torch.empty((ldx,), **f32)
        nbytes = evox_scratch_bytes(params)
        if nbytes == 0:
            _check(EINVAL)
        self.scratch = torch.empty((nbytes + 255) // 256 * 256 // 4, dtype=torch.int32, device=device)
        self.buffers = Buffers(x=_ptr(self.x), v=_ptr(self.v), pbest=_ptr(self.pbest),
                               pfit=_ptr(self.pfit), fit=_ptr(self.fit), gbest=_ptr(self.gbest),
                               xbar=_ptr(self.xbar), mat=_ptr(self.mat), sigma=_ptr(self.sigma),
                               obj=_ptr(self.obj), front=_ptr(self.front), crowd=_ptr(self.crowd),
                               scratch=_ptr(self.scratch),
                               scratch_bytes=self.scratch.numel() * 4)
        # the buffers are the current stream's memory, which work pending there may still read
        current = torch.cuda.current_stream(device)
        if self.stream.cuda_stream != current.cuda_stream:
            self.stream.wait_stream(current)
        self.handle = ctypes.c_void_p()
        _check(lib().evox_state_create(ctypes.byref(self.P), ctypes.byref(self.buffers),
                                       _stream(self.stream), ctypes.byref(self.handle)))

    def __del__(self):
        h = getattr(self, "handle", None)
        if h and _lib is not None:
            _lib.evox_state_destroy(h)
            self.handle = None

    @property
    def D(self):
        return self.P.D

    @property
    def t(self):
        return int(lib().evox_generation(self.handle))

    def set_generation(self, t):
        _check(lib().evox_set_generation(self.handle, t))

    def step(self, n_gens=1):
        if self.P.algo == PSO:
            _check(lib().evox_pso_step(self.handle, n_gens))
        elif self.P.algo == CSO:
            _check(lib().evox_cso_step(self.handle, n_gens))
        elif self.P.algo == DE:
            _check(lib().evox_de_step(self.handle, n_gens))
        elif self.P.algo == ES:
            _check(lib().evox_es_step(self.handle, n_gens))
        elif self.P.algo == PGPE:
            _check(lib().evox_pgpe_step(self.handle, n_gens))
        elif self.P.algo == MAES:
            _check(lib().evox_maes_step(self.handle, n_gens))
        else:
            _check(lib().evox_nsga2_step(self.handle, n_gens))

    def pso_wait(self, seconds):
        """How long the blocks of a resident PSO call wait for each other (< 0: by
        the call's size); the number of calls that one block has had to do."""
        n = ctypes.c_int64(0)
        _check(lib().evox_pso_wait(self.handle, seconds, ctypes.byref(n)))
        return n.value

    def refresh(self, refit=True):
        _check(lib().evox_cso_refresh(self.handle, 1 if refit else 0))

    def best(self, with_x=False):
        import numpy as np
        f = ctypes.c_float(0.0)
        i = ctypes.c_int64(0)
        xb = np.zeros(self.P.D, np.float32) if with_x else None
        _check(lib().evox_best(self.handle, ctypes.byref(f), ctypes.byref(i),
                               xb.ctypes.data_as(ctypes.c_void_p) if with_x else None))
        return (f.value, i.value, xb) if with_x else (f.value, i.value)

    def profile(self, enable):
        _check(lib().evox_profile(self.handle, 1 if enable else 0))

    def profile_read(self):
        ms, n, imp = ctypes.c_double(0), ctypes.c_int64(0), ctypes.c_int64(0)
        _check(lib().evox_profile_read(self.handle, ctypes.byref(ms), ctypes.byref(n),
                                       ctypes.byref(imp)))
        return ms.value, n.value, imp.value

    def view(self, name):
        """The [N, D] (or [D]) part of a buffer, without the padding columns."""
        t = getattr(self, name)
        return t[..., :self.P.D]
