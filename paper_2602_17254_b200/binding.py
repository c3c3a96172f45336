"""ctypes binding of ``libtrivance.so``: same names as the C ABI, argument marshalling only.

Every step of the AllReduce path runs in the library's CUDA kernels.  PyTorch is used by
callers for device memory and streams; this module only needs ``data_ptr()``-like integers.
If the library has not been built, loading fails with an error: there is no CPU fallback.
"""
import ctypes
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtrivance.so")

LATENCY_OPTIMAL, BANDWIDTH_OPTIMAL = 0, 1
ALGO_TRIVANCE, ALGO_BRUCK, ALGO_RECDOUB, ALGO_SWING, ALGO_BUCKET = 0, 1, 2, 3, 4
ALGO_MIRRORED = 16
ALGO_SINGLE = 32
INT32, FLOAT32, BFLOAT16, FLOAT16 = 0, 1, 2, 3      # AllReduce: the first two; training operators: the last three
SUM = 0
KERNEL_AUTO, KERNEL_STEP, KERNEL_FUSED, KERNEL_PIPELINED = 0, 1, 2, 3
MAX_RANKS = 1024

(OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_UNDEFINED_SCHEDULE, ERR_ALLOC, ERR_CUDA, ERR_SCRATCH, ERR_TOO_LARGE,
 ERR_TIMEOUT) = range(9)

# every symbol include/trivance.h declares
SYMBOLS = [
    "trv_plan_create", "trv_plan_create_algo", "trv_plan_destroy", "trv_plan_info", "trv_plan_slices", "trv_plan_step",
    "trv_plan_peers", "trv_plan_send_set", "trv_plan_block_bounds", "trv_allreduce", "trv_scratch_bytes",
    "trv_kernel_supported", "trv_allreduce_ex", "trv_allreduce_host", "trv_host_workspace_bytes",
    "trv_link_loads", "trv_plan_message_bytes", "trv_plan_message_bytes_side", "trv_strerror", "trv_launch_count", "trv_last_kernel_name",
    "trv_allreduce_noalloc", "trv_noalloc_max_scratch_bytes", "trv_cost_model", "trv_pipeline_status",
    "trv_pipeline_selftest_timeout", "trv_tma_giveups", "trv_plan_reserve_scratch", "trv_joint_reduce",
    "trv_layernorm_forward", "trv_layernorm_backward", "trv_layernorm_workspace_bytes",
    "trv_router_forward", "trv_router_workspace_bytes", "trv_balance_loss", "trv_router_backward",
    "trv_orthogonalize", "trv_orthogonalize_workspace_bytes",
]


class Cost(ctypes.Structure):
    """trv_cost_t"""
    _fields_ = [("steps", ctypes.c_int32), ("bytes_sent_per_node", ctypes.c_int64), ("tx_bytes", ctypes.c_int64),
                ("latency_term", ctypes.c_double), ("tx_term", ctypes.c_double), ("total", ctypes.c_double),
                ("lambda_", ctypes.c_double), ("delta", ctypes.c_double), ("theta", ctypes.c_double)]

_lib = None


class TrivanceError(RuntimeError):
    def __init__(self, status, what):
        super().__init__("%s: %s (status %d)" % (what, strerror(status), status))
        self.status = status


def lib():
    """The loaded C-ABI library (loads it on first use; raises if it was never built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("%s is missing: build it with `python -m paper_2602_17254_b200.build` "
                               "(there is no fallback path)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        L.trv_plan_create.argtypes = [vp, i32, ctypes.c_int, ctypes.POINTER(vp)]
        L.trv_plan_create_algo.argtypes = [vp, i32, ctypes.c_int, ctypes.c_int, ctypes.POINTER(vp)]
        L.trv_plan_destroy.argtypes = [vp]
        L.trv_plan_info.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.trv_plan_step.argtypes = [vp, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.trv_plan_peers.argtypes = [vp, i32, i32, vp]
        L.trv_plan_send_set.argtypes = [vp, i32, i32, i32, vp]
        L.trv_plan_block_bounds.argtypes = [vp, sz, i32, vp]
        L.trv_plan_message_bytes.argtypes = [vp, sz, sz, i32, i32, vp]
        L.trv_plan_slices.argtypes = [vp, vp]
        L.trv_plan_message_bytes_side.argtypes = [vp, sz, sz, i32, i32, i32, vp]
        L.trv_pipeline_status.argtypes = [vp, vp]
        L.trv_pipeline_selftest_timeout.argtypes = [vp, sz, vp]
        L.trv_allreduce.argtypes = [vp, vp, sz, ctypes.c_int, ctypes.c_int, vp]
        L.trv_plan_reserve_scratch.argtypes = [vp, sz]
        L.trv_joint_reduce.argtypes = [vp, vp, vp, vp, vp, sz, ctypes.c_int, vp]
        L.trv_scratch_bytes.argtypes = [vp, sz, ctypes.c_int, i32, ctypes.POINTER(sz)]
        L.trv_kernel_supported.argtypes = [vp, ctypes.c_int]
        L.trv_kernel_supported.restype = i32
        L.trv_allreduce_ex.argtypes = [vp, vp, vp, sz, sz, sz, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, sz, vp]
        L.trv_allreduce_noalloc.argtypes = [vp, vp, sz, ctypes.c_int, ctypes.c_int, vp]
        L.trv_noalloc_max_scratch_bytes.argtypes = []
        L.trv_noalloc_max_scratch_bytes.restype = sz
        L.trv_allreduce_host.argtypes = [vp, vp, vp, sz, ctypes.c_int, ctypes.c_int, vp, sz, vp]
        L.trv_host_workspace_bytes.argtypes = [vp, sz, ctypes.POINTER(sz)]
        L.trv_link_loads.argtypes = [vp, sz, sz, vp, vp, vp, vp]
        L.trv_cost_model.argtypes = [vp, sz, sz, ctypes.c_double, ctypes.c_double, ctypes.POINTER(Cost)]
        f32, psz = ctypes.c_float, ctypes.POINTER(sz)
        L.trv_layernorm_forward.argtypes = [vp] * 6 + [sz] * 4 + [f32, ctypes.c_int, ctypes.c_int, vp]
        L.trv_layernorm_backward.argtypes = [vp] * 8 + [sz] * 5 + [ctypes.c_int, ctypes.c_int, vp, sz, vp]
        L.trv_layernorm_workspace_bytes.argtypes = [sz, sz, psz]
        L.trv_router_forward.argtypes = [vp] * 6 + [sz, i32, i32, sz, i32, ctypes.c_int, vp, sz, vp]
        L.trv_router_workspace_bytes.argtypes = [sz, i32, psz]
        L.trv_balance_loss.argtypes = [vp, vp, i32, i32, f32, vp, vp]
        L.trv_router_backward.argtypes = [vp] * 6 + [sz, i32, i32, sz, sz, i32, f32, ctypes.c_int, vp]
        L.trv_orthogonalize.argtypes = [vp, vp] + [sz] * 7 + [i32, vp, f32, ctypes.c_int, vp, sz, vp]
        L.trv_orthogonalize_workspace_bytes.argtypes = [sz, sz, sz, psz]
        L.trv_strerror.argtypes = [ctypes.c_int]
        L.trv_strerror.restype = ctypes.c_char_p
        L.trv_launch_count.argtypes = []
        L.trv_launch_count.restype = ctypes.c_uint64
        L.trv_last_kernel_name.argtypes = []
        L.trv_last_kernel_name.restype = ctypes.c_char_p
        _lib = L
    return _lib


def strerror(status):
    return lib().trv_strerror(int(status)).decode()


def noalloc_max_scratch_bytes():
    return int(lib().trv_noalloc_max_scratch_bytes())


def pipeline_status(scratch_ptr, stream=0):
    """Status code (OK or ERR_TIMEOUT) recorded by the last PIPELINED call that used this device scratch."""
    return int(lib().trv_pipeline_status(scratch_ptr, stream))


def pipeline_selftest_timeout(scratch_ptr, scratch_bytes, stream=0):
    _check(lib().trv_pipeline_selftest_timeout(scratch_ptr, scratch_bytes, stream), "trv_pipeline_selftest_timeout")


def tma_giveups():
    """Thread blocks of TMA-fed kernels that gave up waiting for their tile on the current device (0 in a correct run)."""
    v = ctypes.c_uint32()
    _check(lib().trv_tma_giveups(ctypes.byref(v)), "trv_tma_giveups")
    return v.value


def joint_reduce(left, own, right, out, counts, dtype, stream=0):
    """trv_joint_reduce: out[s] = (left[s] + own[s]) + right[s] on segments given as lists of device addresses (0 = side left out)."""
    k = len(own)
    arr = lambda p: None if p is None else (ctypes.c_void_p * k)(*[int(v) if v else None for v in p])
    cnt = (ctypes.c_size_t * k)(*[int(c) for c in counts])
    _check(lib().trv_joint_reduce(arr(left), arr(own), arr(right), arr(out), cnt, k, int(dtype), ctypes.c_void_p(int(stream))),
           "trv_joint_reduce")


# ---- training operators (pointers are plain integers: device addresses, 0 = NULL)

def layernorm_forward(x, gamma, beta, y, mean, rstd, rows, cols, x_stride, y_stride, eps, dtype, param_dtype, stream=0):
    _check(lib().trv_layernorm_forward(x, gamma, beta, y, mean, rstd, rows, cols, x_stride, y_stride, eps, dtype, param_dtype, stream),
           "trv_layernorm_forward")


def layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, rows, cols, dy_stride, x_stride, dx_stride, dtype, param_dtype,
                       workspace=0, workspace_bytes=0, stream=0):
    _check(lib().trv_layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, rows, cols, dy_stride, x_stride, dx_stride, dtype,
                                        param_dtype, workspace, workspace_bytes, stream), "trv_layernorm_backward")


@functools.lru_cache(maxsize=256)
def layernorm_workspace_bytes(rows, cols):
    b = ctypes.c_size_t()
    _check(lib().trv_layernorm_workspace_bytes(rows, cols, ctypes.byref(b)), "trv_layernorm_workspace_bytes")
    return b.value


def router_forward(logits, mask, ids, gates, counts, prob_sum, tokens, experts, top_k, logits_stride, normalize, dtype, workspace,
                   workspace_bytes, stream=0):
    _check(lib().trv_router_forward(logits, mask, ids, gates, counts, prob_sum, tokens, experts, top_k, logits_stride, normalize, dtype,
                                    workspace, workspace_bytes, stream), "trv_router_forward")


@functools.lru_cache(maxsize=256)
def router_workspace_bytes(tokens, experts):
    b = ctypes.c_size_t()
    _check(lib().trv_router_workspace_bytes(tokens, experts, ctypes.byref(b)), "trv_router_workspace_bytes")
    return b.value


def balance_loss(counts, prob_sum, experts, top_k, coef, loss, stream=0):
    _check(lib().trv_balance_loss(counts, prob_sum, experts, top_k, coef, loss, stream), "trv_balance_loss")


def router_backward(logits, mask, ids, dgates, counts, dlogits, tokens, experts, top_k, logits_stride, dlogits_stride, normalize, coef,
                    dtype, stream=0):
    _check(lib().trv_router_backward(logits, mask, ids, dgates, counts, dlogits, tokens, experts, top_k, logits_stride, dlogits_stride,
                                     normalize, coef, dtype, stream), "trv_router_backward")


def orthogonalize(g, out, batch, rows, cols, g_stride, g_batch_stride, out_stride, out_batch_stride, steps, coefficients, eps, dtype,
                  workspace, workspace_bytes, stream=0):
    """coefficients: None, one (a, b, c) for all steps, or one triple per step."""
    _check(lib().trv_orthogonalize(g, out, batch, rows, cols, g_stride, g_batch_stride, out_stride, out_batch_stride, steps,
                                   _ns_coefficients(coefficients, steps), eps, dtype, workspace, workspace_bytes, stream),
           "trv_orthogonalize")


@functools.lru_cache(maxsize=256)
def orthogonalize_workspace_bytes(batch, rows, cols):
    b = ctypes.c_size_t()
    _check(lib().trv_orthogonalize_workspace_bytes(batch, rows, cols, ctypes.byref(b)), "trv_orthogonalize_workspace_bytes")
    return b.value


@functools.lru_cache(maxsize=64)
def _ns_array(flat):
    return (ctypes.c_float * len(flat))(*flat)


def _ns_coefficients(coefficients, steps):
    """HOST float [steps][3] for the library, which reads it during the call."""
    if coefficients is None:
        return None
    c = [tuple(v) if hasattr(v, "__len__") else v for v in coefficients]
    if len(c) == 3 and not any(isinstance(v, tuple) for v in c):
        c = [tuple(c)] * steps
    if len(c) != steps or any(not isinstance(v, tuple) or len(v) != 3 for v in c):
        raise ValueError("coefficients must be one (a, b, c) or one triple per step")
    return _ns_array(tuple(float(v) for t in c for v in t))


def launch_count():
    return int(lib().trv_launch_count())


def last_kernel_name():
    return lib().trv_last_kernel_name().decode()


def _check(status, what):
    if status != OK:
        raise TrivanceError(status, what)


def ptr_array(ptrs):
    """HOST array of pointers in the form the C ABI takes.  Build it once and pass it to the Plan's
    calls instead of a list when the same buffers are used repeatedly (saves the per-call conversion)."""
    if isinstance(ptrs, ctypes.Array):
        return ptrs
    return (ctypes.c_void_p * len(ptrs))(*[int(p) for p in ptrs])


_ptr_array = ptr_array


def _np_ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p) if a is not None else None


class Plan:
    """trv_plan_t with the C ABI's calls as methods."""

    def __init__(self, dims, variant, algo=ALGO_TRIVANCE):
        d = np.ascontiguousarray(np.asarray(dims, dtype=np.int32).reshape(-1))
        h = ctypes.c_void_p()
        _check(lib().trv_plan_create_algo(_np_ptr(d), d.size, int(variant), int(algo), ctypes.byref(h)), "trv_plan_create")
        self._h = h
        self.dims = tuple(int(v) for v in d)
        self.variant, self.algo = int(variant), int(algo)
        n, nd, rows = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
        _check(lib().trv_plan_info(h, ctypes.byref(n), ctypes.byref(nd), ctypes.byref(rows)), "trv_plan_info")
        self.n, self.ndims, self.rows = n.value, nd.value, rows.value
        ns = ctypes.c_int32()
        _check(lib().trv_plan_slices(h, ctypes.byref(ns)), "trv_plan_slices")
        self.nslices = ns.value

    def destroy(self):
        if getattr(self, "_h", None):
            lib().trv_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # ---- schedule queries (host integer tables)
    def step(self, c, row):
        dim, dist = ctypes.c_int32(), ctypes.c_int32()
        _check(lib().trv_plan_step(self._h, c, row, ctypes.byref(dim), ctypes.byref(dist)), "trv_plan_step")
        return dim.value, dist.value

    def peers(self, c, row):
        out = np.zeros((self.n, 2), np.int32)
        _check(lib().trv_plan_peers(self._h, c, row, _np_ptr(out)), "trv_plan_peers")
        return out

    def send_set(self, c, step, dst):
        out = np.zeros(self.n, np.uint8)
        _check(lib().trv_plan_send_set(self._h, c, step, dst, _np_ptr(out)), "trv_plan_send_set")
        return out.astype(bool)

    def send_mask(self, c, step, dst):
        """Raw bytes of trv_plan_send_set (rings of other sizes: bit 0 = from the left peer, bit 1 = from the right)."""
        out = np.zeros(self.n, np.uint8)
        _check(lib().trv_plan_send_set(self._h, c, step, dst, _np_ptr(out)), "trv_plan_send_set")
        return out

    def block_bounds(self, count, c):
        out = np.zeros(self.n + 1, np.int64)
        _check(lib().trv_plan_block_bounds(self._h, count, c, _np_ptr(out)), "trv_plan_block_bounds")
        return out

    def message_bytes(self, count, elem_size, c, row):
        out = np.zeros(self.n, np.int64)
        _check(lib().trv_plan_message_bytes(self._h, count, elem_size, c, row, _np_ptr(out)), "trv_plan_message_bytes")
        return out

    def message_bytes_side(self, count, elem_size, c, row, side):
        out = np.zeros(self.n, np.int64)
        _check(lib().trv_plan_message_bytes_side(self._h, count, elem_size, c, row, side, _np_ptr(out)),
               "trv_plan_message_bytes_side")
        return out

    def kernel_supported(self, kernel):
        return bool(lib().trv_kernel_supported(self._h, int(kernel)))

    def scratch_bytes(self, count, kernel=KERNEL_AUTO, in_place=True):
        b = ctypes.c_size_t()
        _check(lib().trv_scratch_bytes(self._h, count, int(kernel), 1 if in_place else 0, ctypes.byref(b)), "trv_scratch_bytes")
        return b.value

    def reserve_scratch(self, count):
        """trv_plan_reserve_scratch: allocate the plan-owned scratch trv_allreduce needs up to this count (may wait for
        the device); afterwards trv_allreduce is launch-only for every shape."""
        _check(lib().trv_plan_reserve_scratch(self._h, count), "trv_plan_reserve_scratch")

    def host_workspace_bytes(self, count):
        b = ctypes.c_size_t()
        _check(lib().trv_host_workspace_bytes(self._h, count, ctypes.byref(b)), "trv_host_workspace_bytes")
        return b.value

    # ---- AllReduce (pointers are plain integers: device addresses)
    def allreduce(self, rank_ptrs, count, dtype, stream=0, op=SUM):
        arr = _ptr_array(rank_ptrs)
        _check(lib().trv_allreduce(self._h, arr, count, int(dtype), int(op), ctypes.c_void_p(int(stream))), "trv_allreduce")

    def allreduce_ex(self, in_ptrs, out_ptrs, count, dtype, global_count=None, global_offset=0, kernel=KERNEL_AUTO,
                     scratch_ptr=0, scratch_bytes=0, stream=0, op=SUM):
        a_in = _ptr_array(in_ptrs)
        a_out = a_in if out_ptrs is None or out_ptrs is in_ptrs else _ptr_array(out_ptrs)
        gc = count if global_count is None else global_count
        _check(lib().trv_allreduce_ex(self._h, a_in, a_out, count, gc, global_offset, int(dtype), int(op), int(kernel),
                                      ctypes.c_void_p(int(scratch_ptr)), scratch_bytes, ctypes.c_void_p(int(stream))),
               "trv_allreduce_ex")

    def allreduce_noalloc(self, rank_ptrs, count, dtype, stream=0, op=SUM):
        """trv_allreduce_noalloc: in-place latency-form AllReduce whose scratch is a fixed array inside the
        library (16 MiB), for callers that may not allocate device memory.  Calls sharing a GPU must not overlap."""
        arr = _ptr_array(rank_ptrs)
        _check(lib().trv_allreduce_noalloc(self._h, arr, count, int(dtype), int(op), ctypes.c_void_p(int(stream))),
               "trv_allreduce_noalloc")

    def allreduce_host(self, host_in_ptrs, host_out_ptrs, count, dtype, workspace_ptr, workspace_bytes, stream=0, op=SUM):
        a_in = _ptr_array(host_in_ptrs)
        a_out = a_in if host_out_ptrs is None or host_out_ptrs is host_in_ptrs else _ptr_array(host_out_ptrs)
        _check(lib().trv_allreduce_host(self._h, a_in, a_out, count, int(dtype), int(op), ctypes.c_void_p(int(workspace_ptr)),
                                        workspace_bytes, ctypes.c_void_p(int(stream))), "trv_allreduce_host")

    # ---- link loads
    def link_loads(self, count, elem_size=4):
        T, n, D = self.rows, self.n, self.ndims
        msgs = np.zeros((T, n, D, 2), np.int32)
        byts = np.zeros((T, n, D, 2), np.int64)
        mm = np.zeros(T, np.int32)
        mb = np.zeros(T, np.int64)
        _check(lib().trv_link_loads(self._h, count, elem_size, _np_ptr(msgs), _np_ptr(byts), _np_ptr(mm), _np_ptr(mb)),
               "trv_link_loads")
        return {"msgs": msgs, "bytes": byts, "max_msgs": mm, "max_bytes": mb}


    def cost_model(self, count, elem_size, alpha, beta):
        c = Cost()
        _check(lib().trv_cost_model(self._h, count, elem_size, float(alpha), float(beta), ctypes.byref(c)), "trv_cost_model")
        return c


# ---------------------------------------------------------------- torch conveniences (marshalling only)

def _torch_dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return FLOAT32
    if t.dtype == torch.int32:
        return INT32
    raise TypeError("only float32 and int32 tensors are supported")


def allreduce_tensor(plan, x, out=None, kernel=KERNEL_AUTO, global_count=None, global_offset=0, scratch=None):
    """AllReduce of a CUDA tensor x of shape [n, count] (row r = rank r), in place unless `out` is given.

    Rows must be 16-byte aligned (count a multiple of 4, or a row stride that is).  Runs on torch's
    current stream.  Returns the tensor holding the result.
    """
    import torch
    if not x.is_cuda or x.dim() != 2 or x.shape[0] != plan.n or x.stride(1) != 1:
        raise ValueError("x must be a CUDA tensor of shape [n, count] with unit inner stride")
    dst = x if out is None else out
    if dst.shape != x.shape or dst.dtype != x.dtype or dst.stride(1) != 1:
        raise ValueError("out must match x")
    count = x.shape[1]
    es = x.element_size()
    in_ptrs = [x.data_ptr() + r * x.stride(0) * es for r in range(plan.n)]
    out_ptrs = in_ptrs if out is None else [dst.data_ptr() + r * dst.stride(0) * es for r in range(plan.n)]
    need = plan.scratch_bytes(count, kernel, in_place=out is None)
    sp, sb = 0, 0
    if need:
        if scratch is None or scratch.numel() * scratch.element_size() < need:
            scratch = torch.empty(need, dtype=torch.uint8, device=x.device)
        sp, sb = scratch.data_ptr(), scratch.numel() * scratch.element_size()
    plan.allreduce_ex(in_ptrs, None if out is None else out_ptrs, count, _torch_dtype_code(x), global_count, global_offset,
                      kernel, sp, sb, torch.cuda.current_stream().cuda_stream)
    return dst


# Tensor forms of the training operators.  They stand outside autograd, as the AllReduce does: results carry no gradient function even if an
# input requires gradients, and the backward forms are calls of their own (the forward and backward of a torch.autograd.Function, say).

_FLOAT_CODES = {}       # torch dtype -> type code of the training operators; filled on first use


def _float_code(t, what):
    code = _FLOAT_CODES.get(t.dtype)
    if code is None:
        import torch
        _FLOAT_CODES.update({torch.float32: FLOAT32, torch.bfloat16: BFLOAT16, torch.float16: FLOAT16})
        code = _FLOAT_CODES.get(t.dtype)        # another thread may have filled the table since the first look
        if code is None:
            raise TypeError("%s must be float32, bfloat16 or float16" % what)
    return code


_torch = None           # the module, kept from the first call of a tensor form on


def _stream_of(x):
    """(device index, handle of torch's current stream); the tensor must live on the current device: the library launches there."""
    global _torch
    if _torch is None:
        import torch
        lib()
        _torch = torch      # last: the tensor forms use _lib without asking once this is set
    device = x.get_device()
    if device < 0 or not x.is_cuda or device != _torch._C._cuda_getDevice():
        raise ValueError("tensors must live on the current CUDA device")
    return device, _torch._C._cuda_getCurrentRawStream(device)      # current_stream().cuda_stream without its 3 us of wrapping


def _matrix(t, what, like=None):
    """(rows, columns, row stride) of t, after checking that it is a matrix with unit inner stride, of like's shape, type and device."""
    shape = t.shape
    if len(shape) != 2:
        raise ValueError("%s must be a matrix" % what)
    if like is not None and (shape != like.shape or t.dtype != like.dtype or t.get_device() != like.get_device()):
        raise ValueError("%s has another shape, type or device than expected" % what)
    rows, cols = shape
    if t.is_contiguous():
        return rows, cols, cols or 1
    row, one = t.stride()
    if (one != 1 and cols > 1) or (rows > 1 and row < cols):
        raise ValueError("%s must have unit inner stride and rows that do not overlap" % what)
    return rows, cols, row if rows > 1 else cols or 1


def _vector(t, what, n, device, dtype):
    """Address of a contiguous vector of n elements on a device; 0 for None."""
    if t is None:
        return 0
    if t.numel() != n or t.dim() != 1 or t.dtype != dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError("%s must be a contiguous vector of %d elements of type %s on the device of the others" % (what, n, dtype))
    return t.data_ptr()


def _param_type(x, p):
    """torch type and type code of gamma and beta (p: either, or None): float32 or x's."""
    if p is None:
        return None, FLOAT32
    code = _float_code(p, "gamma and beta")
    if code != FLOAT32 and p.dtype != x.dtype:
        raise TypeError("gamma and beta must be float32 or of x's type")
    return p.dtype, code


def _workspace(need, workspace, like):
    """(tensor to keep, address, bytes)"""
    if workspace is not None:
        if workspace.get_device() != like.get_device():
            raise ValueError("workspace lives on another device")
        return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()
    if not need:
        return None, 0, 0
    workspace = like.new_empty(need, dtype=_torch.uint8)
    return workspace, workspace.data_ptr(), need


def layernorm_forward_tensor(x, gamma=None, beta=None, eps=1e-5, out=None):
    """Layer norm of the rows of a CUDA matrix: (y, mean, rstd); mean and rstd (float32) are for the backward pass.
    Outside autograd: layernorm_backward_tensor is the gradient."""
    rows, cols, xs = _matrix(x, "x")
    device, stream = _stream_of(x)
    ptype, pcode = _param_type(x, beta if gamma is None else gamma)
    y = _torch.empty_like(x) if out is None else out
    ys = _matrix(y, "out", x)[2]
    f32 = _torch.float32
    mean, rstd = x.new_empty(rows, dtype=f32), x.new_empty(rows, dtype=f32)
    status = _lib.trv_layernorm_forward(x.data_ptr(), _vector(gamma, "gamma", cols, device, ptype), _vector(beta, "beta", cols, device, ptype),
                                        y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), rows, cols, xs, ys, eps, _float_code(x, "x"), pcode, stream)
    if status:
        raise TrivanceError(status, "trv_layernorm_forward")
    return y, mean, rstd


def layernorm_backward_tensor(dy, x, mean, rstd, gamma=None, out=None, workspace=None):
    """(dx, dgamma, dbeta) from the gradient of layernorm_forward_tensor's y; dgamma and dbeta are float32."""
    rows, cols, xs = _matrix(x, "x")
    device, stream = _stream_of(x)
    ptype, pcode = _param_type(x, gamma)
    dys = _matrix(dy, "dy", x)[2]
    dx = _torch.empty_like(x) if out is None else out
    dxs = _matrix(dx, "out", x)[2]
    f32 = _torch.float32
    dgamma, dbeta = x.new_empty(cols, dtype=f32), x.new_empty(cols, dtype=f32)
    _kept, ws, size = _workspace(layernorm_workspace_bytes(rows, cols), workspace, x)
    status = _lib.trv_layernorm_backward(dy.data_ptr(), x.data_ptr(), _vector(gamma, "gamma", cols, device, ptype),
                                         _vector(mean, "mean", rows, device, f32), _vector(rstd, "rstd", rows, device, f32), dx.data_ptr(),
                                         dgamma.data_ptr(), dbeta.data_ptr(), rows, cols, dys, xs, dxs, _float_code(x, "x"), pcode, ws, size, stream)
    if status:
        raise TrivanceError(status, "trv_layernorm_backward")
    return dx, dgamma, dbeta


def _token_mask(mask, tokens, device):
    if mask is None:
        return 0
    if mask.element_size() != 1 or mask.is_floating_point():
        raise TypeError("mask must be bool or uint8")
    return _vector(mask, "mask", tokens, device, mask.dtype)


def router_forward_tensor(logits, top_k, mask=None, normalize=True, workspace=None):
    """(ids, gates, counts, prob_sum) of a CUDA matrix of logits [tokens, experts]; see trv_router_forward.
    Outside autograd: router_backward_tensor is the gradient."""
    tokens, experts, ls = _matrix(logits, "logits")
    device, stream = _stream_of(logits)
    i32, f32 = _torch.int32, _torch.float32
    ids = logits.new_empty((tokens, top_k), dtype=i32)
    gates = logits.new_empty((tokens, top_k), dtype=f32)
    counts, prob_sum = logits.new_empty(experts + 1, dtype=i32), logits.new_empty(experts, dtype=f32)
    _kept, ws, size = _workspace(router_workspace_bytes(tokens, experts), workspace, logits)
    status = _lib.trv_router_forward(logits.data_ptr(), _token_mask(mask, tokens, device), ids.data_ptr(), gates.data_ptr(), counts.data_ptr(),
                                     prob_sum.data_ptr(), tokens, experts, top_k, ls, 1 if normalize else 0, _float_code(logits, "logits"), ws, size,
                                     stream)
    if status:
        raise TrivanceError(status, "trv_router_forward")
    return ids, gates, counts, prob_sum


def balance_loss_tensor(counts, prob_sum, top_k, coef):
    """The balance loss (float32, no dimensions) from the counts and probability sums of all ranks."""
    experts = prob_sum.shape[0]
    device, stream = _stream_of(counts)
    f32 = _torch.float32
    loss = prob_sum.new_empty((), dtype=f32)
    status = _lib.trv_balance_loss(_vector(counts, "counts", experts + 1, device, _torch.int32), _vector(prob_sum, "prob_sum", experts, device, f32),
                                   experts, top_k, coef, loss.data_ptr(), stream)
    if status:
        raise TrivanceError(status, "trv_balance_loss")
    return loss


def router_backward_tensor(logits, ids, counts, coef, dgates=None, mask=None, normalize=True, out=None):
    """Gradient of the balance loss (times coef) and of the gates' users with respect to the logits; see trv_router_backward."""
    tokens, experts, ls = _matrix(logits, "logits")
    device, stream = _stream_of(logits)
    top_k = ids.shape[1]
    i32 = _torch.int32
    for t, what, dt in ((ids, "ids", i32), (dgates, "dgates", _torch.float32)):
        if t is not None and (t.shape != (tokens, top_k) or t.dtype != dt or t.get_device() != device or not t.is_contiguous()):
            raise ValueError("%s must be a contiguous [tokens, top_k] tensor of %s on the logits' device" % (what, dt))
    dl = _torch.empty_like(logits) if out is None else out
    ds = _matrix(dl, "out", logits)[2]
    status = _lib.trv_router_backward(logits.data_ptr(), _token_mask(mask, tokens, device), ids.data_ptr(), 0 if dgates is None else dgates.data_ptr(),
                                      _vector(counts, "counts", experts + 1, device, i32), dl.data_ptr(), tokens, experts, top_k, ls, ds,
                                      1 if normalize else 0, coef, _float_code(logits, "logits"), stream)
    if status:
        raise TrivanceError(status, "trv_router_backward")
    return dl


def orthogonalize_tensor(g, steps=5, coefficients=None, eps=1e-7, out=None, workspace=None):
    """Newton-Schulz orthogonalisation of a CUDA matrix [rows, cols] or a batch [batch, rows, cols]: a bfloat16 tensor of its shape."""
    import torch
    if g.dim() not in (2, 3):
        raise ValueError("g must be a matrix or a batch of matrices")
    device, stream = _stream_of(g)
    code = _float_code(g, "g")
    o = torch.empty(g.shape, dtype=torch.bfloat16, device=g.device) if out is None else out
    if o.shape != g.shape or o.dtype != torch.bfloat16 or o.get_device() != device:
        raise ValueError("out must be a bfloat16 tensor of g's shape on its device")
    rows, cols = g.shape[-2:]
    batch = g.shape[0] if g.dim() == 3 else 1
    strides = []
    for t, what in ((g, "g"), (o, "out")):
        st = t.stride()
        if g.numel() and ((cols > 1 and st[-1] != 1) or (rows > 1 and st[-2] < cols)):
            raise ValueError("%s must have unit inner stride and rows that do not overlap" % what)
        row = st[-2] if rows > 1 else max(cols, 1)
        strides += [row, st[0] if batch > 1 else rows * row]
    _kept, ws, size = _workspace(orthogonalize_workspace_bytes(batch, rows, cols), workspace, g)
    orthogonalize(g.data_ptr(), o.data_ptr(), batch, rows, cols, strides[0], strides[1], strides[2], strides[3], steps, coefficients, eps, code,
                  ws, size, stream)
    return o
