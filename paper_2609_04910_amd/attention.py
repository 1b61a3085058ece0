"""Thin ctypes binding of the C ABI in include/gs_attention.h: softmax attention,
its gradients, and attention over a paged cache.

Argument marshalling only, as in gauss_sum.py: every step of the computation
runs in the HIP kernels of ``libgs_attention.so``, PyTorch provides device memory
and the stream, there is no fallback, and errors are GaussSumError.

Entry points (the C names without their ``gs_`` prefix):
  attention_fwd(q, k, v, ...)                        -> out, lse
  attention_bwd(q, k, v, out, lse, dout, ...)        -> dq, dk, dv
  attention_append(k, v, k_pages, v_pages, page_table, seq_lens, ...)
  attention_paged(q, k_pages, v_pages, page_table, seq_lens, ...) -> out
  attention_fwd_workspace_size / attention_bwd_workspace_size / attention_paged_workspace_size
and ``attention(q, k, v, ...)`` is the forward call under autograd.

Layouts.  Dense: q is B x M x Hq x D, k is B x N x Hkv x D, v is B x N x Hkv x C,
with q_lens / k_lens (int32, B) the rows in use of each sequence where not all
are.  Packed, with q_offsets / k_offsets (int32, B + 1; k_offsets defaults to
q_offsets): q is T x Hq x D, k and v are S x Hkv x (D, C), the sequences one
behind the other.  Any strides with contiguous columns; Hq a multiple of Hkv;
fp16 or bf16, results in the inputs' dtype, lse (log sum exp of the scores) in
fp32 as B x Hq x M or Hq x T.

Rows that belong to no sequence are 0 (lse: -inf) in results allocated here and
left as they were in the caller's own (out=, lse=; low= goes with out).

stream=: the call's kernels go to that stream of the tensors' GPU, and its results
and workspace are allocated there.  Inputs have to be ready on it, and other streams
wait for it before they read the results.
"""
import ctypes
import functools
import os
import struct
import threading

from . import gauss_sum as gs

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgs_attention.so")
EXPORTED = ("gs_attention_fwd", "gs_attention_fwd_workspace_size", "gs_attention_bwd",
            "gs_attention_bwd_workspace_size", "gs_attention_paged", "gs_attention_paged_workspace_size",
            "gs_attention_append")
MAX_DIM = 256  # GAUSS_SUM_MAX_DIM
REST_OUT, REST_LSE = 1, 2  # GS_ATTENTION_REST_OUT, GS_ATTENTION_REST_LSE


class Problem(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("M", ctypes.c_int64), ("N", ctypes.c_int64), ("Hq", ctypes.c_int64),
                ("Hkv", ctypes.c_int64), ("D", ctypes.c_int64), ("C", ctypes.c_int64), ("window", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("packed", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("zero_rest", ctypes.c_int32), ("scale", ctypes.c_float)]


class Array(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class Cache(ctypes.Structure):
    _fields_ = [("k", Array), ("v", Array), ("pages", ctypes.c_int64), ("page_size", ctypes.c_int64),
                ("table_width", ctypes.c_int64), ("table", ctypes.c_void_p), ("lens", ctypes.c_void_p)]


_lib = None


def load(path=LIB_PATH, torch_runtime=True):
    """Load libgs_attention.so (built in-tree by ``__graft_entry__.build()``); torch
    first, as in gauss_sum.load."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("HIP library %s is missing: run __graft_entry__.build() first" % path)
    if torch_runtime:
        import torch  # noqa: F401
    lib = ctypes.CDLL(path)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    # structures are passed as byref(...): plain pointers keep the calls short
    lib.gs_attention_fwd.argtypes = [vp] * 9 + [vp, sz, vp]
    lib.gs_attention_bwd.argtypes = [vp] * 13 + [vp, sz, vp]
    lib.gs_attention_paged.argtypes = [vp] * 6 + [vp, sz, vp]
    lib.gs_attention_append.argtypes = [vp] * 6
    lib.gs_attention_fwd_workspace_size.argtypes = [vp]
    lib.gs_attention_bwd_workspace_size.argtypes = [vp, i32, i32, i32]
    lib.gs_attention_paged_workspace_size.argtypes = [vp, vp]
    for name in EXPORTED:
        getattr(lib, name).restype = sz if name.endswith("_size") else i32
    if path == LIB_PATH:
        _lib = lib
    return lib


# The structures of a call are packed into one buffer a thread (a call reads them
# before it returns): making them as ctypes objects takes longer than the call.
_PROBLEM, _ARRAY, _CACHE = "8q4if4x", "4q", "13q"
_AT_ARRAYS, _ARRAY_BYTES, _CACHE_BYTES = 88, 32, 104
_PACK_FWD = struct.Struct("=" + _PROBLEM + 5 * _ARRAY).pack_into
_PACK_BWD = struct.Struct("=" + _PROBLEM + 9 * _ARRAY).pack_into
_PACK_PAGED = struct.Struct("=" + _PROBLEM + 2 * _ARRAY + _CACHE).pack_into
_local = threading.local()


def _buffer():
    """(buffer, its address) of this thread."""
    try:
        return _local.buffer
    except AttributeError:
        buf = ctypes.create_string_buffer(_AT_ARRAYS + 9 * _ARRAY_BYTES + _CACHE_BYTES)
        _local.buffer = buf, ctypes.addressof(buf)
        return _local.buffer


def _numbers(t, packed):
    """The four numbers of a gs_attention_array (zeros: not given)."""
    if t is None:
        return 0, 0, 0, 0
    s = t.stride()
    if packed:
        return t.data_ptr(), 0, s[0], s[1]
    return t.data_ptr(), s[0], s[1], s[2]


def _check_columns(name, t, dims):
    if t.dim() != dims:
        raise ValueError("%s must have %d dimensions, got %d" % (name, dims, t.dim()))
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("the columns of %s must be contiguous" % name)


def _check_widths(D, C):
    if not (1 <= D <= MAX_DIM and 1 <= C <= MAX_DIM):
        raise ValueError("D and C must be 1 to %d, got %d and %d" % (MAX_DIM, D, C))


def _check_index(name, t, n, device):
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.int32:
        raise TypeError("%s must be an int32 tensor" % name)
    if t.dim() != 1 or (n is not None and t.shape[0] != n) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous 1-d tensor%s, got %s"
                         % (name, "" if n is None else " of %d" % n, tuple(t.shape)))
    if t.device != device:
        raise ValueError("%s must be on %s" % (name, device))


def _dtype(*named):
    """The one dtype of the tensors: fp16 or bf16."""
    code = gs._dtype_code(named[0][1].dtype)
    if code == gs.GS_F32:
        raise TypeError("%s must be float16 or bfloat16" % named[0][0])
    for name, t in named[1:]:
        if t.dtype != named[0][1].dtype:
            raise TypeError("%s and %s must share a dtype" % (named[0][0], name))
    return code


def _check_gpu(*named):
    device = named[0][1].device
    for name, t in named:
        if not t.is_cuda:
            raise ValueError("%s must be a GPU tensor" % name)
        if t.device != device:
            raise ValueError("%s must be on %s" % (name, device))


def _check_call(q, k, v, causal, window, q_offsets, k_offsets, q_lens, k_lens):
    """Refuses what a forward or backward call cannot take."""
    packed = q_offsets is not None
    if k_offsets is not None and not packed:
        raise ValueError("k_offsets needs q_offsets")
    if packed and (q_lens is not None or k_lens is not None):
        raise ValueError("q_lens / k_lens are for dense sequences, q_offsets / k_offsets for packed ones")
    dims = 3 if packed else 4
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_columns(name, t, dims)
    Hq, D = q.shape[-2:]
    Hkv = v.shape[-2]
    if k.shape[-2] != Hkv or k.shape[-1] != D or k.shape[:-2] != v.shape[:-2]:
        raise ValueError("k must be %s (rows and heads of v, columns of q), got %s"
                         % ("x".join(map(str, v.shape[:-1] + (D,))), tuple(k.shape)))
    if Hkv < 1 or Hq % Hkv or Hq == 0:
        raise ValueError("%d query heads over %d key heads: must be a multiple" % (Hq, Hkv))
    if not packed and q.shape[0] != k.shape[0]:
        raise ValueError("q has %d sequences, k has %d" % (q.shape[0], k.shape[0]))
    _check_widths(D, v.shape[-1])
    if window < 0 or (window and not causal):
        raise ValueError("window must be 0, or positive with causal")
    _dtype(("q", q), ("k", k), ("v", v))
    if packed:
        _check_index("q_offsets", q_offsets, None, q.device)
        if q_offsets.shape[0] < 1:
            raise ValueError("q_offsets must hold one number more than there are sequences")
        if k_offsets is not None:
            _check_index("k_offsets", k_offsets, q_offsets.shape[0], q.device)
    else:
        for name, t in (("q_lens", q_lens), ("k_lens", k_lens)):
            if t is not None:
                _check_index(name, t, q.shape[0], q.device)
    _check_gpu(("q", q), ("k", k), ("v", v))


def _check_stream(stream, device):
    """A kernel enqueued on another GPU's stream would run there, on this one's addresses."""
    if stream.device != device:
        raise ValueError("stream must be on %s, got one on %s" % (device, stream.device))


class _Call:
    """Checked sizes of a forward or backward call."""
    __slots__ = ("sizes", "modes", "scale", "packed", "index", "out_shape", "lse_shape", "gpu", "grad")

    def __init__(self, q, k, v, scale, causal, window, q_offsets, k_offsets, q_lens, k_lens):
        qs, ks, vs = q.shape, k.shape, v.shape
        self.gpu = q.get_device()
        # the usual call, told by its sizes alone; any other goes through the checks
        if not (q_offsets is None and q_lens is None and k_lens is None and k_offsets is None
                and len(qs) == 4 and len(vs) == 4 and window == 0 and ks == (qs[0], vs[1], vs[2], qs[3])
                and 0 < qs[3] <= MAX_DIM and 0 < vs[3] <= MAX_DIM and vs[2] and qs[2] and qs[2] % vs[2] == 0 and vs[0] == qs[0]
                and q.dtype in _dtypes() and k.dtype == q.dtype and v.dtype == q.dtype
                and q.stride(3) == 1 and k.stride(3) == 1 and v.stride(3) == 1
                and self.gpu >= 0 and k.get_device() == self.gpu and v.get_device() == self.gpu):
            _check_call(q, k, v, causal, window, q_offsets, k_offsets, q_lens, k_lens)
        Hq, D = qs[-2:]
        Hkv, C = vs[-2:]
        self.packed = packed = q_offsets is not None
        if packed:
            B, M, N = q_offsets.shape[0] - 1, qs[0], ks[0]
            self.index = q_offsets, (q_offsets if k_offsets is None else k_offsets)
            self.lse_shape = Hq, M
        else:
            B, M, N = qs[0], qs[1], ks[1]
            self.index = q_lens, k_lens
            self.lse_shape = B, Hq, M
        self.out_shape = qs[:-1] + (C,)
        self.sizes = B, M, N, Hq, Hkv, D, C, int(window)
        self.modes = _dtypes()[q.dtype], int(packed), int(bool(causal))
        self.scale = D ** -0.5 if scale is None else float(scale)


@functools.lru_cache(maxsize=None)
def _dtypes():
    import torch
    return {torch.float16: gs.GS_F16, torch.bfloat16: gs.GS_BF16}


@functools.lru_cache(maxsize=4096)
def _bwd_bytes(sizes, modes, want):
    """Workspace of a backward call, by its sizes."""
    p = Problem(*sizes, *modes, 0, 1.0)
    return int(load().gs_attention_bwd_workspace_size(_ref(p), *want))


@functools.lru_cache(maxsize=4096)
def _fwd_bytes(sizes, modes):
    p = Problem(*sizes, *modes, 0, 1.0)
    return int(load().gs_attention_fwd_workspace_size(_ref(p)))


@functools.lru_cache(maxsize=4096)
def _paged_bytes(sizes, modes, page_size, table_width):
    p = Problem(*sizes, *modes, 0, 1.0)
    cache = Cache(Array(), Array(), 0, page_size, table_width, None, None)
    return int(load().gs_attention_paged_workspace_size(_ref(p), _ref(cache)))


def _launch(name, gpu, stream, *args):
    """The library call on the tensors' GPU and the given (or its current) stream."""
    import torch
    call = getattr(_lib or load(), name)
    if gpu == torch._C._cuda_getDevice():
        st = call(*args, torch._C._cuda_getCurrentRawStream(gpu) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(gpu):
            st = call(*args, gs._stream(stream))
    if st != 0:
        raise gs.GaussSumError(st, name)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _check_out(t, name, shape, dtype, device):
    import torch
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a tensor" % name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must be %s, got %s" % (name, "x".join(map(str, shape)), tuple(t.shape)))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s must be on %s" % (name, device))


def _check_like_out(t, name, c, q):
    _check_out(t, name, c.out_shape, q.dtype, q.device)
    _check_columns(name, t, len(c.out_shape))


def _fwd(c, q, k, v, out, lse, low, workspace, stream):
    import torch
    if stream is not None:
        _check_stream(stream, q.device)
    rest = 0
    if out is not None:
        _check_like_out(out, "out", c, q)
    if lse is not None:
        gs._check_tensor(lse, "lse", c.lse_shape, q.device, torch.float32)
    need = _fwd_bytes(c.sizes, c.modes)
    wbytes = 0
    with gs._HERE if stream is None else gs._on(stream):
        if out is None:
            rest = REST_OUT
            out = torch.empty(c.out_shape, dtype=q.dtype, device=q.device)
        if lse is None:
            lse = torch.empty(c.lse_shape, dtype=torch.float32, device=q.device)
            rest |= REST_LSE
        if need or workspace is not None:
            workspace, wbytes = gs._workspace_arg(workspace, need, q.device)
    packed, index = c.packed, c.index
    buf, at = _buffer()
    _PACK_FWD(buf, 0, *c.sizes, *c.modes, rest, c.scale, *_numbers(q, packed), *_numbers(k, packed),
              *_numbers(v, packed), *_numbers(out, packed), *_numbers(low, packed))
    at += _AT_ARRAYS
    _launch("gs_attention_fwd", c.gpu, stream, at - _AT_ARRAYS, at, at + 32, at + 64, gs._ptr(index[0]),
            gs._ptr(index[1]), at + 96, None if low is None else at + 128, lse.data_ptr(), gs._ptr(workspace), wbytes)
    if stream is not None:
        gs._keep_alive(stream, out, lse, workspace=workspace)
    return out, lse


def attention_fwd(q, k, v, scale=None, causal=False, window=0, q_offsets=None, k_offsets=None, q_lens=None,
                  k_lens=None, out=None, lse=None, low=None, workspace=None, stream=None):
    """(out, lse): out_m = sum_n w_mn v_n / sum_n w_mn with w_mn = exp(scale q_m.k_n) over the
    keys that row m sees, lse_m = log sum_n w_mn.

    scale defaults to D ** -0.5.  causal: row i of qn sees the keys j <= i + kn - qn of its
    sequence's kn; window > 0 (with causal): only the last `window` of them.  A row that sees
    nothing gives out = 0 and lse = -inf.  low: a tensor like out that receives what the rounding
    of out leaves (out - rounded), which attention_bwd can use."""
    c = _Call(q, k, v, scale, causal, window, q_offsets, k_offsets, q_lens, k_lens)
    if low is not None:
        _check_like_out(low, "low", c, q)
    return _fwd(c, q, k, v, out, lse, low, workspace, stream)


def attention_fwd_workspace_size(B, M, N, Hq, Hkv, D, C, dtype=gs.GS_F16, packed=False):
    """Workspace bytes of attention_fwd (packed: M and N are the rows of all sequences)."""
    return _fwd_bytes((B, M, N, Hq, Hkv, D, C, 0), (dtype, int(packed), 0))


def attention_bwd_workspace_size(B, M, N, Hq, Hkv, D, C, dtype=gs.GS_F16, packed=False, causal=False, window=0,
                                 want_dq=True, want_dk=True, want_dv=True):
    """Workspace bytes of attention_bwd (packed: M and N are the rows of all sequences)."""
    return _bwd_bytes((B, M, N, Hq, Hkv, D, C, int(window)), (dtype, int(packed), int(bool(causal))),
                      (int(bool(want_dq)), int(bool(want_dk)), int(bool(want_dv))))


def _bwd(c, q, k, v, out, lse, dout, want, low, workspace, stream):
    import torch
    if stream is not None:
        _check_stream(stream, q.device)
    want = int(bool(want[0])), int(bool(want[1])), int(bool(want[2]))
    with gs._HERE if stream is None else gs._on(stream):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if want[0] else None
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device) if want[1] else None
        dv = torch.empty(v.shape, dtype=q.dtype, device=q.device) if want[2] else None
        workspace, wbytes = gs._workspace_arg(workspace, _bwd_bytes(c.sizes, c.modes, want), q.device)
    packed, index = c.packed, c.index
    buf, at = _buffer()
    _PACK_BWD(buf, 0, *c.sizes, *c.modes, REST_OUT, c.scale, *_numbers(q, packed), *_numbers(k, packed),
              *_numbers(v, packed), *_numbers(out, packed), *_numbers(low, packed), *_numbers(dout, packed),
              *_numbers(dq, packed), *_numbers(dk, packed), *_numbers(dv, packed))
    at += _AT_ARRAYS
    _launch("gs_attention_bwd", c.gpu, stream, at - _AT_ARRAYS, at, at + 32, at + 64, gs._ptr(index[0]),
            gs._ptr(index[1]), at + 96, None if low is None else at + 128, lse.data_ptr(), at + 160,
            at + 192 if want[0] else None, at + 224 if want[1] else None, at + 256 if want[2] else None,
            gs._ptr(workspace), wbytes)
    if stream is not None:
        gs._keep_alive(stream, dq, dk, dv, workspace=workspace)
    return dq, dk, dv


def attention_bwd(q, k, v, out, lse, dout, scale=None, causal=False, window=0, q_offsets=None, k_offsets=None,
                  q_lens=None, k_lens=None, want=(True, True, True), low=None, workspace=None, stream=None):
    """(dq, dk, dv) of L = sum <dout, out> for the out, lse and (optional) low of attention_fwd with the
    same arguments; None where not wanted.  dk and dv are summed over the query heads that share a key
    head."""
    import torch
    c = _Call(q, k, v, scale, causal, window, q_offsets, k_offsets, q_lens, k_lens)
    for name, t in (("out", out), ("dout", dout), ("low", low)):
        if name != "low" or t is not None:
            _check_like_out(t, name, c, q)
    gs._check_tensor(lse, "lse", c.lse_shape, q.device, torch.float32)
    return _bwd(c, q, k, v, out, lse, dout, want, low, workspace, stream)


def _make_autograd():
    import torch

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, call):
            # needs_input_grad tells of the inputs, also where no graph is made (call.grad)
            want_low = call.grad and any(ctx.needs_input_grad)
            low = torch.empty(call.out_shape, dtype=q.dtype, device=q.device) if want_low else None
            out, lse = _fwd(call, q, k, v, None, None, low, None, None)
            ctx.save_for_backward(q, k, v, out, lse, low, *(t for t in call.index if t is not None))
            ctx.call = call
            return out

        @staticmethod
        def backward(ctx, g):
            # with create_graph the gradients are marked as not differentiable again;
            # the wrapper that does so takes 20 us, so other calls go without
            return (marked if torch.is_grad_enabled() else gradients)(ctx, g)

    def gradients(ctx, g):
        q, k, v, out, lse, low = ctx.saved_tensors[:6]
        if g.dtype != q.dtype:
            g = g.to(q.dtype)
        if g.shape[-1] > 1 and g.stride(-1) != 1:
            g = g.contiguous()
        return _bwd(ctx.call, q, k, v, out, lse, g, ctx.needs_input_grad[:3], low, None, None) + (None,)

    marked = torch.autograd.function.once_differentiable(gradients)
    return Attention


_autograd = None


def attention(q, k, v, scale=None, causal=False, window=0, q_offsets=None, k_offsets=None, q_lens=None, k_lens=None):
    """attention_fwd under autograd: out, with gradients for q, k and v (arguments as there)."""
    import torch
    global _autograd
    if _autograd is None:
        _autograd = _make_autograd()
    c = _Call(q, k, v, scale, causal, window, q_offsets, k_offsets, q_lens, k_lens)
    c.grad = torch.is_grad_enabled()
    return _autograd.apply(q, k, v, c)


def _cache_call(x, name, k_pages, v_pages, page_table, seq_lens, q_offsets, Hq, D, C, code, window):
    """Checked (sizes, modes) of a call on T x H x width rows x."""
    import torch
    for n, t in (("k_pages", k_pages), ("v_pages", v_pages)):
        _check_columns(n, t, 4)
    Hkv = v_pages.shape[2]
    if k_pages.shape[:3] != v_pages.shape[:3] or k_pages.shape[3] != D or v_pages.shape[3] != C:
        raise ValueError("k_pages must be pages x page_size x Hkv x %d and v_pages the same x %d, got %s and %s"
                         % (D, C, tuple(k_pages.shape), tuple(v_pages.shape)))
    _check_widths(D, C)
    if k_pages.shape[1] < 1:
        raise ValueError("pages must hold at least one row")
    if Hkv < 1 or Hq % Hkv or Hq == 0:
        raise ValueError("%d query heads over %d key heads: must be a multiple" % (Hq, Hkv))
    if not isinstance(page_table, torch.Tensor) or page_table.dtype != torch.int32:
        raise TypeError("page_table must be an int32 tensor")
    if page_table.dim() != 2 or not page_table.is_contiguous():
        raise ValueError("page_table must be a contiguous sequences x pages tensor")
    if page_table.device != x.device:
        raise ValueError("page_table must be on %s" % x.device)
    B, T = page_table.shape[0], x.shape[0]
    _check_index("seq_lens", seq_lens, B, x.device)
    if q_offsets is not None:
        _check_index("q_offsets", q_offsets, B + 1, x.device)
        M = T
    else:
        if (T % B if B else T):
            raise ValueError("%d rows of %s for %d sequences: give q_offsets" % (T, name, B))
        M = T // B if B else 0
    if window < 0:
        raise ValueError("window must not be negative")
    sizes = B, M, 0, Hq, Hkv, D, C, int(window)
    return sizes, (code, int(q_offsets is not None), 1)


def _cache_numbers(k_pages, v_pages, page_table, seq_lens):
    """The thirteen numbers of a gs_attention_cache."""
    return (*_numbers(k_pages, False), *_numbers(v_pages, False), k_pages.shape[0], k_pages.shape[1],
            page_table.shape[1], page_table.data_ptr(), seq_lens.data_ptr())


def _row_numbers(t, sizes, modes):
    """T x H x width rows: packed, or M of every sequence."""
    s = t.stride()
    return t.data_ptr(), 0 if modes[1] else sizes[1] * s[0], s[0], s[1]


def attention_append(k, v, k_pages, v_pages, page_table, seq_lens, q_offsets=None, stream=None):
    """Writes the keys k (T x Hkv x D) and values v (T x Hkv x C) of new tokens into the pages of
    a cache, pages x page_size x Hkv x (D, C): token i of the qn new ones of sequence b goes to
    position seq_lens[b] - qn + i, which is row position % page_size of page
    page_table[b, position // page_size].  seq_lens (int32, B) counts the new tokens.  The T rows are
    T / B of every sequence, or as q_offsets (int32, B + 1) says.  Positions outside the table
    and page numbers outside the cache are passed over."""
    _check_columns("k", k, 3)
    _check_columns("v", v, 3)
    if k.shape[:2] != v.shape[:2]:
        raise ValueError("k and v must share rows and heads, got %s and %s" % (tuple(k.shape), tuple(v.shape)))
    code = _dtype(("k", k), ("v", v), ("k_pages", k_pages), ("v_pages", v_pages))
    H = k.shape[1]
    sizes, modes = _cache_call(k, "k", k_pages, v_pages, page_table, seq_lens, q_offsets, H, k.shape[2], v.shape[2],
                               code, 0)
    if sizes[4] != H:
        raise ValueError("k has %d heads, the pages have %d" % (H, sizes[4]))
    _check_gpu(("k", k), ("v", v), ("k_pages", k_pages), ("v_pages", v_pages))
    if stream is not None:
        _check_stream(stream, k.device)
    buf, at = _buffer()
    _PACK_PAGED(buf, 0, *sizes, *modes, 0, 1.0, *_row_numbers(k, sizes, modes), *_row_numbers(v, sizes, modes),
                *_cache_numbers(k_pages, v_pages, page_table, seq_lens))
    _launch("gs_attention_append", k.get_device(), stream, at, at + 88, at + 120, at + 152, gs._ptr(q_offsets))


def attention_paged_workspace_size(B, M, Hq, Hkv, D, C, page_size, table_width, dtype=gs.GS_F16, packed=False):
    """Workspace bytes of attention_paged (M: tokens of a sequence; packed: of all sequences)."""
    return _paged_bytes((B, M, 0, Hq, Hkv, D, C, 0), (dtype, int(packed), 1), page_size, table_width)


def attention_paged(q, k_pages, v_pages, page_table, seq_lens, q_offsets=None, scale=None, window=0, out=None,
                    return_lse=False, workspace=None, stream=None):
    """Attention of a chunk of new tokens (or one) of every sequence, q: T x Hq x D, over a paged
    cache that holds their keys and values already (attention_append; arguments as there):
    token i of the qn new ones of sequence b sees the keys up to its own position,
    seq_lens[b] - qn + i, with window > 0 the last `window` of them.  Returns out (T x Hq x C), or
    (out, lse) with lse Hq x T.  A row that sees a key whose page number lies outside the cache is NaN;
    positions behind the table's last page hold no key."""
    import torch
    _check_columns("q", q, 3)
    if not (isinstance(v_pages, torch.Tensor) and v_pages.dim() == 4):
        raise ValueError("v_pages must have 4 dimensions")
    code = _dtype(("q", q), ("k_pages", k_pages), ("v_pages", v_pages))
    T, Hq, D = q.shape
    C = v_pages.shape[3]
    sizes, modes = _cache_call(q, "q", k_pages, v_pages, page_table, seq_lens, q_offsets, Hq, D, C, code, window)
    _check_gpu(("q", q), ("k_pages", k_pages), ("v_pages", v_pages))
    if stream is not None:
        _check_stream(stream, q.device)
    rest, lse, wbytes = 0, None, 0
    if out is not None:
        _check_out(out, "out", (T, Hq, C), q.dtype, q.device)
        _check_columns("out", out, 3)
    with gs._HERE if stream is None else gs._on(stream):
        if out is None:
            rest = REST_OUT
            out = torch.empty((T, Hq, C), dtype=q.dtype, device=q.device)
        if return_lse:
            lse = torch.empty((Hq, T), dtype=torch.float32, device=q.device)
            rest |= REST_LSE
        need = _paged_bytes(sizes, modes, k_pages.shape[1], page_table.shape[1])
        if need or workspace is not None:
            workspace, wbytes = gs._workspace_arg(workspace, need, q.device)
    buf, at = _buffer()
    _PACK_PAGED(buf, 0, *sizes, *modes, rest, D ** -0.5 if scale is None else float(scale),
                *_row_numbers(q, sizes, modes), *_row_numbers(out, sizes, modes),
                *_cache_numbers(k_pages, v_pages, page_table, seq_lens))
    _launch("gs_attention_paged", q.get_device(), stream, at, at + 88, at + 152, gs._ptr(q_offsets), at + 120,
            gs._ptr(lse), gs._ptr(workspace), wbytes)
    if stream is not None:
        gs._keep_alive(stream, out, lse, workspace=workspace)
    return (out, lse) if return_lse else out
