"""ctypes binding of the C ABI in include/chicle_train.h: argument checks and marshalling only.

The method names are the C entry points without the `chicle_` prefix.  Everything is a torch CUDA tensor
(PyTorch-ROCm supplies device memory and the stream); results are new tensors unless an output is given.
Work is enqueued on the current stream of the device and nothing waits for it; results and workspace come from
torch's allocator on that stream, so a tensor that was made on another stream has to be ready there, as for any
torch operation.  Nothing is recorded for automatic differentiation: while that is on, tensors that require a gradient are
refused (but for gradients that are clipped, as by torch's own clipping), and what is written in place gets a new version.  If the shared library is missing or a call fails this raises; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from array import array
from typing import Optional, Sequence

from .binding import EDEVICE, EINVAL, OK, ChicleError

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libchicle_train.so")
_lib = None

TRAIN_EXPORTS = [
    "chicle_softmax_loss_bytes", "chicle_softmax_loss", "chicle_softmax_loss_grad", "chicle_embed",
    "chicle_embed_grad_bytes", "chicle_embed_grad", "chicle_layer_norm", "chicle_layer_norm_grad_bytes",
    "chicle_layer_norm_grad", "chicle_clip_grads_bytes", "chicle_clip_grads", "chicle_train_take_flags",
    "chicle_train_last_error",
]


def train_library_path() -> str:
    return _LIB_PATH


def load_train_library():
    """dlopen the built library; build it first (hipcc) only when no built library exists."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        from .build import build_train_library
        build_train_library()
    import torch  # noqa: F401  (its HIP runtime owns the tensors and streams: the library binds to that one)
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    sig = {
        "chicle_softmax_loss_bytes": (sz, [vp, i64, vp, i64, i64, i64, i64, i32, i32]),
        "chicle_softmax_loss": (i32, [vp, i64, vp, i64, vp, i32, i64, i64, i64, i32, vp, vp, vp, sz, vp, vp]),
        "chicle_softmax_loss_grad": (i32, [vp, i64, vp, i64, vp, i32, vp, i64, i64, i64, i32, vp, vp, i64, vp, i64, vp, sz, vp, vp]),
        "chicle_embed": (i32, [vp, i64, i64, vp, i32, i64, i64, i32, f32, vp, i64, vp, vp]),
        "chicle_embed_grad_bytes": (sz, [i64, i64, i64]),
        "chicle_embed_grad": (i32, [vp, i32, vp, i64, i64, i64, i64, i32, f32, i32, vp, i64, vp, sz, vp, vp]),
        "chicle_layer_norm": (i32, [vp, i64, vp, vp, i64, i64, i32, f32, vp, i64, vp, vp, vp]),
        "chicle_layer_norm_grad_bytes": (sz, [i64, i64, i32]),
        "chicle_layer_norm_grad": (i32, [vp, i64, vp, i64, vp, vp, vp, i64, i64, i32, vp, i64, vp, vp, vp, sz, vp]),
        "chicle_clip_grads_bytes": (sz, [i32]),
        "chicle_clip_grads": (i32, [vp, vp, vp, vp, i32, f32, vp, vp, sz, vp]),
        "chicle_train_take_flags": (i32, [vp, vp, vp]),
        "chicle_train_last_error": (ctypes.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _at(a: array) -> int:
    """The address of a host array, which stays where it is while it is not changed."""
    return a.buffer_info()[0] if len(a) else 0


class TrainOps:
    """The operators on one GPU.  Holds the library, the device and one flag word; may be used by several threads and on several streams."""

    def __init__(self, device: str = "cuda:0"):
        import torch
        self._L = load_train_library()
        if not torch.cuda.is_available():
            raise ChicleError(EDEVICE, "no GPU visible; this library has no CPU path")
        self._torch = torch
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ChicleError(EINVAL, "device must be a GPU")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self._new_version = torch.autograd.graph.increment_version
        self._types = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
        self._wide = {torch.int32: 0, torch.int64: 1}
        # (the handle of the current stream, without an object around it)
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        # in this word kernels note a label or token out of range; made here, so that any thread's first call, and a captured one, finds it
        self._flag_word = torch.zeros(1, dtype=torch.int32, device=self.device)
        torch.cuda.synchronize(self.device)             # it is zero before any stream's work looks at it

    # -- helpers
    def _call(self, fn, *args):
        """Run a C entry point with the library's GPU current; args end before the stream."""
        t = self._torch.cuda
        if t.current_device() == self._index:
            rc = fn(*args, self._raw_stream(self._index))
        else:
            with t.device(self._index):
                rc = fn(*args, self._raw_stream(self._index))
        if rc != OK:
            raise ChicleError(rc, self._L.chicle_train_last_error().decode())

    def _no_graph(self, name: str):
        raise ChicleError(EINVAL, "%s requires a gradient, and nothing is recorded here: detach it, or call under torch.no_grad()" % name)

    def _empty(self, shape, dtype):
        return self._torch.empty(shape, dtype=dtype, device=self.device)

    def _workspace(self, nbytes: int):
        return self._torch.empty(nbytes, dtype=self._torch.uint8, device=self.device)

    def _flags(self):
        return self._flag_word.data_ptr()

    def _matrix(self, a, name: str, type_of=None, cols: Optional[int] = None):
        """A 2-D tensor of a supported type on this GPU, rows of unit stride that do not overlap: (type, row distance)."""
        if a.device != self.device or a.dim() != 2 or a.dtype not in self._types:
            raise ChicleError(EINVAL, "%s must be a 2-D float32, bfloat16 or float16 tensor on %s" % (name, self.device))
        if type_of is not None and a.dtype != type_of.dtype:
            raise ChicleError(EINVAL, "%s must have the type %s" % (name, type_of.dtype))
        if a.requires_grad and self._torch.is_grad_enabled():
            self._no_graph(name)
        n, d = a.shape
        if d < 1 or (cols is not None and d != cols):
            raise ChicleError(EINVAL, "%s has %d columns" % (name, d))
        s0, s1 = a.stride()
        if (d > 1 and s1 != 1) or (n > 1 and s0 < d):
            raise ChicleError(EINVAL, "%s must be row-major with unit column stride" % name)
        return self._types[a.dtype], s0 if n > 1 else d

    def _vector(self, a, name: str, size: int, dtype):
        if a.device != self.device or a.dim() != 1 or a.shape[0] != size or a.dtype != dtype or not a.is_contiguous():
            raise ChicleError(EINVAL, "%s must be a contiguous %s tensor of %d values on %s" % (name, dtype, size, self.device))
        if a.requires_grad and self._torch.is_grad_enabled():
            self._no_graph(name)
        return a.data_ptr()

    def _indices(self, a, name: str, size: Optional[int] = None):
        if a.device != self.device or a.dtype not in self._wide or a.dim() != 1 or not a.is_contiguous() or (size is not None and a.shape[0] != size):
            raise ChicleError(EINVAL, "%s must be a contiguous int32 or int64 tensor on %s, one value per row" % (name, self.device))
        return a.data_ptr(), self._wide[a.dtype]

    # -- softmax loss
    def softmax_loss(self, x, w, labels):
        """(loss, lse) of rows x [n, d] against classes w [classes, d]; a negative label: none, loss 0."""
        t, ldx = self._matrix(x, "x")
        n, d = x.shape
        _, ldw = self._matrix(w, "w", x, d)
        c = w.shape[0]
        lp, wide = self._indices(labels, "labels", n)
        f32 = self._torch.float32
        loss, lse = self._empty(n, f32), self._empty(n, f32)
        xp, wp = x.data_ptr(), w.data_ptr()
        nbytes = self._L.chicle_softmax_loss_bytes(xp, ldx, wp, ldw, n, d, c, t, 0)
        ws = self._workspace(nbytes)
        self._call(self._L.chicle_softmax_loss, xp, ldx, wp, ldw, lp, wide, n, d, c, t, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), nbytes,
                   self._flags())
        return loss, lse

    def softmax_loss_grad(self, x, w, labels, row_weight):
        """(loss, dx, dw): the loss of every row, and the gradients of sum_i row_weight_i loss_i by x and w."""
        t, ldx = self._matrix(x, "x")
        n, d = x.shape
        _, ldw = self._matrix(w, "w", x, d)
        c = w.shape[0]
        lp, wide = self._indices(labels, "labels", n)
        rp = self._vector(row_weight, "row_weight", n, self._torch.float32)
        loss, dx, dw = self._empty(n, self._torch.float32), self._empty((n, d), x.dtype), self._empty((c, d), x.dtype)
        xp, wp = x.data_ptr(), w.data_ptr()
        nbytes = self._L.chicle_softmax_loss_bytes(xp, ldx, wp, ldw, n, d, c, t, 1)
        ws = self._workspace(nbytes)
        self._call(self._L.chicle_softmax_loss_grad, xp, ldx, wp, ldw, lp, wide, rp, n, d, c, t, loss.data_ptr(), dx.data_ptr(), d, dw.data_ptr(), d,
                   ws.data_ptr(), nbytes, self._flags())
        return loss, dx, dw

    # -- table lookup
    def embed(self, table, ids, scale: float = 1.0):
        """scale * table[ids], ids of any shape; a negative id gives zeros."""
        t, ld = self._matrix(table, "table")
        rows, d = table.shape
        flat = ids.reshape(-1)
        ip, wide = self._indices(flat, "ids")
        n = flat.shape[0]
        out = self._empty((*ids.shape, d), table.dtype)
        self._call(self._L.chicle_embed, table.data_ptr(), ld, rows, ip, wide, n, d, t, scale, out.data_ptr(), d, self._flags())
        return out

    def embed_grad(self, ids, dout, n_rows: int, scale: float = 1.0, into=None):
        """The table's gradient [n_rows, d]: scale * the sum of dout's rows by id; `into`: added to that tensor, which is returned."""
        flat = ids.reshape(-1)
        ip, wide = self._indices(flat, "ids")
        n = flat.shape[0]
        if dout.dim() != 2:
            if tuple(dout.shape[:-1]) != tuple(ids.shape):
                raise ChicleError(EINVAL, "dout needs a row per id")
            dout = dout.reshape(n, dout.shape[-1])
        t, ldd = self._matrix(dout, "dout")
        d = dout.shape[1]
        if dout.shape[0] != n or n_rows < 1:
            raise ChicleError(EINVAL, "dout needs a row per id, and the table a row")
        if into is None:
            out, ldo = self._empty((n_rows, d), dout.dtype), d
        else:
            out, ldo = into, self._matrix(into, "into", dout, d)[1]
            if into.shape[0] != n_rows:
                raise ChicleError(EINVAL, "into needs n_rows rows")
        nbytes = self._L.chicle_embed_grad_bytes(n, d, n_rows)
        ws = self._workspace(nbytes)
        self._call(self._L.chicle_embed_grad, ip, wide, dout.data_ptr(), ldd, n, d, n_rows, t, scale, int(into is not None), out.data_ptr(), ldo,
                   ws.data_ptr(), nbytes, self._flags())
        if into is not None:
            self._new_version(into)
        return out

    # -- layer norm
    def layer_norm(self, x, gamma, beta, eps: float = 1e-5):
        """(y, mean, rstd) of rows x [n, d]."""
        t, ldx = self._matrix(x, "x")
        n, d = x.shape
        gp, bp = self._vector(gamma, "gamma", d, x.dtype), self._vector(beta, "beta", d, x.dtype)
        f32 = self._torch.float32
        y, mean, rstd = self._empty((n, d), x.dtype), self._empty(n, f32), self._empty(n, f32)
        self._call(self._L.chicle_layer_norm, x.data_ptr(), ldx, gp, bp, n, d, t, eps, y.data_ptr(), d, mean.data_ptr(), rstd.data_ptr())
        return y, mean, rstd

    def layer_norm_grad(self, dy, x, gamma, mean, rstd):
        """(dx, dgamma, dbeta) from dy and what layer_norm returned."""
        t, ldx = self._matrix(x, "x")
        n, d = x.shape
        _, lddy = self._matrix(dy, "dy", x, d)
        if dy.shape[0] != n:
            raise ChicleError(EINVAL, "dy needs a row per row of x")
        f32 = self._torch.float32
        gp, mp, rp = self._vector(gamma, "gamma", d, x.dtype), self._vector(mean, "mean", n, f32), self._vector(rstd, "rstd", n, f32)
        dx, dgamma, dbeta = self._empty((n, d), x.dtype), self._empty(d, x.dtype), self._empty(d, x.dtype)
        nbytes = self._L.chicle_layer_norm_grad_bytes(n, d, t)
        ws = self._workspace(nbytes)
        self._call(self._L.chicle_layer_norm_grad, dy.data_ptr(), lddy, x.data_ptr(), ldx, gp, mp, rp, n, d, t, dx.data_ptr(), d, dgamma.data_ptr(),
                   dbeta.data_ptr(), ws.data_ptr(), nbytes)
        return dx, dgamma, dbeta

    # -- clipping
    def _pointers(self, tensors, name: str):
        """Addresses, numbers of values and types of contiguous tensors on this GPU (a list at a time: there are many)."""
        k = len(tensors)
        kinds = [self._types.get(g.dtype) for g in tensors]
        if None in kinds or [g.get_device() for g in tensors] != [self._index] * k or False in [g.is_contiguous() for g in tensors]:
            raise ChicleError(EINVAL, "%s must be contiguous float32, bfloat16 or float16 tensors on %s" % (name, self.device))
        return array("Q", [g.data_ptr() for g in tensors]), array("q", [g.numel() for g in tensors]), array("i", kinds)

    def _clip(self, grads: Sequence, out: Optional[Sequence], max_norm: float):
        k = len(grads)
        where, sizes, types = self._pointers(grads, "gradients")
        to = where if out is grads else None
        if out is not None and to is None:
            to, out_sizes, out_types = self._pointers(out, "outputs")
            if out_sizes != sizes or out_types != types:
                raise ChicleError(EINVAL, "an output per gradient, of its type and number of values")
        norm = self._empty((), self._torch.float32)
        nbytes = self._L.chicle_clip_grads_bytes(k)
        ws = self._workspace(nbytes)
        self._call(self._L.chicle_clip_grads, _at(where), None if to is None else _at(to), _at(sizes), _at(types), k, max_norm,
                   norm.data_ptr(), ws.data_ptr(), nbytes)
        if out is not None:
            self._new_version(out)
        return norm

    def grad_norm(self, grads: Sequence):
        """The 2-norm of all the tensors together, a 0-d float32 tensor."""
        return self._clip(grads, None, 0.0)

    def clip_grads(self, grads: Sequence, max_norm: float, out: Optional[Sequence] = None):
        """grads times min(1, max_norm / (norm + 1e-6)), in place or into `out`; returns the norm before it.  What is written overlaps
        nothing but, where it is the same tensor, its own gradient."""
        return self._clip(grads, grads if out is None else out, max_norm)

    def sync(self):
        """Wait for the current stream; raise if a label or token was past the end that no sync has raised yet.  What another stream
        reports meanwhile is raised by this sync or by a later one."""
        taken = self._empty(1, self._torch.int32)
        self._call(self._L.chicle_train_take_flags, self._flags(), taken.data_ptr())
        bits = int(taken.item())
        if bits:
            raise ChicleError(EDEVICE, "%s out of range" % " and ".join(s for b, s in ((1, "a label"), (2, "a token")) if bits & b))
