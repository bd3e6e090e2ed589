"""Language-model operators on torch tensors: the output layer's cross entropy
with its gradients, and orthogonalised updates.

PyTorch only allocates device memory and supplies the stream; the operators run
in libdsm.so through the binding in ``dsm``.  An object here is the plan of one
problem: it checks tensors, keeps the workspace, and enqueues on torch's current
stream.  Calls of one object share its workspace: on different streams they are put
one after another (under graph capture that is the caller's part, as is keeping the
object while the graph is replayed), and from several threads each call's launches are
enqueued whole before the next call's.
"""
import contextlib
import threading

import torch

from . import dsm

DTYPES = {torch.float32: dsm.DSM_F32, torch.bfloat16: dsm.DSM_BF16}


def _dtype(dtype):
    if dtype not in DTYPES:
        raise ValueError(f"dtype must be torch.float32 or torch.bfloat16, got {dtype}")
    return DTYPES[dtype]


class _Plan:
    def __init__(self):
        self._lock = threading.Lock()

    def _allocate(self, workspace_bytes, device):
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"the operators run on a GPU, got device {device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.workspace_bytes = workspace_bytes
        self.workspace = torch.empty(max(workspace_bytes, 256), dtype=torch.uint8,
                                     device=self.device)
        self._stream = torch.cuda.current_stream(self.device)

    def _enter(self):
        """The current stream, after what this plan last did on another one."""
        stream = torch.cuda.current_stream(self.device)
        if stream != self._stream:
            if not torch.cuda.is_current_stream_capturing():
                stream.wait_stream(self._stream)
                self.workspace.record_stream(stream)
            self._stream = stream
        return stream.cuda_stream

    def _on_device(self):
        if torch.cuda.current_device() == self.device.index:
            return contextlib.nullcontext()
        return torch.cuda.device(self.device)

    @contextlib.contextmanager
    def _enqueue(self):
        """The stream for one call's launches, which no other call's come between."""
        with self._lock, self._on_device():
            yield self._enter()

    def _check(self, name, t, dtype, shape):
        if t.device != self.device:
            raise ValueError(f"{name} is on {t.device}, the plan on {self.device}")
        if t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")


class LinearCE(_Plan):
    """Softmax cross entropy of the logits h w^T (dsm_linear_ce).

    tokens, dim, vocab: the sizes of h (tokens, dim) and w (vocab, dim); dtype:
    of h, w and their gradients, torch.float32 or torch.bfloat16; grads: whether
    a call computes the gradients.
    """

    def __init__(self, tokens, dim, vocab, dtype=torch.float32, grads=True, device="cuda"):
        super().__init__()
        self.problem = dsm.dsm_ce_problem(int(tokens), int(dim), int(vocab), _dtype(dtype),
                                          1 if grads else 0)
        self.dtype, self.grads = dtype, bool(grads)
        self.h_shape = torch.Size((int(tokens), int(dim)))
        self.w_shape = torch.Size((int(vocab), int(dim)))
        self.t_shape = self.h_shape[:1]
        self._allocate(dsm.dsm_ce_workspace(self.problem), device)

    def _rows(self, name, t, shape):
        self._check(name, t, self.dtype, shape)
        if shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}'s rows must be contiguous, got strides {t.stride()}")
        if shape[0] <= 1:
            return shape[1]
        if t.stride(0) < shape[1]:
            raise ValueError(f"{name}'s rows overlap: strides {t.stride()}")
        return t.stride(0)

    def _vector(self, name, t, dtype, shape):
        self._check(name, t, dtype, shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()

    def __call__(self, h, w, target, weight=None, mean=True, dh=None, dw=None, loss=None,
                 total=None, lse=None):
        """{"total", "loss"} and, with gradients, {"dh", "dw"}: total (a scalar)
        is the sum of weight * loss, divided by the number of targets inside the
        vocabulary when mean; loss (tokens,) and lse (tokens,), which is written
        where given, are 0 where the target lies outside; dh and dw are total's
        gradients.  Outputs are written into the tensors given, or into new ones."""
        buf = dsm.dsm_ce_buffers()
        buf.h_stride = self._rows("h", h, self.h_shape)
        buf.w_stride = self._rows("w", w, self.w_shape)
        buf.h, buf.w = h.data_ptr(), w.data_ptr()
        buf.target = self._vector("target", target, torch.int64, self.t_shape)
        if weight is not None:
            buf.weight = self._vector("weight", weight, torch.float32, self.t_shape)
        if total is None:
            total = torch.empty((), dtype=torch.float32, device=self.device)
        if loss is None:
            loss = torch.empty(self.t_shape, dtype=torch.float32, device=self.device)
        buf.total = self._vector("total", total, torch.float32, torch.Size(()))
        buf.loss = self._vector("loss", loss, torch.float32, self.t_shape)
        out = {"total": total, "loss": loss}
        if lse is not None:
            buf.lse = self._vector("lse", lse, torch.float32, self.t_shape)
            out["lse"] = lse
        if self.grads:
            if dh is None:
                dh = torch.empty(self.h_shape, dtype=self.dtype, device=self.device)
            if dw is None:
                dw = torch.empty(self.w_shape, dtype=self.dtype, device=self.device)
            buf.dh_stride = self._rows("dh", dh, self.h_shape)
            buf.dw_stride = self._rows("dw", dw, self.w_shape)
            buf.dh, buf.dw = dh.data_ptr(), dw.data_ptr()
            out["dh"], out["dw"] = dh, dw
        elif dh is not None or dw is not None:
            raise ValueError("dh or dw given to a plan without gradients")
        buf.workspace, buf.workspace_bytes = self.workspace.data_ptr(), self.workspace_bytes
        with self._enqueue() as buf.stream:
            dsm.dsm_linear_ce(self.problem, buf, mean)
        return out


class Ortho(_Plan):
    """Orthogonalised updates of `count` matrices of one shape (dsm_orthogonalize,
    dsm_ortho_step).

    Tensors are (count, rows, cols), or (rows, cols) for one matrix, with
    contiguous rows; the matrices may lie apart (a view of several layers).  With
    `offsets` (elements) and `row_stride`, they are instead any tensors that hold
    the matrices at these places, for instance the arenas of ``arena.Arenas``.
    dtype: torch.float32 or torch.bfloat16 (orthogonalize only); steps, eps and
    coeffs (steps x 3) as in dsm_ortho_problem.
    """

    def __init__(self, rows, cols, count=1, dtype=torch.float32, steps=5, eps=1e-7, coeffs=None,
                 offsets=None, row_stride=None, device="cuda"):
        super().__init__()
        self.rows, self.cols, self.count = int(rows), int(cols), int(count)
        self.dtype, self._given = dtype, offsets is not None
        self._args = dict(dtype=_dtype(dtype), steps=int(steps), eps=float(eps), coeffs=coeffs)
        self._problems = {}
        if self._given:
            if len(offsets) != self.count:
                raise ValueError(f"{len(offsets)} offsets for {self.count} matrices")
            self._stride = self.cols if row_stride is None else int(row_stride)
            self._span = (max([int(o) for o in offsets], default=-1) + 1 +
                          max(self.rows - 1, 0) * self._stride + max(self.cols - 1, 0))
            if min(self.rows, self.cols, self.count) == 0:
                self._span = 0
            self._problem = dsm.make_ortho_problem(self.rows, self.cols, offsets,
                                                   row_stride=self._stride, **self._args)
        else:
            self._problem = dsm.make_ortho_problem(self.rows, self.cols, [0] * self.count,
                                                   **self._args)
        self._allocate(dsm.dsm_ortho_workspace(self._problem), device)

    def _placed(self, tensors):
        """The problem for these tensors' strides, which have to agree."""
        if self._given:
            for name, t in tensors:
                if t.device != self.device or t.dtype != self.dtype:
                    raise ValueError(f"{name} must be {self.dtype} on {self.device}, "
                                     f"got {t.dtype} on {t.device}")
                if not t.is_contiguous():
                    raise ValueError(f"{name} must be contiguous where offsets are given")
                if t.numel() < self._span:
                    raise ValueError(f"{name} holds {t.numel()} elements, the matrices reach "
                                     f"to {self._span}")
            return self._problem
        places = set()
        for name, t in tensors:
            shape = (self.count, self.rows, self.cols)
            if self.count == 1 and t.dim() == 2:
                t = t.unsqueeze(0)
            self._check(name, t, self.dtype, torch.Size(shape))
            if t.numel() == 0:
                continue
            if self.cols > 1 and t.stride(2) != 1:
                raise ValueError(f"{name}'s rows must be contiguous, got strides {t.stride()}")
            row = self.cols if self.rows == 1 else t.stride(1)
            each = 0 if self.count == 1 else t.stride(0)
            if row < self.cols:
                raise ValueError(f"{name}'s rows overlap: strides {t.stride()}")
            # Apart, or side by side as columns of a larger matrix.
            apart = each >= (self.rows - 1) * row + self.cols
            beside = each >= self.cols and (self.count - 1) * each + self.cols <= row
            if self.count > 1 and not apart and not beside:
                raise ValueError(f"{name}'s matrices overlap: strides {t.stride()}")
            places.add((row, each))
        if len(places) > 1:
            raise ValueError(f"the tensors' strides differ: {sorted(places)}")
        place = places.pop() if places else (self.cols, 0)
        if place not in self._problems:
            self._problems[place] = dsm.make_ortho_problem(
                self.rows, self.cols, [i * place[1] for i in range(self.count)],
                row_stride=place[0], **self._args)
        return self._problems[place]

    def _buffers(self, **pointers):
        buf = dsm.dsm_ortho_buffers(**{k: None if t is None else t.data_ptr()
                                       for k, t in pointers.items()})
        buf.workspace, buf.workspace_bytes = self.workspace.data_ptr(), self.workspace_bytes
        return buf

    def orthogonalize(self, u, out=None):
        """out (u itself, or a new tensor of u's layout) = the orthogonalised u."""
        if out is None:
            if self._given:
                raise ValueError("out is wanted where offsets are given (u itself will do)")
            out = torch.empty_strided(u.size(), u.stride(), dtype=u.dtype, device=u.device)
        problem = self._placed([("u", u), ("out", out)])
        buf = self._buffers(in_=u, out=out)
        with self._enqueue() as buf.stream:
            dsm.dsm_orthogonalize(problem, buf)
        return out

    def step(self, x, m, g, lr, mu, scale=1.0, wd=0.0, nesterov=True):
        """m <- mu m + g and x <- x - lr (scale O(u) + wd x), u = g + mu m or m; m
        may be None for u = g."""
        problem = self._placed([(n, t) for n, t in (("x", x), ("m", m), ("g", g)) if t is not None])
        buf = self._buffers(in_=g, m=m, x=x)
        with self._enqueue() as buf.stream:
            dsm.dsm_ortho_step(problem, buf, lr, mu, scale, wd, nesterov)

    def direction(self, m, g, out, mu, scale=1.0, nesterov=True):
        """m <- mu m + g and out (g itself will do) = scale O(u): a direction input
        for dsm_local_step."""
        problem = self._placed([(n, t) for n, t in (("m", m), ("g", g), ("out", out))
                                if t is not None])
        buf = self._buffers(in_=g, m=m, out=out)
        with self._enqueue() as buf.stream:
            dsm.dsm_ortho_step(problem, buf, 1.0, mu, scale, 0.0, nesterov)
        return out
