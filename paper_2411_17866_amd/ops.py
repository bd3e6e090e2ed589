"""Language-model operators on torch tensors: the output layer's cross entropy
with its gradients, orthogonalised updates, and what a model's blocks take up to the
gradients of a local step: the linear layer, the norms around a block, clipping.

PyTorch only allocates device memory and supplies the stream; the operators run
in libdsm.so through the binding in ``dsm``.  An object here is the plan of one
problem: it checks tensors, keeps the workspace, and enqueues on torch's current
stream.  Calls of one object share its workspace: on different streams they are put
one after another (under graph capture that is the caller's part, as is keeping the
object while the graph is replayed), and from several threads each call's launches are
enqueued whole before the next call's.
"""
import contextlib
import operator
import threading

import numpy as np
import torch

from . import dsm

DTYPES = {torch.float32: dsm.DSM_F32, torch.bfloat16: dsm.DSM_BF16}


# The current stream's handle without a Stream object around it (a microsecond of a call), and the
# current device without looking whether the GPU has been initialised: the plan has done that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _dtype(dtype):
    if dtype not in DTYPES:
        raise ValueError(f"dtype must be torch.float32 or torch.bfloat16, got {dtype}")
    return DTYPES[dtype]


class _Plan:
    _index = -1  # of the device, as Tensor.get_device gives it

    def __init__(self):
        self._lock = threading.Lock()

    def _allocate(self, workspace_bytes, device):
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError(f"the operators run on a GPU, got device {device}")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self._index = self.device.index
        self.workspace_bytes = workspace_bytes
        self.workspace = torch.empty(max(workspace_bytes, 256), dtype=torch.uint8,
                                     device=self.device)
        self._stream = torch.cuda.current_stream(self.device)
        self._handle = self._stream.cuda_stream

    def _enter(self):
        """The current stream, after what this plan last did on another one."""
        if _raw_stream is not None and self._index >= 0 and _raw_stream(self._index) == self._handle:
            return self._handle
        stream = torch.cuda.current_stream(self.device)
        if stream != self._stream:
            if not torch.cuda.is_current_stream_capturing():
                stream.wait_stream(self._stream)
                self.workspace.record_stream(stream)
            self._stream = stream
        self._handle = stream.cuda_stream
        return self._handle

    def _on_device(self):
        if torch.cuda.current_device() == self.device.index:
            return contextlib.nullcontext()
        return torch.cuda.device(self.device)

    def _launch(self, call):
        """call(stream): one call's launches, which no other call's come between."""
        with self._lock:
            if _device() == self._index:
                call(self._enter())
            else:
                with torch.cuda.device(self.device):
                    call(self._enter())

    def _launch_with(self, entry, problem, buf):
        """entry(problem, buf) on the current stream, as _launch."""
        with self._lock:
            if _device() == self._index:
                buf.stream = self._enter()
                entry(problem, buf)
            else:
                with torch.cuda.device(self.device):
                    buf.stream = self._enter()
                    entry(problem, buf)

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

    def _rows(self, name, t, shape, dtype=None):
        """The stride of a matrix with contiguous rows."""
        self._check(name, t, self.dtype if dtype is None else dtype, shape)
        if shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}'s rows must be contiguous, got strides {t.stride()}")
        if shape[0] <= 1:
            return shape[1]
        if t.stride(0) < shape[1]:
            raise ValueError(f"{name}'s rows overlap: strides {t.stride()}")
        return t.stride(0)

    def _matrix(self, name, t, shape, dtype=None):
        """(address, stride) of a matrix with contiguous rows."""
        dtype = self.dtype if dtype is None else dtype
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index:
            self._check(name, t, dtype, shape)
        return t.data_ptr(), shape[1] if t.is_contiguous() else self._rows(name, t, shape, dtype)

    def _vector(self, name, t, dtype, shape):
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index:
            self._check(name, t, dtype, shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()


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


ACTS = {"none": dsm.DSM_ACT_NONE, "relu": dsm.DSM_ACT_RELU, "gelu": dsm.DSM_ACT_GELU,
        "gelu_tanh": dsm.DSM_ACT_GELU_TANH, "silu": dsm.DSM_ACT_SILU}
NORMS = {"none": dsm.DSM_NORM_NONE, "layer": dsm.DSM_NORM_LAYER, "rms": dsm.DSM_NORM_RMS}


def _named(table, what, name):
    if name not in table:
        raise ValueError(f"{what} must be one of {', '.join(table)}, got {name!r}")
    return table[name]


class Linear(_Plan):
    """A linear layer with bias, activation and residual, and its gradients (dsm_linear,
    dsm_linear_backward).

    tokens, dim, wide: the sizes of x (tokens, dim), w (wide, dim) and y (tokens, wide);
    dtype: of all of them, torch.float32 or torch.bfloat16; act: "none", "relu", "gelu",
    "gelu_tanh" or "silu"; grads: whether backward is called too; dw_dtype: of dw, dtype
    or torch.float32, as the arenas keep gradients.  Biases and their gradients are fp32.
    """

    def __init__(self, tokens, dim, wide, dtype=torch.float32, act="none", grads=True, dw_dtype=None, device="cuda"):
        super().__init__()
        self.dtype, self.dw_dtype = dtype, dtype if dw_dtype is None else dw_dtype
        self.act, self.grads = act, bool(grads)
        self.problem = dsm.dsm_linear_problem(int(tokens), int(dim), int(wide), _dtype(dtype), _named(ACTS, "act", act),
                                              _dtype(self.dw_dtype), 1 if grads else 0)
        self.x_shape = torch.Size((int(tokens), int(dim)))
        self.w_shape = torch.Size((int(wide), int(dim)))
        self.y_shape = torch.Size((int(tokens), int(wide)))
        self.bias_shape = self.w_shape[:1]
        self._allocate(dsm.dsm_linear_workspace(self.problem), device)

    def _empty(self, shape, dtype=None):
        return torch.empty(shape, dtype=self.dtype if dtype is None else dtype, device=self.device)

    def _buffers(self):
        return dsm.dsm_linear_buffers(workspace=self.workspace.data_ptr(), workspace_bytes=self.workspace_bytes)

    def __call__(self, x, w, bias=None, residual=None, y=None, z=None):
        """{"y"}: act(x w^T + bias) + residual; and, for a plan with gradients and an
        activation or where z is given, {"z"}: x w^T + bias, which backward takes.  Outputs
        are written into the tensors given (y may be the residual), or into new ones."""
        buf = self._buffers()
        buf.x, buf.x_stride = self._matrix("x", x, self.x_shape)
        buf.w, buf.w_stride = self._matrix("w", w, self.w_shape)
        if bias is not None:
            buf.bias = self._vector("bias", bias, torch.float32, self.bias_shape)
        if residual is not None:
            buf.residual, buf.residual_stride = self._matrix("residual", residual, self.y_shape)
        if y is None:
            y = self._empty(self.y_shape)
        if z is None and self.grads and self.act != "none":
            z = torch.empty_like(y)
        buf.y, buf.y_stride = self._matrix("y", y, self.y_shape)
        out = {"y": y}
        if z is not None:
            buf.z, buf.z_stride = self._matrix("z", z, self.y_shape)
            out["z"] = z
        self._launch_with(dsm.dsm_linear, self.problem, buf)
        return out

    def backward(self, dy, x=None, w=None, z=None, dx=None, dw=None, dbias=None, wanted=("dx", "dw", "dbias")):
        """The gradients named in `wanted`, {"dx", "dw", "dbias"}, from y's gradient dy and
        what the forward pass had: x (for dw), w (for dx), and z unless there is no
        activation.  (The residual's gradient is dy.)  Outputs are written into the tensors
        given, or into new ones."""
        if not self.grads:
            raise ValueError("the plan is without gradients")
        for name, t in (("dx", dx), ("dw", dw), ("dbias", dbias)):
            if t is not None and name not in wanted:
                raise ValueError(f"{name} is given but not wanted")
        for name in wanted:
            if name not in ("dx", "dw", "dbias"):
                raise ValueError(f"wanted holds {name!r}")
        for name, t, needed in (("x", x, "dw" in wanted), ("w", w, "dx" in wanted), ("z", z, self.act != "none")):
            if t is None and needed:
                raise ValueError(f"{name} is wanted for these gradients")
        buf = self._buffers()
        if x is not None:
            buf.x, buf.x_stride = self._matrix("x", x, self.x_shape)
        if w is not None:
            buf.w, buf.w_stride = self._matrix("w", w, self.w_shape)
        buf.dy, buf.dy_stride = self._matrix("dy", dy, self.y_shape)
        if self.act != "none":
            buf.z, buf.z_stride = self._matrix("z", z, self.y_shape)
        out = {}
        if "dx" in wanted:
            if dx is None:
                dx = self._empty(self.x_shape) if x is None else torch.empty_like(x)
            out["dx"] = dx
            buf.dx, buf.dx_stride = self._matrix("dx", dx, self.x_shape)
        if "dw" in wanted:
            if dw is None:
                dw = self._empty(self.w_shape, self.dw_dtype) if w is None else torch.empty_like(w, dtype=self.dw_dtype)
            out["dw"] = dw
            buf.dw, buf.dw_stride = self._matrix("dw", dw, self.w_shape, self.dw_dtype)
        if "dbias" in wanted:
            out["dbias"] = dbias = self._empty(self.bias_shape, torch.float32) if dbias is None else dbias
            buf.dbias = self._vector("dbias", dbias, torch.float32, self.bias_shape)
        self._launch_with(dsm.dsm_linear_backward, self.problem, buf)
        return out


class ResidualNorm(_Plan):
    """The norms before and after a block, fused with its gate and residual scale, and
    their gradients (dsm_residual_norm, dsm_residual_norm_backward):

        p = post(f);  s = h + scale gate p;  y = norm(s)

    tokens, dim, dtype: of the rows h, f, s, y and their gradients; norm, post: "layer",
    "rms" or "none"; eps, post_eps (eps where None): of them; grads: whether backward is
    called too.  Vectors and their gradients are fp32.
    """

    def __init__(self, tokens, dim, dtype=torch.float32, norm="layer", post="none", eps=1e-5, post_eps=None, grads=True,
                 device="cuda"):
        super().__init__()
        self.dtype, self.norm, self.post, self.grads = dtype, norm, post, bool(grads)
        self.shape = torch.Size((int(tokens), int(dim)))
        self.vector_shape = self.shape[1:]
        self._args = (int(tokens), int(dim), _dtype(dtype), _named(NORMS, "norm", norm), _named(NORMS, "post", post),
                      1 if grads else 0, float(eps), float(eps if post_eps is None else post_eps))
        self._scaled = 1.0, dsm.dsm_norm_problem(*self._args, 1.0)
        self._allocate(dsm.dsm_norm_workspace(self._scaled[1]), device)

    def _problem(self, scale):
        last = self._scaled
        if last[0] != scale:
            self._scaled = last = scale, dsm.dsm_norm_problem(*self._args, float(scale))
        return last[1]

    def _buffers(self, f, gate, weight, bias, post_weight, post_bias):
        """With the vectors, of those that the kinds of norms have."""
        if self.norm == "none" and (weight is not None or bias is not None):
            raise ValueError("weight or bias is given without a norm")
        if self.post == "none":
            if post_weight is not None or post_bias is not None:
                raise ValueError("post_weight or post_bias is given without a post norm")
        elif f is None:
            raise ValueError("f is None: there is no block's output for post")
        if f is None and gate is not None:
            raise ValueError("f is None: there is no block's output for gate")
        buf = dsm.dsm_norm_buffers(workspace=self.workspace.data_ptr(), workspace_bytes=self.workspace_bytes)
        if weight is not None:
            buf.weight = self._vector("weight", weight, torch.float32, self.vector_shape)
        if bias is not None:
            buf.bias = self._vector("bias", bias, torch.float32, self.vector_shape)
        if gate is not None:
            buf.gate = self._vector("gate", gate, torch.float32, self.vector_shape)
        if post_weight is not None:
            buf.post_weight = self._vector("post_weight", post_weight, torch.float32, self.vector_shape)
        if post_bias is not None:
            buf.post_bias = self._vector("post_bias", post_bias, torch.float32, self.vector_shape)
        if f is not None:
            buf.f, buf.f_stride = self._matrix("f", f, self.shape)
        return buf

    def __call__(self, h, f=None, weight=None, bias=None, gate=None, scale=1.0, post_weight=None, post_bias=None, s=None,
                 y=None):
        """{"s", "y"}: s where there is f, y where there is a norm; written into the tensors
        given (s may be h or f, y h or f), or into new ones.  Absent weights and gate are 1, absent
        biases 0."""
        buf = self._buffers(f, gate, weight, bias, post_weight, post_bias)
        if f is None and s is not None:
            raise ValueError("f is None: s is h")
        if y is not None and self.norm == "none":
            raise ValueError("y is given without a norm")
        buf.h, buf.h_stride = self._matrix("h", h, self.shape)
        out = {}
        if f is not None:
            out["s"] = s = torch.empty_like(h) if s is None else s
            buf.s, buf.s_stride = self._matrix("s", s, self.shape)
        if self.norm != "none":
            out["y"] = y = torch.empty_like(h) if y is None else y
            buf.y, buf.y_stride = self._matrix("y", y, self.shape)
        self._launch_with(dsm.dsm_residual_norm, self._problem(scale), buf)
        return out

    def backward(self, dy, s, f=None, ds=None, weight=None, bias=None, gate=None, scale=1.0, post_weight=None,
                 post_bias=None, dh=None, df=None, dweight=None, dbias=None, dgate=None, dpost_weight=None,
                 dpost_bias=None):
        """The gradients of what the forward pass was given: {"dh"}, {"df"} where there is f,
        and those of the vectors given.  dy: y's gradient (None without a norm); s: the
        forward pass's s, or h where there was no f; ds: the gradient that s has from
        elsewhere, or None.  Outputs are written into the tensors given (dh may be dy or ds,
        df dy, ds or f), or into new ones."""
        if not self.grads:
            raise ValueError("the plan is without gradients")
        buf = self._buffers(f, gate, weight, bias, post_weight, post_bias)
        if f is None and df is not None:
            raise ValueError("f is None: there is no df")
        if (dy is None) != (self.norm == "none"):
            raise ValueError("dy is wanted where there is a norm, and only there")
        if dy is None and ds is None:
            raise ValueError("ds is wanted where there is no norm")
        if dy is not None:
            buf.h, buf.h_stride = self._matrix("s", s, self.shape)
            buf.dy, buf.dy_stride = self._matrix("dy", dy, self.shape)
        if ds is not None:
            buf.ds, buf.ds_stride = self._matrix("ds", ds, self.shape)
        like = dy if ds is None else ds
        out = {"dh": torch.empty_like(like) if dh is None else dh}
        buf.dh, buf.dh_stride = self._matrix("dh", out["dh"], self.shape)
        if f is not None:
            out["df"] = torch.empty_like(like) if df is None else df
            buf.df, buf.df_stride = self._matrix("df", out["df"], self.shape)
        for name, t, given in (("dweight", weight, dweight), ("dbias", bias, dbias), ("dgate", gate, dgate),
                               ("dpost_weight", post_weight, dpost_weight), ("dpost_bias", post_bias, dpost_bias)):
            if t is not None:
                out[name] = given = torch.empty_like(t) if given is None else given
                setattr(buf, name, self._vector(name, given, torch.float32, self.vector_shape))
            elif given is not None:
                raise ValueError(f"{name} is given without {name[1:]}")
        self._launch_with(dsm.dsm_residual_norm_backward, self._problem(scale), buf)
        return out


class _Clip(_Plan):
    def _table(self, sizes, groups, n_groups, eps, device):
        """sizes: [(numel, dtype)]; the tensors' table, whose addresses each call fills."""
        self._entries = (dsm.dsm_clip_tensor * len(sizes))()
        for e, (numel, dtype), group in zip(self._entries, sizes, groups):
            e.numel, e.block, e.stride, e.dtype, e.group = numel, max(numel, 1), max(numel, 1), _dtype(dtype), group
        # The same memory as columns, to fill at once.
        self._columns = np.frombuffer(self._entries, dtype=np.int64).reshape(len(sizes), -1).T if sizes else None
        self._placed = None
        self.n_groups, self.eps = int(n_groups), float(eps)
        self._allocate(dsm.dsm_clip_workspace(self._entries, self.n_groups), device)

    def _norm(self, norm):
        if norm is None:
            return torch.empty(self.n_groups, dtype=torch.float32, device=self.device)
        self._vector("norm", norm, torch.float32, torch.Size((self.n_groups,)))
        return norm

    def _run(self, max_norm, norm, data, columns):
        """data: addresses; columns: first, block and stride where they differ from what stands there (a
        dictionary that the last call gave stands there)."""
        def call(stream):
            if self._columns is not None:
                self._columns[0] = data
                if columns is not self._placed:
                    self._placed = columns
                    for name, values in columns.items():
                        self._columns[_COLUMNS[name]] = values
            dsm.dsm_grad_clip(self._entries, self.n_groups, float("inf") if max_norm is None else float(max_norm),
                              norm.data_ptr(), self.workspace.data_ptr(), self.workspace_bytes, self.eps, stream)

        self._launch(call)
        return norm


# The words of a dsm_clip_tensor.
_COLUMNS = {"data": 0, "first": 1, "numel": 2, "block": 3, "stride": 4}
_SHAPE_DTYPE = operator.attrgetter("shape", "dtype")


class GradClip(_Clip):
    """Clipping of gradients by the global norm of a list of tensors, or of each group of
    them (dsm_grad_clip).

    tensors: tensors (or anything with their shape and dtype) of the sizes that calls
    take; groups: the group of each, 0 .. n - 1 (None: one group); eps: added to the norm.
    """

    def __init__(self, tensors, groups=None, eps=1e-6, device="cuda"):
        super().__init__()
        tensors = list(tensors)
        groups = [0] * len(tensors) if groups is None else [int(g) for g in groups]
        if len(groups) != len(tensors):
            raise ValueError(f"{len(groups)} groups for {len(tensors)} tensors")
        if any(g < 0 for g in groups):
            raise ValueError("a group is negative")
        self._like = [(torch.Size(t.shape), t.dtype) for t in tensors]
        # Groups in order: the order of a call's tensors is the caller's.
        self._order = sorted(range(len(tensors)), key=groups.__getitem__)
        sizes = [(self._like[i][0].numel(), self._like[i][1]) for i in self._order]
        whole = np.array([max(n, 1) for n, _ in sizes], dtype=np.int64)
        self._whole = {"block": whole, "stride": whole}
        self._table(sizes, [groups[i] for i in self._order], max(groups, default=0) + 1, eps, device)

    def _place(self, i, t):
        """(block, stride) of tensor i, checked."""
        shape, dtype = self._like[i]
        if t.shape != shape or t.dtype != dtype or t.device != self.device:
            raise ValueError(f"tensors[{i}] must be {dtype} of shape {tuple(shape)} on {self.device}, "
                             f"got {t.dtype}, {tuple(t.shape)}, {t.device}")
        if t.is_contiguous():
            return max(t.numel(), 1), max(t.numel(), 1)
        if t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1) and t.stride(0) >= t.shape[1]:
            return t.shape[1], t.stride(0)
        raise ValueError(f"tensors[{i}] has neither contiguous elements nor contiguous rows: strides {t.stride()}")

    def __call__(self, tensors, max_norm=None, norm=None):
        """norm (n_groups,): the groups' norms, before clipping.  Where one exceeds max_norm its
        tensors are scaled to it in place (None: norms alone).  Tensors have contiguous elements,
        or are matrices with contiguous rows.  They may not overlap."""
        if len(tensors) != len(self._like):
            raise ValueError(f"{len(tensors)} tensors for a plan of {len(self._like)}")
        # Hundreds of tensors: no Python code for each where all is well.
        if (list(map(_SHAPE_DTYPE, tensors)) == self._like and all(map(torch.Tensor.is_contiguous, tensors)) and
                set(map(torch.Tensor.get_device, tensors)) <= {self._index}):
            place = self._whole
        else:
            places = [self._place(i, tensors[i]) for i in self._order]
            place = {"block": [p[0] for p in places], "stride": [p[1] for p in places]}
        data = list(map(torch.Tensor.data_ptr, map(tensors.__getitem__, self._order)))
        if len(set(data)) < len(data):  # (tensors without elements may share an address)
            given = [a for a, i in zip(data, self._order) if tensors[i].numel()]
            if len(set(given)) < len(given):
                raise ValueError("a tensor is given twice")
        return self._run(max_norm, self._norm(norm), data, place)


class ArenaClip(_Clip):
    """Clipping of the workers' gradients in an ``arena.Arenas`` by the global norm of each
    worker's tensors, or of all workers' together; padding between tensors does not count."""

    def __init__(self, arenas, together=False, eps=1e-6):
        super().__init__()
        self._n, self._numel = arenas.n, list(arenas.numel)
        self._offsets = [int(o) for o in arenas.offsets]
        self._layout = (arenas.replica_layout, arenas.n_state_buffers, arenas.arena_elems)
        count = len(self._numel)
        self._table([(n, torch.float32) for n in self._numel] * self._n,
                    [0 if together else i for i in range(self._n) for _ in range(count)], 1 if together else self._n, eps,
                    arenas.x.device)

    def __call__(self, arenas, max_norm=None, norm=None):
        """norm: (n_workers,), or (1,) together; as GradClip's."""
        if (arenas.n, list(arenas.numel), (arenas.replica_layout, arenas.n_state_buffers, arenas.arena_elems)) != (
                self._n, self._numel, self._layout):
            raise ValueError("the plan is for arenas of another problem")
        if arenas.g_rep.device != self.device:
            raise ValueError(f"the arenas are on {arenas.g_rep.device}, the plan on {self.device}")
        layout, buffers, elems = self._layout
        block = stride = apart = max(elems, 1)  # apart: elements from one worker's copy to the next
        if layout == dsm.DSM_REPLICAS_STATE_BLOCKED:
            block = apart = dsm.DSM_STATE_BLOCK_ELEMS
            stride = buffers * self._n * block
        data = arenas.g_rep.data_ptr() + 4 * apart * np.arange(self._n, dtype=np.int64).repeat(len(self._numel))
        first = np.tile(np.array(self._offsets, dtype=np.int64), self._n)
        return self._run(max_norm, self._norm(norm), data, {"first": first, "block": block, "stride": stride})
