"""Device-memory plumbing around the binding: PyTorch is used only to allocate HBM buffers,
to copy layered numpy data in and out of the library's flat layouts, and for streams."""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import binding as B
from .workloads import Workload


ACTS = {"none": B.PG_ACT_NONE, "relu": B.PG_ACT_RELU, "gelu": B.PG_ACT_GELU, "silu": B.PG_ACT_SILU}
TYPES = {torch.float32: B.PG_F32, torch.bfloat16: B.PG_BF16}


class Checkpoint:
    """n x rows x cols activations in 8 bits: the device buffer `data` in the library's format."""

    def __init__(self, n: int, rows: int, cols: int, data: torch.Tensor):
        self.n, self.rows, self.cols, self.data = n, rows, cols, data


class _Here:
    """The current stream of the current device."""

    def __init__(self, stream: int):
        self.stream = stream

    def __enter__(self) -> int:
        return self.stream

    def __exit__(self, *exc):
        pass


class _There:
    """Another device, or a stream of its own."""

    def __init__(self, device, stream):
        self.device, self.other, self.stream = device, torch.cuda.device(device), torch.cuda.stream(stream)

    def __enter__(self) -> int:
        self.other.__enter__()
        self.stream.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *exc):
        self.stream.__exit__(*exc)
        self.other.__exit__(*exc)


class GossipBuffers:
    """Context + the caller-owned device buffers of one PowerGossip problem."""

    def __init__(self, n_workers, edges, edge_w, shapes, rank, power_steps, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("GossipBuffers needs a GPU: the PowerGossip path has no CPU fallback")
        self.shapes = [(int(p), int(q)) for p, q in shapes]
        self.n, self.n_edges, self.L = int(n_workers), int(np.asarray(edge_w).size), len(self.shapes)
        self.ctx = B.pg_init(n_workers, edges, edge_w, [s[0] for s in self.shapes],
                             [s[1] for s in self.shapes], rank, power_steps)
        self.device = torch.device(device)
        self.N = B.pg_param_floats(self.ctx)
        self.x = [torch.zeros(self.N, dtype=torch.float32, device=self.device) for _ in range(self.n)]
        self.q = torch.zeros(max(1, B.pg_qstate_floats(self.ctx)), dtype=torch.float32, device=self.device)
        self.ws = torch.zeros(B.pg_workspace_bytes(self.ctx), dtype=torch.uint8, device=self.device)
        assert self.ws.data_ptr() % 256 == 0
        self.ptrs = [t.data_ptr() for t in self.x]
        self.device = self.x[0].device
        self._tables = {}
        self.ranks = [B.pg_layer_rank(self.ctx, l) for l in range(self.L)]
        with torch.cuda.device(self.device):
            B.pg_upload(self.ctx)

    @classmethod
    def from_workload(cls, wl: Workload, device="cuda:0", fill=True):
        gb = cls(wl.n_workers, wl.edges, wl.edge_w, wl.shapes, wl.rank, wl.power_steps, device)
        if fill:
            gb.fill_from_workload(wl)
        return gb

    def close(self):
        if self.ctx:
            torch.cuda.synchronize()
            B.pg_destroy(self.ctx)
            self.ctx = None

    # ---- host <-> device, layer by layer --------------------------------
    def _layer_view(self, buf: torch.Tensor, l: int) -> torch.Tensor:
        """The p x q matrix of layer l inside a worker buffer (rows pg_layer_stride floats apart)."""
        p, q = self.shapes[l]
        off, ld = B.pg_layer_offset(self.ctx, l), B.pg_layer_stride(self.ctx, l)
        return buf[off:off + p * ld].view(p, ld)[:, :q]

    def layer_of(self, buf: torch.Tensor, l: int) -> torch.Tensor:
        """The same of every buffer in (..., pg_param_floats): a view (..., p, q)."""
        p, q = self.shapes[l]
        off, ld = B.pg_layer_offset(self.ctx, l), B.pg_layer_stride(self.ctx, l)
        return buf[..., off:off + p * ld].unflatten(-1, (p, ld))[..., :q]

    def set_layer(self, i: int, l: int, a: np.ndarray):
        p, q = self.shapes[l]
        self._layer_view(self.x[i], l).copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(p, q)))

    def get_layer(self, i: int, l: int) -> np.ndarray:
        return self._layer_view(self.x[i], l).cpu().numpy()

    def set_q(self, e: int, l: int, a: np.ndarray):
        r, q = self.ranks[l], self.shapes[l][1]
        off = B.pg_q_offset(self.ctx, e, l)
        self.q[off:off + r * q].copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(-1)))

    def get_q(self, e: int, l: int) -> np.ndarray:
        r, q = self.ranks[l], self.shapes[l][1]
        off = B.pg_q_offset(self.ctx, e, l)
        return self.q[off:off + r * q].cpu().numpy().reshape(r, q)

    def get_phat(self, e: int, l: int) -> np.ndarray:
        r, p = self.ranks[l], self.shapes[l][0]
        off = B.pg_ws_phat_offset(self.ctx, e, l)
        return self.ws[off:off + 4 * r * p].view(torch.float32).cpu().numpy().reshape(r, p)

    def get_flags(self, e: int, l: int) -> np.ndarray:
        off = B.pg_ws_flag_offset(self.ctx, e, l)
        return self.ws[off:off + 4 * self.ranks[l]].view(torch.int32).cpu().numpy()

    def fill_from_workload(self, wl: Workload, layers: Optional[Sequence[int]] = None):
        """Fill every worker's parameters and every edge's projection state from the seeded
        generator (all layers, or only the listed ones; the others stay zero)."""
        ls = range(self.L) if layers is None else layers
        for l in ls:
            base = wl.base(l)
            for i in range(self.n):
                self.set_layer(i, l, wl.worker_layer(i, l, base))
            for e in range(self.n_edges):
                self.set_q(e, l, wl.q_init(e, l))

    def fill_from_arrays(self, X, Q, layers: Optional[Sequence[int]] = None):
        """Fill from host arrays X[i][j] (p, q) and Q[e][j] (r, q) holding the listed layers
        (default: all, in order)."""
        ls = list(range(self.L)) if layers is None else list(layers)
        for j, l in enumerate(ls):
            for i in range(self.n):
                self.set_layer(i, l, X[i][j])
            for e in range(self.n_edges):
                self.set_q(e, l, Q[e][j])

    # ---- the two entry points -------------------------------------------
    def round(self, stream: Optional[torch.cuda.Stream] = None):
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        B.pg_round(self.ctx, self.ptrs, self.q.data_ptr(), self.ws.data_ptr(), s.cuda_stream)

    def round_static(self, stream: Optional[torch.cuda.Stream] = None):
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        B.pg_round_static(self.ctx, self.ptrs, self.q.data_ptr(), s.cuda_stream)

    def alloc_grads(self):
        """Gradient buffers laid out like the parameter buffers (zero-filled)."""
        self.g = [torch.zeros(self.N, dtype=torch.float32, device=self.device) for _ in range(self.n)]
        self.gptrs = [t.data_ptr() for t in self.g]

    def set_grad_layer(self, i: int, l: int, a: np.ndarray):
        p, q = self.shapes[l]
        self._layer_view(self.g[i], l).copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(p, q)))

    def round_sgd(self, eta: float, stream: Optional[torch.cuda.Stream] = None):
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        B.pg_round_sgd(self.ctx, self.ptrs, self.gptrs, eta, self.q.data_ptr(), self.ws.data_ptr(), s.cuda_stream)

    def alloc_pstate(self):
        """The R^p half of Algorithm 2's alternating vector (zero-filled)."""
        self.pstate = torch.zeros(max(1, B.pg_pstate_floats(self.ctx)), dtype=torch.float32, device=self.device)

    def set_p(self, e: int, l: int, a: np.ndarray):
        r, p = self.ranks[l], self.shapes[l][0]
        off = B.pg_p_offset(self.ctx, e, l)
        self.pstate[off:off + r * p].copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32).reshape(-1)))

    def get_p(self, e: int, l: int) -> np.ndarray:
        r, p = self.ranks[l], self.shapes[l][0]
        off = B.pg_p_offset(self.ctx, e, l)
        return self.pstate[off:off + r * p].cpu().numpy().reshape(r, p)

    def iterate(self, k_done: int, iterations: int, eta: Optional[float] = None,
                stream: Optional[torch.cuda.Stream] = None):
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        B.pg_iterate(self.ctx, self.ptrs, self.q.data_ptr(), self.pstate.data_ptr(), k_done, iterations,
                     None if eta is None else self.gptrs, 0.0 if eta is None else eta,
                     self.ws.data_ptr(), s.cuda_stream)

    def run(self, rounds: int, stream: Optional[torch.cuda.Stream] = None):
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        B.pg_run(self.ctx, self.ptrs, self.q.data_ptr(), self.ws.data_ptr(), s.cuda_stream, rounds)

    # ---- rows of activations ---------------------------------------------
    # Tensors of shape (n, rows, width), float32 or bfloat16, all of a call the same; elements of a row side by side, other strides as they
    # are (an input expanded over workers or rows is fine).  `counts`: int32 (n,) on the device, the rows that exist.  Layers by index.
    # Outputs not given are allocated; rows behind a worker's count stay as they were there (zero where allocated).

    def checkpoint(self, rows: int, cols: int) -> Checkpoint:
        nbytes = B.pg_checkpoint_bytes(self.ctx, rows, cols)
        if nbytes == (1 << 64) - 1:
            raise B.PGError(B.PG_ERR_ARG)
        return Checkpoint(self.n, rows, cols, torch.empty(max(1, nbytes), dtype=torch.uint8, device=self.device))

    def checkpoint_store(self, x: torch.Tensor, counts=None, out: Optional[Checkpoint] = None, stream=None) -> Checkpoint:
        with self._on(stream) as s:
            dtype, rows, cols = self._shape(x)
            if out is None:
                out = self.checkpoint(rows, cols)
                if counts is not None:
                    out.data.zero_()
            B.pg_checkpoint_store(self.ctx, rows, cols, self._counts(counts), TYPES[dtype], self._rows(x, rows, cols, dtype),
                                  self._kept(out, rows, cols), s)
        return out

    def checkpoint_load(self, kept: Checkpoint, dtype=None, counts=None, out=None, stream=None) -> torch.Tensor:
        """Its values in `dtype`: that of `out`, or bfloat16."""
        with self._on(stream) as s:
            dtype, rows, cols = self._shape(kept, dtype, out)
            out = self._out(out, rows, cols, dtype, counts)
            B.pg_checkpoint_load(self.ctx, rows, cols, self._counts(counts), TYPES[dtype], self._kept(kept, rows, cols),
                                 self._rows(out, rows, cols, dtype), s)
        return out

    def linear(self, l: int, x, bias: Optional[int] = None, act: str = "none", residual=None, keep: Optional[Checkpoint] = None, counts=None,
               out=None, dtype=None, stream=None) -> torch.Tensor:
        """act(x W^T + b) + residual; `keep` receives act's input.  x is a tensor or a Checkpoint (then `dtype`, or that of `out` or `residual`, is
        the result's)."""
        with self._on(stream) as s:
            p, q = self.shapes[l]
            dtype, rows, _ = self._shape(x, dtype, out, residual)
            out = self._out(out, rows, p, dtype, counts)
            ws = self._workspace(B.pg_linear_workspace_bytes(self.ctx, l, rows, TYPES[dtype]))
            x8 = isinstance(x, Checkpoint)
            B.pg_linear(self.ctx, self._table(self.ptrs), l, -1 if bias is None else bias, rows, self._counts(counts), TYPES[dtype],
                        None if x8 else self._rows(x, rows, q, dtype), self._kept(x, rows, q) if x8 else None, ACTS[act],
                        self._rows(residual, rows, p, dtype), self._rows(out, rows, p, dtype), self._kept(keep, rows, p), None if ws is None else ws.data_ptr(), s)
        return out

    def linear_backward(self, l: int, dz: torch.Tensor, x=None, bias: Optional[int] = None, act: str = "none", z: Optional[Checkpoint] = None,
                        residual=None, accumulate: bool = False, want_dx: bool = True, want_grads: bool = True, counts=None, out=None,
                        stream=None) -> Optional[torch.Tensor]:
        """Gradients of linear from that of its sum: those of weights and bias into the gradient buffers (`alloc_grads`), that of x, times
        act'(z) where x came out of an activation, plus `residual`, as the result."""
        with self._on(stream) as s:
            p, q = self.shapes[l]
            dtype, rows, _ = self._shape(dz)
            out = self._out(out, rows, q, dtype, counts) if want_dx else None
            ws = self._workspace(B.pg_linear_workspace_bytes(self.ctx, l, rows, TYPES[dtype]))
            x8 = isinstance(x, Checkpoint)
            B.pg_linear_backward(self.ctx, self._table(self.ptrs), self._table(self.gptrs) if want_grads else None, l, -1 if bias is None else bias, rows, self._counts(counts),
                                 TYPES[dtype], self._rows(dz, rows, p, dtype), None if x8 else self._rows(x, rows, q, dtype),
                                 self._kept(x, rows, q) if x8 else None, ACTS[act], self._kept(z, rows, q), self._rows(residual, rows, q, dtype),
                                 self._rows(out, rows, q, dtype), 1 if accumulate else 0, None if ws is None else ws.data_ptr(), s)
        return out

    def activation_backward(self, act: str, dy: torch.Tensor, z: Checkpoint, counts=None, out=None, stream=None) -> torch.Tensor:
        """dy act'(z)."""
        with self._on(stream) as s:
            dtype, rows, cols = self._shape(dy)
            out = self._out(out, rows, cols, dtype, counts)
            B.pg_activation_backward(self.ctx, rows, cols, self._counts(counts), TYPES[dtype], ACTS[act], self._rows(dy, rows, cols, dtype),
                                     self._kept(z, rows, cols), self._rows(out, rows, cols, dtype), s)
        return out

    def norm(self, l: int, x: torch.Tensor, residual=None, eps: float = 1e-6, keep: Optional[Checkpoint] = None, counts=None, out=None,
             sum_out=None, rstd_out=None, stream=None):
        """Root-mean-square norm of x + residual with layer l as gain: (y, the sum, rstd).  With `keep` the result goes there and y is None
        unless `out` is given; without a residual the sum is x, or a copy where `out` takes its place."""
        with self._on(stream) as s:
            dtype, rows, cols = self._shape(x)
            if keep is None or out is not None:
                out = self._out(out, rows, cols, dtype, counts)
            in_place = out is not None and out.data_ptr() == x.data_ptr()      # then x does not stay the sum
            if residual is not None or sum_out is not None or in_place:
                sum_out = self._out(sum_out, rows, cols, dtype, counts)
            if rstd_out is None:
                rstd_out = (torch.empty if counts is None else torch.zeros)(self.n, rows, device=self.device)
            elif rstd_out.shape != (self.n, rows) or rstd_out.dtype != torch.float32 or not rstd_out.is_contiguous() or rstd_out.device != self.device:
                raise ValueError("rstd: a contiguous float32 tensor of shape (workers, rows) on the buffers' device")
            if self.shapes[l] != (cols, 1):
                raise ValueError(f"layer {l} is no gain of {cols} entries")
            B.pg_norm(self.ctx, self._table(self.ptrs), l, rows, self._counts(counts), TYPES[dtype], eps, self._rows(x, rows, cols, dtype),
                      self._rows(residual, rows, cols, dtype), self._rows(sum_out, rows, cols, dtype), self._rows(out, rows, cols, dtype),
                      self._kept(keep, rows, cols), rstd_out.data_ptr(), s)
        return out, x if sum_out is None else sum_out, rstd_out

    def norm_backward(self, l: int, dy: torch.Tensor, total: torch.Tensor, rstd: torch.Tensor, residual=None, accumulate: bool = False,
                      want_grads: bool = True, counts=None, out=None, stream=None) -> torch.Tensor:
        """Gradient of the sum `total` that norm returned (plus `residual`); the gain's into the gradient buffers."""
        with self._on(stream) as s:
            dtype, rows, cols = self._shape(dy)
            if self.shapes[l] != (cols, 1):
                raise ValueError(f"layer {l} is no gain of {cols} entries")
            if rstd.shape != (self.n, rows) or rstd.dtype != torch.float32 or not rstd.is_contiguous() or rstd.device != self.device:
                raise ValueError("rstd: a contiguous float32 tensor of shape (workers, rows) on the buffers' device")
            out = self._out(out, rows, cols, dtype, counts)
            ws = self._workspace(B.pg_norm_workspace_bytes(self.ctx, l, rows)) if want_grads else None
            B.pg_norm_backward(self.ctx, self._table(self.ptrs), self._table(self.gptrs) if want_grads else None, l, rows, self._counts(counts), TYPES[dtype],
                               self._rows(dy, rows, cols, dtype), self._rows(total, rows, cols, dtype), rstd.data_ptr(),
                               self._rows(residual, rows, cols, dtype), self._rows(out, rows, cols, dtype), 1 if accumulate else 0,
                               None if ws is None else ws.data_ptr(), s)
        return out

    def _on(self, stream):
        """The buffers' device and the caller's stream: what is allocated inside belongs to that stream."""
        if stream is None and torch.cuda.current_device() == self.device.index:
            return _Here(torch.cuda.current_stream(self.device.index).cuda_stream)
        return _There(self.device, stream)

    def _table(self, ptrs):
        """The addresses as the library takes them, made again only when they change."""
        key = tuple(ptrs)
        if key not in self._tables:
            if len(self._tables) >= 16:
                self._tables.clear()
            self._tables[key] = B.ptr_table(key)
        return self._tables[key]

    def _workspace(self, nbytes: int) -> Optional[torch.Tensor]:
        """A workspace of the call's own: no two calls, or graphs of them, share one."""
        if nbytes == (1 << 64) - 1:
            raise B.PGError(B.PG_ERR_ARG)
        return torch.empty(nbytes, dtype=torch.uint8, device=self.device) if nbytes else None

    def _shape(self, x, dtype=None, *others):
        """(type, rows, width) of the leading argument; a Checkpoint's type is the one asked for, or that of the others."""
        if isinstance(x, Checkpoint):
            given = [dtype] + [o.dtype for o in others if o is not None]
            return self._type(next((t for t in given if t is not None), torch.bfloat16)), x.rows, x.cols
        if x.dim() != 3:
            raise ValueError(f"rows of activations have three dimensions, not {x.dim()}")
        if dtype is not None and dtype != x.dtype:
            raise ValueError(f"the result has the type of its rows, {x.dtype}, not {dtype}")
        return self._type(x.dtype), x.shape[1], x.shape[2]

    @staticmethod
    def _type(dtype):
        if dtype not in TYPES:
            raise TypeError(f"activations are float32 or bfloat16, not {dtype}")
        return dtype

    def _rows(self, x, rows: int, cols: int, dtype):
        if x is None:
            return None
        if x.dtype != dtype or x.device != self.device or x.shape != (self.n, rows, cols):
            raise ValueError(f"rows of activations: {tuple(x.shape)} {x.dtype} on {x.device}, wanted {(self.n, rows, cols)} {dtype} on {self.device}")
        worker, row, one = x.stride()
        if cols > 1 and one != 1:
            raise ValueError("elements of a row lie side by side")
        return B.pg_rows(x.data_ptr(), row if rows > 1 else 0, worker if self.n > 1 else 0)

    def _kept(self, kept: Optional[Checkpoint], rows: int, cols: int):
        if kept is None:
            return None
        if (kept.n, kept.rows, kept.cols) != (self.n, rows, cols) or kept.data.device != self.device:
            raise ValueError(f"checkpoint of {(kept.n, kept.rows, kept.cols)} on {kept.data.device}, wanted {(self.n, rows, cols)} on {self.device}")
        if kept.data.dtype != torch.uint8 or not kept.data.is_contiguous() or kept.data.numel() < B.pg_checkpoint_bytes(self.ctx, rows, cols):
            raise ValueError(f"checkpoint of {(kept.n, kept.rows, kept.cols)}: its data are pg_checkpoint_bytes contiguous bytes")
        return kept.data.data_ptr()

    def _counts(self, counts):
        if counts is None:
            return None
        if counts.dtype != torch.int32 or counts.shape != (self.n,) or not counts.is_contiguous() or counts.device != self.device:
            raise ValueError("counts: a contiguous int32 tensor of one entry per worker on the buffers' device")
        return counts.data_ptr()

    def _out(self, out, rows: int, cols: int, dtype, counts):
        if out is not None:
            return out
        make = torch.empty if counts is None else torch.zeros
        return make(self.n, rows, cols, dtype=dtype, device=self.device)
