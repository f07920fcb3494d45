"""Residual blocks on node embeddings: a head over the rows that a partition's features or a layer's activations are, trained and served with
the operators of residual blocks (``grappa.h``).

A block is pre-norm:  h = x + r,  out = h + act(norm(h) W1 + b1) W2 + b2, where r is the block's own output of before (the norm adds it).
Activations and the weights' copies are bf16, master weights, gradients and the optimizer's moments fp32 (one flat vector each, as
``grp_optimizer_step`` takes them): h, each block's output and the gradient that runs through them are rounded to bf16 at every block.  ``serve`` runs the products in
8 bits, with weights quantized once, by the 8-bit matrix instructions, whose sums are shorter than fp32 (``grp_linear`` in ``grappa.h``).

Parameters are set by writing into ``theta`` or its views ``params``: the next ``forward`` or ``serve`` makes the weights' copies anew.  That goes by torch's own
count of writes, which a kernel (``grp_optimizer_step`` on ``theta``), a collective, a replayed graph and ``.data`` pass by: ``refresh()`` has to follow these.  A captured pass
reads the copies at their places, as they are when it is replayed: after a write, ``refresh()`` comes before the replay.

Streams: ``forward``, ``backward`` and ``step`` work on what the object keeps, so they are ordered one after another by the caller, as calls on one stream are.
``serve`` keeps nothing of a call: several may run side by side on streams of their own, after the writes of ``theta`` (the constructor's, ``step``'s) and
before the next; the 8-bit weights that the first one makes are waited for by the others.  A capture does not wait: a ``serve`` goes before it.  The object
outlives the work on all of them.
"""
from __future__ import annotations

import torch

from . import binding as g


class ResidualBlocks:
    """``depth`` blocks of width ``dim`` with ``hidden`` units each, for at most ``rows`` rows at a time."""

    @torch.inference_mode(False)        # (tensors of inference mode have no count of writes)
    def __init__(self, dim: int, hidden: int, depth: int, rows: int, act: int = g.ACT_GELU, eps: float = 1e-6, seed: int = 0, device="cuda"):
        if dim < 1 or hidden < 1 or depth < 1 or rows < 1:
            raise ValueError("dim, hidden, depth and rows must be positive")
        self.dim, self.hidden, self.depth, self.rows, self.act, self.eps = dim, hidden, depth, rows, act, eps
        shapes = [(dim,), (dim, hidden), (hidden,), (hidden, dim), (dim,)]            # norm, W1, b1, W2, b2
        sizes = [torch.Size(s).numel() for s in shapes]
        total = depth * sum(sizes)
        self._theta = torch.zeros(total, device=device)
        self.grad, self.m, self.v = (torch.zeros_like(self.theta) for _ in range(3))
        self.steps = 0

        def views(flat):
            parts = [p.view(s) for p, s in zip(flat.split(sizes * depth), shapes * depth)]
            return [tuple(parts[5 * i:5 * i + 5]) for i in range(depth)]

        self.params, self.grads = views(self.theta), views(self.grad)
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        for p in self.params:
            p[0].fill_(1.0)
            p[1].copy_(torch.randn(dim, hidden, generator=gen, device=device) * dim ** -0.5)
            p[3].copy_(torch.randn(hidden, dim, generator=gen, device=device) * hidden ** -0.5 / depth)
        bf = dict(device=device, dtype=torch.bfloat16)
        self.w1, self.w2 = [torch.empty(dim, hidden, **bf) for _ in range(depth)], [torch.empty(hidden, dim, **bf) for _ in range(depth)]
        self._served, self._quantized, self._made = None, None, None
        self._round_weights()
        self._kept = None                   # rows of the last forward pass
        # kept by forward for backward, per block: h, norm(h), the pre-activation and the activation; what a block adds to h
        self.h, self.y, self.out = ([torch.empty(rows, dim, **bf) for _ in range(depth)] for _ in range(3))
        self.z, self.a = ([torch.empty(rows, hidden, **bf) for _ in range(depth)] for _ in range(2))
        self.dh, self.dy, self.dz = torch.empty(rows, dim, **bf), torch.empty(rows, dim, **bf), torch.empty(rows, hidden, **bf)
        self.norm = torch.zeros(1, device=device)
        self.gradients = g.grp_gradients_create([self.grad])

    @property
    def theta(self) -> torch.Tensor:
        """All parameters, fp32; to be written into (``theta.copy_(saved)``), not replaced."""
        return self._theta

    def refresh(self):
        """Makes the weights' copies anew: to be called after ``theta`` was written by what torch does not see."""
        self._round_weights()
        self._quantized = None
        if self._served is not None:
            self._weights8()

    def _seen(self):
        """The count of writes of ``theta`` that copies made now have seen: none where a graph is captured, which makes them at its replays."""
        return None if self.theta.is_cuda and torch.cuda.is_current_stream_capturing() else self.theta._version

    def _round_weights(self):
        for i, p in enumerate(self.params):
            self.w1[i].copy_(p[1])
            self.w2[i].copy_(p[3])
        self._rounded = self._seen()

    def _room(self, nbytes: int):
        """A workspace for the calls that follow on the current stream (kept by a graph that is captured as long as it lives)."""
        return torch.empty(nbytes, dtype=torch.uint8, device=self.theta.device) if nbytes else None

    def _linear(self, m, n, k, a, w, bias, act, r, c, z):
        ws = self._room(g.grp_linear_workspace_bytes(g.LINEAR_FORWARD, m, n, k, g.DTYPE_BF16))
        g.grp_linear(m, n, k, a, k, w, n, g.DTYPE_BF16, None, None, bias, act, r, n, c, n, g.DTYPE_BF16, z, n, ws)

    def _check(self, x):
        if x.dtype != torch.bfloat16 or x.dim() != 2 or x.shape[1] != self.dim or x.shape[0] > self.rows or not x.is_contiguous() or x.device != self.theta.device:
            raise ValueError(f"rows of {self.dim} bfloat16 numbers are needed, at most {self.rows}, contiguous, on {self.theta.device}")
        return x.shape[0]

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """``x``: bf16 [m x dim]; the result is kept until the next call."""
        m, d, f = self._check(x), self.dim, self.hidden
        self._kept = None
        if self._rounded != self.theta._version:
            self._round_weights()
        for i, p in enumerate(self.params):
            # the first block's input has nothing added; the others add what the block before made to its h
            src, add = (x, None) if i == 0 else (self.out[i - 1], self.h[i - 1])
            g.grp_rmsnorm(m, d, src, d, g.DTYPE_BF16, add, d, p[0], self.eps, self.h[i], d, self.y[i], d, g.DTYPE_BF16)
            self._linear(m, f, d, self.y[i], self.w1[i], p[2], self.act, None, self.a[i], self.z[i])
            last = i == self.depth - 1
            self._linear(m, d, f, self.a[i], self.w2[i], p[4], g.ACT_NONE, self.h[i] if last else None, self.out[i], None)
        self._kept = m
        return self.out[-1][:m]

    def backward(self, dout: torch.Tensor) -> torch.Tensor:
        """Gradients of the parameters (``grad``) and of ``x`` from the result's, for the rows of the last ``forward``, as many as it had."""
        m, d, f = self._check(dout), self.dim, self.hidden
        if m != self._kept:
            raise ValueError(f"the gradient has {m} rows, the last forward pass {'was not made' if self._kept is None else f'had {self._kept}'}")
        self.dh[:m].copy_(dout)
        bytes_ = [g.grp_linear_workspace_bytes(kind, m, *nk, g.DTYPE_BF16) for kind in (g.LINEAR_DX, g.LINEAR_DW) for nk in ((d, f), (f, d))]
        ws = self._room(max(bytes_ + [g.grp_rmsnorm_backward_workspace_bytes(m, d)]))
        for i in reversed(range(self.depth)):
            p, q = self.params[i], self.grads[i]
            g.grp_linear_dx(m, d, f, self.dh, d, self.w2[i], d, self.act, self.z[i], f, self.dz, f, g.DTYPE_BF16, ws)
            g.grp_linear_dw(m, d, f, self.a[i], f, self.dh, d, q[3], d, q[4], ws)
            g.grp_linear_dx(m, f, d, self.dz, f, self.w1[i], f, g.ACT_NONE, None, 0, self.dy, d, g.DTYPE_BF16, ws)
            g.grp_linear_dw(m, f, d, self.y[i], d, self.dz, f, q[1], f, q[2], ws)
            g.grp_rmsnorm_backward(m, d, self.dy, d, g.DTYPE_BF16, self.h[i], d, g.DTYPE_BF16, p[0], self.eps, self.dh, d, self.dh, d, q[0], ws)
        return self.dh[:m]

    def step(self, opt: "g.OptimizerDesc", max_norm: float) -> torch.Tensor:
        """Clips the gradient, takes the optimizer's step; the gradient's norm (device, fp32 [1])."""
        g.grp_clip_gradients(self.gradients, max_norm, self.norm)
        self.steps += 1
        g.grp_optimizer_step(opt, self.theta.numel(), self.steps, self.theta, self.grad, self.m, self.v)
        self._round_weights()
        self._quantized = None              # (made anew by the next serve)
        return self.norm

    def _weights8(self):
        """The weights in 8 bits, [K x N] as rows of their transpose; made where theta was written, always in the same place, and waited for by other streams."""
        if self._served is None:
            def room(w):
                return torch.empty(w.shape[1], w.shape[0], dtype=torch.float8_e4m3fn, device=w.device), torch.empty(w.shape[1], device=w.device)
            with torch.inference_mode(False):
                self._served = [(room(p[1]), room(p[3])) for p in self.params]
        if self._quantized != self.theta._version:
            for p, pair in zip(self.params, self._served):
                for w, (q, s) in zip((p[1], p[3]), pair):
                    t = w.t().contiguous()
                    g.grp_quantize_rows(t.shape[0], t.shape[1], t, t.shape[1], g.DTYPE_FP32, q, t.shape[1], s)
            self._quantized = self._seen()
            if self._quantized is not None and self.theta.is_cuda:
                self._made = g._stream(None), torch.cuda.current_stream().record_event()
        elif self._made is not None and self._made[0] != g._stream(None) and not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().wait_event(self._made[1])
        return self._served

    def serve(self, x: torch.Tensor) -> torch.Tensor:
        """``forward`` with products in 8 bits (nothing is kept for a backward pass)."""
        m, d, f = self._check(x), self.dim, self.hidden
        dev = x.device
        y8, s1 = torch.empty(m, d, dtype=torch.float8_e4m3fn, device=dev), torch.empty(m, device=dev)
        a8, s2 = torch.empty(m, f, dtype=torch.float8_e4m3fn, device=dev), torch.empty(m, device=dev)
        a, out = torch.empty(m, f, dtype=torch.bfloat16, device=dev), x
        ws = self._room(max(g.grp_linear_workspace_bytes(g.LINEAR_FORWARD, m, n, k, g.DTYPE_E4M3) for n, k in ((f, d), (d, f))))
        for (p, ((w1, w1s), (w2, w2s))) in zip(self.params, self._weights8()):
            nxt = torch.empty_like(x)
            g.grp_rmsnorm(m, d, out, d, g.DTYPE_BF16, None, 0, p[0], self.eps, None, 0, y8, d, g.DTYPE_E4M3, s1)
            g.grp_linear(m, f, d, y8, d, w1, d, g.DTYPE_E4M3, s1, w1s, p[2], self.act, None, 0, a, f, g.DTYPE_BF16, None, 0, ws)
            g.grp_quantize_rows(m, f, a, f, g.DTYPE_BF16, a8, f, s2)
            g.grp_linear(m, d, f, a8, f, w2, f, g.DTYPE_E4M3, s2, w2s, p[4], g.ACT_NONE, out, d, nxt, d, g.DTYPE_BF16, None, 0, ws)
            out = nxt
        return out
