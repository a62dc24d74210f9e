"""A surrogate learned from collected samples with its activations kept in 8
bits, and answering in 8-bit integers.

    python -m paper_2407_18352_amd.surrogate8 [--points N] [--dims 5,256,256,1] [--steps K]

The command prices European calls (the accurate path), records the region's
inputs and outputs as collect mode does, trains a multilayer perceptron on the
records, and answers new points with its layers in 8 bits.  The class holds
what a training loop and a server need of the library: ``forward`` keeps every
layer's input in 8 bits (a little over half of bf16's memory), ``backward``
computes the gradients from them, ``answering`` lays the weights out for
``answer``.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import _abi, api


def _rows(t):
    """`t` with the values of a row after one another and rows of their own."""
    return t if t.stride(1) == 1 and t.stride(0) >= t.shape[1] else t.contiguous()


def _hold(captured, tensors):
    """A graph reads and writes where the tensors are now: their memory stays, whatever becomes of them."""
    if torch.cuda.is_current_stream_capturing():
        for t in tensors:
            captured.setdefault((t.data_ptr(), t.numel()), t.detach())


class Surrogate8:
    """A ReLU perceptron of the widths ``dims``: fp32 weights ``W[l]``
    [out][in] and biases ``b[l]`` with gradients in ``.grad``; products in
    bf16.  ``backward`` is that of the last ``forward``: another one in between
    replaces what was kept.  Calls may come on one stream after another, each
    works after the one before; from several threads at a time they may not.
    What calls captured into a graph read and write ``captured`` keeps for the
    graph's replays; it may be cleared once the graph is gone."""

    def __init__(self, dims, seed: int = 0):
        g = torch.Generator().manual_seed(seed)
        self.dims = [int(d) for d in dims]
        self.W = [(torch.randn((o, i), generator=g) * math.sqrt(2 / i)).cuda().requires_grad_()
                  for i, o in zip(self.dims, self.dims[1:])]
        self.b = [torch.zeros(o, device="cuda").requires_grad_() for o in self.dims[1:]]
        for p in self.parameters():
            p.grad = torch.zeros_like(p)
        self.kept, self.scratch, self.Wh, self.stream = [], None, [], torch.cuda.current_stream()
        self.captured = {}              # by its address

    def parameters(self):
        return self.W + self.b

    def _buffers(self):
        return [t for k in self.kept for t in (k.codes, k.exps)] + self.Wh + ([] if self.scratch is None else [self.scratch])

    def _in_order(self):
        """Kept values, weights in bf16 and scratch memory are used again by
        every call: a call on another stream than the last waits for it.  (A
        capture into a graph begins after a synchronization, and a stream in it
        may not wait for one outside.)"""
        now = torch.cuda.current_stream()
        if now != self.stream and not torch.cuda.is_current_stream_capturing():
            now.wait_stream(self.stream)
            for t in self._buffers():
                t.record_stream(now)
        self.stream = now

    @torch.no_grad()
    def forward(self, x):
        """Outputs [n][dims[-1]] (fp32) of inputs [n][dims[0]]; keeps what
        ``backward`` reads."""
        self._in_order()
        n, a = x.shape[0], _rows(x.to(torch.bfloat16))
        if not self.kept or self.kept[0].rows != n:
            self.kept = [api.Checkpoint8(n, d, _abi.ACT_RELU if l else _abi.ACT_IDENTITY) for l, d in enumerate(self.dims[:-1])]
        self.Wh = [w.to(torch.bfloat16) for w in self.W]
        _hold(self.captured, self._buffers() + self.parameters())
        api.checkpoint8_save(self.kept[0], a)
        for l in range(1, len(self.dims) - 1):
            a = torch.nn.functional.linear(a, self.Wh[l - 1], self.b[l - 1].to(torch.bfloat16))
            api.checkpoint8_save(self.kept[l], a, a)          # a = relu(a), kept
        return torch.nn.functional.linear(a, self.Wh[-1]).float() + self.b[-1]

    @torch.no_grad()
    def backward(self, dy, accumulate: bool = False):
        """Gradients of the loss in ``.grad`` (made where an optimizer has taken
        them away) from that of the outputs."""
        self._in_order()
        dy = _rows(dy.to(torch.bfloat16))
        for p in self.parameters():
            if p.grad is None:
                p.grad = torch.zeros_like(p)
        for l in range(len(self.W) - 1, -1, -1):
            W = self.Wh[l] if l else None
            dx = torch.empty((dy.shape[0], self.dims[l]), dtype=torch.bfloat16, device="cuda") if l else None
            need = api.backward8_scratch_bytes(self.kept[l], dy, W)
            if self.scratch is None or self.scratch.numel() < need:
                self.scratch = torch.empty(need, dtype=torch.uint8, device="cuda")
            _hold(self.captured, self._buffers() + [self.W[l].grad, self.b[l].grad])
            api.backward8(self.kept[l], dy, self.W[l].grad, self.b[l].grad, W=W, dx=dx, accumulate=accumulate,
                          scratch=self.scratch)
            dy = dx

    @torch.no_grad()
    def answering(self):
        """The layers with their weights in 8 bits, as they are now."""
        return [api.Linear8(w, b) for w, b in zip(self.W, self.b)]


@torch.no_grad()
def answer(layers, x):
    """Outputs (fp32) of a surrogate's 8-bit layers for inputs [n][in]."""
    n, x = x.shape[0], _rows(x)
    scratch = torch.empty(max(l.scratch_bytes(n) for l in layers), dtype=torch.uint8, device="cuda")
    for i, layer in enumerate(layers):
        last = i + 1 == len(layers)
        y = torch.empty((n, layer.n_out), dtype=torch.float32 if last else torch.bfloat16, device="cuda")
        api.linear8(layer, x, y, _abi.ACT_IDENTITY if last else _abi.ACT_RELU, scratch=scratch)
        x = y
    return x


# ---- the command ------------------------------------------------------------

RANGES = [(10, 200), (10, 200), (0, 0.1), (0.05, 0.6), (0.1, 5)]   # price, strike, rate, volatility, years


def call_prices(s, k, r, v, t, out):
    """The accurate path: European calls, by their closed form."""
    d1 = (torch.log(s / k) + (r + v * v / 2) * t) / (v * t.sqrt())
    d2 = d1 - v * t.sqrt()
    n = torch.special.ndtr
    torch.sub(s * n(d1), k * torch.exp(-r * t) * n(d2), out=out)


def collect(points: int, seed: int):
    """(inputs [points][5], outputs [points][1]) of one invocation of the
    region, recorded through its tensor maps."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    fields = [torch.rand(points, generator=g, device="cuda") * (hi - lo) + lo for lo, hi in RANGES]
    prices = torch.empty(points, device="cuda")
    spec = {"rank": 1, "slices": [((0,), (1,))], "sweep": ((0,), (points,), (1,)), "bnd": [_abi.BND_NONE]}
    to, back = api.Map(spec, fields, _abi.TO), api.Map(spec, [prices], _abi.FROM)
    call_prices(*fields, prices)
    record = torch.empty((points, 6), device="cuda")      # a point's inputs, then its output
    api.collect_pair(to, record, 6, back, record[:, 5:], 6)
    return record[:, :5], record[:, 5:]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--points", type=int, default=65536)
    ap.add_argument("--dims", default="5,256,256,1")
    ap.add_argument("--steps", type=int, default=300)
    a = ap.parse_args(argv)
    x, y = collect(a.points, 1)
    mean, std = x.mean(0), x.std(0)
    unit = y.std()
    model = Surrogate8([int(d) for d in a.dims.split(",")])
    opt = torch.optim.Adam(model.parameters(), lr=2e-3)
    xn, yn = (x - mean) / std, y / unit
    loss = None
    for step in range(a.steps):
        off = model.forward(xn) - yn
        loss = off.square().mean()
        if step % 50 == 0:
            print("step %4d: rms error %.4f of the prices' spread" % (step, loss.sqrt().item()), flush=True)
        model.backward(off * (2 / off.numel()))
        opt.step()
    xs, ys = collect(a.points, 2)
    got = answer(model.answering(), (xs - mean) / std) * unit
    rms = ((got - ys).square().mean().sqrt() / unit).item()
    print("step %4d: rms error %.4f; answering new points in 8 bits: %.4f" % (a.steps, loss.sqrt().item(), rms))
    return loss.sqrt().item(), rms


if __name__ == "__main__":
    main()
