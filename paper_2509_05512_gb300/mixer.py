"""A stack of residual channel-mixing blocks: pointwise quaternion layers in 8-bit floating point,
each joined to the stream with a norm, a gate and dropout, and followed by the next block's norm:

    n_0 = norm(x);   h_l = n_l W_l;   y_l, n_(l+1) = join(y_(l-1), h_l)      (y_(-1) = x)

One block is two launches forward, the product and the join, which writes the next block's rows in 8
bits beside bf16 (for the weight gradient); with a statistic over the whole row (groups=1), where
that join sums in another order, the product quantises its rows itself.  Backward it is seven.  The
letters are kept in bf16 and quantised once per update (`quantize`), both ways round; the weight
gradients come from the bf16 weight-gradient kernel.  Every mask is a function of the seed, the
block and a device counter that `forward` leaves to `advance`, so that a captured training step
draws new masks at each replay.

    python -m paper_2509_05512_gb300.mixer --steps 30

trains such a stack on synthetic maps and prints the loss; with --top 10, by distillation from the
largest logits of a teacher, its channels taken for classes.  `Mixer.serve` runs a few pixels with
4-bit letters.
"""
from __future__ import annotations

import argparse

from . import quan


class Mixer:
    """Parameters, their 8-bit forms and the tensors one step keeps."""

    def __init__(self, channels: int, depth: int, *, groups: int = 4, p: float = 0.0,
                 alpha: float = 1.0, eps: float = 1e-5, seed: int = 0, device="cuda"):
        import torch
        if channels % 4 or depth < 1:
            raise ValueError("channels must be a multiple of 4, depth at least 1")
        self.channels, self.depth = channels, depth
        self.groups, self.p, self.alpha, self.eps, self.seed = groups, p, alpha, eps, seed
        g = torch.Generator(device=device).manual_seed(seed)
        Q = channels // 4
        self.letters = [[(torch.randn((Q, 1, 1, Q), generator=g, device=device) /
                          channels ** 0.5).to(torch.bfloat16) for _ in range(4)]
                        for _ in range(depth)]
        ones = lambda: torch.ones(channels, device=device)
        self.pre = [ones() for _ in range(depth + 1)]  # in front of each block, and the last
        self.post = [ones() for _ in range(depth)]
        self.gate = [torch.full((channels,), 0.5, device=device) for _ in range(depth)]
        self.counter = torch.zeros((), dtype=torch.int64, device=device)
        self.quantize()

    def quantize(self) -> None:
        """The letters' 8-bit forms, after the letters changed.  Those of `quantize_4bit` are of the
        letters before then (and stay allocated, for a graph that was captured with them)."""
        self.w4_current = False
        self.w = [quan.quantize_f8_weights(*w) for w in self.letters]
        self.wt = [quan.quantize_f8_weights(*w, transpose=True) for w in self.letters]

    def quantize_4bit(self, group: int = 64) -> None:
        """The letters in 4 bits, for `serve`; again after each `update` or `quantize`.  (An update
        that a graph replays changes the letters without this object's knowledge.)"""
        self.w4 = [quan.quantize_w4_weights(*w, group=group) for w in self.letters]
        self.w4_current = True

    def serve(self, x):
        """The stack on a few pixels, bf16 x [..., channels] (CUDA), without dropout and with the
        letters of quantize_4bit: about a quarter of the bf16 letters' bytes, which bound a single
        pixel.  Keeps nothing."""
        if not self.w4_current:
            raise RuntimeError("the letters are not in 4 bits since they changed: quantize_4bit()")
        _, n = quan.residual_join(x, pre=self.pre[0], groups=self.groups, eps=self.eps)
        y = x
        for l in range(self.depth):
            h = quan.qpointwise_w4(n, self.w4[l])
            y, n = quan.residual_join(y, h, **self._join(l, x.numel(), False))
        return n

    def _join(self, l: int, elements: int, training: bool) -> dict:
        """The keyword arguments of block l's join, both ways."""
        return dict(post=self.post[l], gate=self.gate[l], pre=self.pre[l + 1], alpha=self.alpha,
                    groups=self.groups, eps=self.eps, p=self.p if training else 0.0,
                    seed=self.seed, offset=l * -(-elements // 8), counter=self.counter)

    def forward(self, x, training: bool = True):
        """bf16 x [N, H, W, channels] (CUDA) -> the last norm's output; keeps what `backward`
        needs."""
        self.training = training
        _, n, rows = self._norm(0, x, None, None,
                                dict(pre=self.pre[0], groups=self.groups, eps=self.eps))
        self.y, self.h, self.n = [x], [], [n]
        for l in range(self.depth):
            h = quan.qpointwise_f8(rows, self.w[l])
            y, n, rows = self._norm(l + 1, self.y[l], h, rows, self._join(l, x.numel(), training))
            self.h.append(h)
            self.y.append(y)
            self.n.append(n)
        return self.n[-1]

    def _norm(self, l: int, x, h, rows, args):
        """A join, and what block l's product reads: the norm in 8 bits (in the place of the block
        before's rows, which its product has read), or in bf16."""
        if self.groups == 4 and l < self.depth:
            return quan.residual_join_f8(x, h, keep=True, n8=rows, **args)
        y, n = quan.residual_join(x, h, **args)
        return y, n, n

    def advance(self) -> None:
        """Moves the masks past this step's."""
        self.counter += self.depth * -(-self.y[0].numel() // 8)

    def backward(self, dn):
        """Gradients from dn = dL/d(forward's result): dict of dx, letters (four fp32 tensors a
        block), pre, post and gate (fp32, as the parameters)."""
        dy = None
        grads = {"letters": [None] * self.depth, "post": [None] * self.depth,
                 "gate": [None] * self.depth, "pre": [None] * (self.depth + 1)}
        for l in reversed(range(self.depth)):
            dy, dh, grads["post"][l], grads["gate"][l], grads["pre"][l + 1] = \
                quan.residual_join_backward(dy, dn, self.y[l + 1], self.h[l],
                                            **self._join(l, dn.numel(), self.training))
            grads["letters"][l] = quan.qconv2d_backward_weight(self.n[l], dh, kh=1, kw=1)
            dn = quan.qpointwise_f8_backward_data(dh, self.wt[l])
        grads["dx"], _, _, _, grads["pre"][0] = quan.residual_join_backward(
            dy, dn, self.y[0], pre=self.pre[0], groups=self.groups, eps=self.eps)
        return grads

    def update(self, grads, lr: float) -> None:
        """One step of gradient descent on every parameter, and the letters' 8-bit forms."""
        for l in range(self.depth):
            for w, d in zip(self.letters[l], grads["letters"][l]):
                w.copy_(w.float() - lr * d)
        for name in ("pre", "post", "gate"):
            for v, d in zip(getattr(self, name), grads[name]):
                v.sub_(d, alpha=lr)
        self.quantize()


def distillation(model, x, index, teacher, *, temperature=1.0, training=True):
    """A stack whose channels are classes against a teacher's top logits (index, teacher
    [N, H, W, top], as torch.topk gives them): the mean loss over the pixels with a slot in use (a device
    scalar) and the gradient of model.forward's result, for model.backward."""
    out = model.forward(x, training=training)
    slots = (index >= 0) & (index < out.shape[-1]) & (teacher != -float("inf"))
    pixels = slots.any(dim=-1)
    weight = pixels.float() / pixels.sum().clamp(min=1)
    loss, dn = quan.distill_loss_and_gradient(out, index, teacher, weight,
                                              temperature=temperature)
    return (loss * weight).sum(), dn


def train(steps: int = 30, N: int = 8, H: int = 16, channels: int = 256, depth: int = 3,
          lr: float = 0.2, p: float = 0.1, seed: int = 0, top: int = 0, temperature: float = 1.0,
          report=print) -> list:
    """Fits a stack on fixed synthetic maps to the output of another one, or with top > 0, its
    channels taken for classes, to that many largest logits of the other's; the losses."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.randn((N, H, H, channels), generator=gen, device="cuda").to(torch.bfloat16)
    target = Mixer(channels, depth, seed=seed + 2).forward(x, training=False).float()
    model = Mixer(channels, depth, p=p, seed=seed)
    if top:
        teacher, index = torch.topk(target, top, dim=-1)
    losses = []
    for step in range(steps):
        if top:
            loss, dn = distillation(model, x, index, teacher, temperature=temperature)
        else:
            diff = model.forward(x).float() - target
            loss, dn = diff.square().mean(), (2.0 / (N * H * H) * diff).to(torch.bfloat16)
        losses.append(float(loss))
        grads = model.backward(dn)
        model.update(grads, lr)
        model.advance()
        if report:
            report("step %d: loss %.4f" % (step, losses[-1]))
    return losses


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--images", type=int, default=8)
    ap.add_argument("--size", type=int, default=16, help="pixels a side of the maps")
    ap.add_argument("--channels", type=int, default=256)
    ap.add_argument("--depth", type=int, default=3)
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--top", type=int, default=0,
                    help="distil that many of a teacher's largest logits a pixel")
    ap.add_argument("--temperature", type=float, default=1.0)
    a = ap.parse_args(argv)
    train(a.steps, a.images, a.size, channels=a.channels, depth=a.depth, p=a.dropout, top=a.top,
          temperature=a.temperature)


if __name__ == "__main__":
    main()
