"""An attention block on quaternion maps, from the library's entry points.

    qkv   = W_qkv (x) h                    1x1 quaternion convolution
    a     = attention(q, k, v) + bias      between all pixels of an image, the bias
                                           learned by buckets of the relative position
    y     = W_out (x) a                    1x1 quaternion convolution
    out   = x + scale gate dropout(norm(y) gamma)
    h_out = norm(out) next_gamma           what the next block's W_qkv reads

x and h travel together from block to block: h is the norm of x, computed by the
block before (``norm_in`` for the first).  ``backward`` takes the gradients of
both outputs and returns those of both inputs, so that no map is read for a norm
or a residual sum of its own.

``cache`` and ``query`` are the form for single pixels: keys and values of a map
that arrives row by row are written once, and a query at any place reads the
first ``kv_len`` of them.

    python -m paper_2509_05512_amd.attention_block

trains two blocks for a few steps on random maps and asks them single pixels.
"""
import math

import torch

from . import quan


class AttentionBlock:
    """params: float32 tensors by name, for an optimizer; ``load`` casts and
    packs the kernels that the convolutions read after a change to them."""

    def __init__(self, c, heads, kv_heads=None, radius=8, buckets=17, p=0.0, last=False, dtype=torch.bfloat16,
                 device="cuda", seed=0):
        kv_heads = heads if kv_heads is None else kv_heads
        if c % heads or heads % kv_heads:
            raise ValueError("c must be a multiple of heads, heads of kv_heads")
        self.c, self.heads, self.kv = c, heads, c // heads * kv_heads
        self.p, self.dtype = p, dtype
        self.bucket = quan.quan_relpos_buckets(radius, buckets, device)
        draw = torch.Generator().manual_seed(seed)
        # a quaternion kernel sums 4 c products
        wide = c + 2 * self.kv
        self.params = {
            "qkv": torch.randn((4, wide, c, 1, 1), generator=draw) / math.sqrt(4 * c),
            "proj": torch.randn((4, c, c, 1, 1), generator=draw) / math.sqrt(4 * c),
            "table": 0.1 * torch.randn((heads, buckets, buckets), generator=draw),
            "gamma": torch.ones((4, c)),
            "scale": torch.full((4, c), 0.1),
        }
        if not last:
            self.params["next_gamma"] = torch.ones((4, c))
        self.params = {name: t.to(device) for name, t in self.params.items()}
        self.load()

    def load(self):
        self.kernels = {name: self.params[name].to(self.dtype) for name in ("qkv", "proj")}
        self.packed = {name: quan.quan_qconv2d_pack_weights(*w) for name, w in self.kernels.items()}

    def _conv(self, name, x):
        return quan.quan_qconv2d_forward_packed(x, self.packed[name], self.kernels[name].shape[1:])

    def _parts(self, qkv):
        """q, k, v: slices of the channels of one map, not copied."""
        return qkv[:, :, :self.c], qkv[:, :, self.c:self.c + self.kv], qkv[:, :, self.c + self.kv:]

    def _relpos(self):
        return self.params["table"], self.bucket, self.bucket

    def _step(self):
        at = self.params
        return dict(gamma=at["gamma"], scale=at["scale"], next_gamma=at.get("next_gamma"))

    def forward(self, x, h, gate=None, rng=None, save=False):
        """(out, h_out), h_out None for the last block; with save (out, h_out,
        saved) for backward.  Dropout is on where rng is given."""
        p = 0.0 if rng is None else self.p
        qkv = self._conv("qkv", h)
        attended = quan.quan_attention_forward(*self._parts(qkv), self.heads, relpos=self._relpos(), save=save)
        a, stats, rest = attended if save else (attended, None, None)
        y = self._conv("proj", a)
        out, h_out = quan.quan_residual_forward(x, y, gate=gate, p=p, rng=rng, **self._step())
        if not save:
            return out, h_out
        return out, h_out, (h, qkv, a, stats, rest, y, out, gate, p, rng)

    def backward(self, saved, dout, dh_out=None):
        """(dx, dh, dgate, gradients of params by name)"""
        h, qkv, a, stats, rest, y, out, gate, p, rng = saved
        step, grads = self._step(), {}
        last = step["next_gamma"] is None
        res = quan.quan_residual_backward(y, dout, gate=gate, p=p, rng=rng, out=None if last else out, dh=dh_out,
                                          **step)
        grads["gamma"], grads["scale"] = res.dgamma, res.dscale
        if not last:
            grads["next_gamma"] = res.dnext_gamma
        da = self._conv_backward("proj", a, res.dy, grads)
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = self._parts(dqkv)
        grads["table"] = quan.quan_attention_backward(*self._parts(qkv), a, stats, rest, da, self.heads,
                                                      relpos=self._relpos(), dq=dq, dk=dk, dv=dv)[3]
        dh = self._conv_backward("qkv", h, dqkv, grads)
        return res.dx, dh, res.dgate, grads

    def _conv_backward(self, name, x, dy, grads):
        dws, _ = quan.quan_qconv2d_backward_weight(x, dy, (1, 1), with_bias=False)
        grads[name] = torch.stack(dws)
        return quan.quan_qconv2d_backward_data(dy, *self.kernels[name], x.shape[3:])

    def cache(self, n, height, width):
        """Keys and values of maps [height, width], none written yet."""
        device = self.bucket.device
        return tuple(quan.empty_qmap(n, self.kv, height, width, self.dtype, device) for _ in range(2))

    def write(self, cache, h, row):
        """Keys and values of the rows that h holds, from `row` on."""
        _, k, v = self._parts(self._conv("qkv", h))
        for held, new in zip(cache, (k, v)):
            held[:, :, :, row:row + h.shape[3]].copy_(new)

    def query(self, cache, x, h, pos, kv_len=None, gate=None):
        """(out, h_out) of one pixel per image, x and h [N, 4, C, 1, 1], at pos
        int32 [N, 2] (y, x) of a cache whose first kv_len int32 [N] pixels are
        there."""
        q, _, _ = self._parts(self._conv("qkv", h))
        a = quan.quan_attention_forward(q, *cache, self.heads, relpos=self._relpos(), kv_len=kv_len, pos=pos)
        return quan.quan_residual_forward(x, self._conv("proj", a), gate=gate, **self._step())


class Stack:
    """Blocks behind one norm, the last without a norm of its output."""

    def __init__(self, depth, c, heads, **options):
        seed = options.pop("seed", 0)
        self.blocks = [AttentionBlock(c, heads, last=i + 1 == depth, seed=seed + i, **options) for i in range(depth)]
        self.norm_in = torch.ones((4, c), device=self.blocks[0].bucket.device)

    def forward(self, x, rngs=None, save=False):
        """The last block's map; with save (map, saved).  rngs: one per block."""
        first, held = x, []
        h = quan.quan_rmsnorm_forward(x, self.norm_in)
        for i, block in enumerate(self.blocks):
            got = block.forward(x, h, rng=None if rngs is None else rngs[i], save=save)
            x, h = got[:2]
            held.append(got[-1])
        return (x, (first, held)) if save else x

    def backward(self, saved, dout):
        """(dx, gradients of norm_in, [gradients of each block's params])"""
        first, held = saved
        grads, dh = [], None
        for block, kept in zip(reversed(self.blocks), reversed(held)):
            dout, dh, _, g = block.backward(kept, dout, dh)
            grads.append(g)
        dx, dnorm = quan.quan_rmsnorm_backward(first, dh, self.norm_in, dres=dout)
        return dx, dnorm, grads[::-1]


def train(stack, x, target, steps, rate, seed=0):
    """Plain gradient descent on the mean squared error; the losses."""
    losses = []
    for step in range(steps):
        # one seed, an offset per step and block: masks that no two calls share
        rngs = [torch.tensor([seed, step * len(stack.blocks) + i], dtype=torch.int64, device=x.device)
                for i in range(len(stack.blocks))]
        out, saved = stack.forward(x, rngs, save=True)
        off = out.float() - target.float()
        losses.append(off.square().mean())
        dout = quan.to_device_layout((off * (2.0 / off.numel())).to(x.dtype))
        _, dnorm, grads = stack.backward(saved, dout)
        stack.norm_in -= rate * dnorm
        for block, g in zip(stack.blocks, grads):
            for name, value in g.items():
                block.params[name] -= rate * value
            block.load()
    return [float(v) for v in losses]


def main():
    if not torch.cuda.is_available():
        raise SystemExit("this needs an MI355X (gfx950) GPU")
    n, c, heads, side = 8, 64, 4, 20
    draw = torch.Generator().manual_seed(0)

    def random_map(h, w):
        return quan.to_device_layout(torch.randn((n, 4, c, h, w), generator=draw).to(torch.bfloat16).cuda())

    stack = Stack(2, c, heads, radius=side - 1, buckets=17, p=0.1)
    x, target = random_map(side, side), random_map(side, side)
    losses = train(stack, x, target, steps=10, rate=20.0)
    print("loss of each step: " + " ".join(f"{v:.4f}" for v in losses))

    # one block asked for the pixel (side / 2, side / 2) while its rows arrive
    block = stack.blocks[0]
    h = quan.quan_rmsnorm_forward(x, stack.norm_in)
    whole, _ = block.forward(x, h)
    cache, at = block.cache(n, side, side), side // 2
    pos = torch.full((n, 2), at, dtype=torch.int32, device="cuda")
    px, ph = (quan.to_device_layout(t[..., at:at + 1, at:at + 1]) for t in (x, h))
    for row in range(0, side, 5):
        block.write(cache, quan.to_device_layout(h[..., row:row + 5, :]), row)
        there = torch.full((n,), (row + 5) * side, dtype=torch.int32, device="cuda")
        out, _ = block.query(cache, px, ph, pos, kv_len=there)
        off = (out.float() - whole[..., at:at + 1, at:at + 1].float()).abs().max()
        print(f"{row + 5} of {side} rows: largest difference from the whole map's pixel {float(off):.4f}")


if __name__ == "__main__":
    main()
