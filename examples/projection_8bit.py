"""The query/key/value projection of an attention block with 8-bit floats, trained for a few steps.

A projection's weights are kept in fp32 and quantised once a step (E4M3 codes, a scale for each block of 128 x 128).  Forwards:
activations are quantised and multiplied, the query and key heads normalised and rotated by their tokens' positions.  Backwards: the
gradients of the heads go into the projection's result, where they came from, and from there into the input and the weights.

    python examples/projection_8bit.py [--steps 20] [--tokens 4096] [--channels 576] [--heads 8]

The sizes are those of the attention projection in benchmark configuration 5 (16 images of 16 x 16, 576 -> 1728).  The loss is the mean squared
distance from a teacher: the same projection with other weights, in fp32.
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2512_05746_amd as hq  # noqa: E402

EPS = 1e-6


def tables(positions, rotary, device):
    angle = torch.outer(torch.arange(positions, dtype=torch.float64), 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary))
    return angle.cos().float().to(device), angle.sin().float().to(device)


class Projection:
    """x [tokens, channels] -> queries, keys (normalised, rotated) and values, each [tokens, heads, channels / heads]."""

    def __init__(self, channels, heads, tokens, device, seed):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.d = heads, channels // heads
        self.weight = torch.randn((3 * channels, channels), generator=gen, device=device) * 0.02
        self.bias = torch.zeros(3 * channels, device=device)
        self.q_weight, self.k_weight = torch.ones(self.d, device=device), torch.ones(self.d, device=device)
        self.cos, self.sin = tables(tokens, self.d, device)

    def parameters(self):
        return self.weight, self.bias, self.q_weight, self.k_weight

    def split(self, qkv):
        return qkv.view(qkv.shape[0], 3, self.heads, self.d).unbind(1)

    def quantise(self):
        """Once a step, after the weights have changed."""
        self.codes, self.codes_t, self.scale = hq.hq_fp8_quantize_blocks(self.weight, transposed=True)

    def forward(self, x, positions):
        qkv = hq.hq_act_quant_fp8_linear(x, self.codes, self.scale, self.bias.to(x.dtype), y_dtype=x.dtype)
        q, k, v = self.split(qkv)
        q_out, k_out = hq.hq_qk_norm_rope(q, k, self.q_weight, self.k_weight, self.cos, self.sin, positions, eps=EPS)
        return (q_out, k_out, v), (x, q, k, positions)

    def backward(self, dq, dk, dv, saved):
        """Gradients of x and of the parameters, in their order."""
        x, q, k, positions = saved
        dqkv = torch.empty((x.shape[0], 3 * self.heads * self.d), dtype=x.dtype, device=x.device)
        to_q, to_k, to_v = self.split(dqkv)
        _, _, dqw, dkw = hq.hq_qk_norm_rope_backward(dq, dk, q, k, self.q_weight, self.k_weight, self.cos, self.sin, positions,
                                                     eps=EPS, out=(to_q, to_k))
        to_v.copy_(dv)
        dx, dw, db = hq.hq_fp8_linear_backward(dqkv, x, self.codes_t, self.scale, bias_grad=True)
        return dx, (dw, db, dqw, dkw)

    def plain(self, x, positions):
        """The same in fp32, without quantisation, of elementary operations."""
        q, k, v = self.split(x.float() @ self.weight.t() + self.bias)
        cos, sin, half = self.cos[positions][:, None], self.sin[positions][:, None], self.d // 2
        out = []
        for t, w in ((q, self.q_weight), (k, self.k_weight)):
            n = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS) * w
            a, b = n[..., :half], n[..., half:]
            out.append(torch.cat([a * cos - b * sin, b * cos + a * sin], -1))
        return out[0], out[1], v


def train(steps=20, tokens=4096, channels=576, heads=8, images=16, dtype=torch.bfloat16, rate=0.05, device="cuda"):
    """Losses before each step and after the last."""
    gen = torch.Generator(device=device).manual_seed(0)
    student, teacher = (Projection(channels, heads, tokens // images, device, seed) for seed in (1, 2))
    x = torch.randn((tokens, channels), generator=gen, device=device).to(dtype)
    positions = torch.arange(tokens // images, device=device).repeat(images)
    wanted = teacher.plain(x, positions)
    # momentum, scaled by each parameter's largest gradient so far
    moments, largest = [torch.zeros_like(p) for p in student.parameters()], [torch.zeros((), device=device) for _ in student.parameters()]
    losses = []
    for step in range(steps + 1):
        student.quantise()
        got, saved = student.forward(x, positions)
        off = [g.float() - w for g, w in zip(got, wanted)]
        losses.append(sum((o * o).mean() for o in off))
        if step == steps:
            break
        _, grads = student.backward(*[(2.0 / o.numel() * 1024.0 * o).to(dtype) for o in off], saved)   # (scaled by 1024 on the way)
        for i, (p, g) in enumerate(zip(student.parameters(), grads)):
            moments[i].mul_(0.9).add_(g / 1024.0)
            largest[i] = torch.maximum(largest[i], g.abs().max() / 1024.0)
            p.add_(moments[i] / largest[i].clamp(min=1e-30), alpha=-rate * float(p.abs().mean().clamp(min=1e-3)))
    return [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--channels", type=int, default=576)
    ap.add_argument("--heads", type=int, default=8)
    args = ap.parse_args()
    losses = train(args.steps, args.tokens, args.channels, args.heads)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %3d  loss %.5f" % (i, losses[i]))
    print("last      loss %.5f" % losses[-1])


if __name__ == "__main__":
    main()
