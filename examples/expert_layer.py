"""A feed-forward layer of experts on 8-bit products: the forward pass, the backward pass, and a step of few tokens.

    logits -> route -> rows in the order of their experts
    x      -> quantise -> experts' up products (gathering the rows) -> silu -> quantise -> experts' down products -> combine

The backward pass quantises what it multiplies along the other axis as well: gradients by rows for the data gradients, transposed (along
the rows of an expert, in blocks of 128) for the weight gradients.  Run on an MI355X:

    python examples/expert_layer.py [--tokens T] [--experts E] [--k K] [--width D] [--hidden F]

prints the distance of the result and of every gradient from the same layer in 32 bits, and the times of the passes.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2512_02551_amd as hg  # noqa: E402


def quantise_weights(w):
    """w [experts][out][in] -> (q, scales) for the forward product and (q, scales) of the transposed form for the data gradient, by 128 x 128 blocks."""
    parts = [hg.quantise(one, block_rows=128, transposed=True) for one in w]
    return [torch.stack([p[i].view(torch.uint8) if i % 2 == 0 else p[i] for p in parts]) for i in range(4)]


class ExpertLayer:
    """up [experts][hidden][width], down [experts][width][hidden]; sigmoid or softmax routing, k experts a token."""

    ALIGN = 128                 # an expert's rows are whole blocks: weight gradients sum over blocks of 128 rows

    def __init__(self, up, down, k, score="softmax", bias=None):
        self.k, self.score, self.bias = k, score, bias
        self.up, self.down = quantise_weights(up), quantise_weights(down)

    def load(self, up, down):
        """New weights: their 8-bit forms, both ways round, in the place of the old ones, where a captured step reads them."""
        for old, new in zip(self.up + self.down, quantise_weights(up) + quantise_weights(down)):
            old.copy_(new)

    @staticmethod
    def _product(a, scale_a, weights, transposed, **more):
        q, s = weights[2:] if transposed else weights[:2]
        return hg.scaled_product(a, scale_a, q.view(torch.float8_e4m3fn), s, **more)

    def forward(self, x, logits):
        weights, chosen, offsets, rows, tokens = hg.route(logits, self.k, self.bias, self.score, align=self.ALIGN)
        qx, sx, _, _ = hg.quantise(x)
        h = self._product(qx, sx, self.up, False, c="bf16", offsets=offsets, index=tokens)
        a = torch.nn.functional.silu(h)
        qa, sa, _, _ = hg.quantise(a)
        y = self._product(qa, sa, self.down, False, c="bf16", offsets=offsets)
        self.kept = x, logits, weights, chosen, offsets, rows, tokens, h, a, y
        return hg.combine(y, rows, weights)

    def backward(self, dout):
        """(dx, dlogits, dup, ddown)."""
        x, logits, weights, chosen, offsets, rows, tokens, h, a, y = self.kept
        dy, dweights = hg.combine_backward(y, rows, tokens, weights, dout)
        dlogits = hg.route_backward(logits, chosen, dweights, self.score)
        qy, sy, qyt, syt = hg.quantise(dy, transposed=True)
        _, _, qat, sat = hg.quantise(a, rows=False, transposed=True)
        ddown = hg.scaled_product(qyt, syt, qat, sat, K=dy.shape[0], c="f32", offsets=offsets, along="depth")
        da = self._product(qy, sy, self.down, True, c="bf16", offsets=offsets)
        s = torch.sigmoid(h.float())
        dh = (da * (s * (1 + h.float() * (1 - s)))).to(torch.bfloat16)
        qh, sh, qht, sht = hg.quantise(dh, transposed=True)
        _, _, qxt, sxt = hg.quantise(x, rows=False, transposed=True, index=tokens)
        dup = hg.scaled_product(qht, sht, qxt, sxt, K=dh.shape[0], c="f32", offsets=offsets, along="depth")
        dxs = self._product(qh, sh, self.up, True, c="bf16", offsets=offsets)
        return hg.combine(dxs, rows), dlogits, dup, ddown


class DecodeStep:
    """The forward pass for a fixed number of tokens with everything planned and allocated once, captured in a HIP graph."""

    def __init__(self, layer, tokens, experts, width, hidden):
        new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        k, blocks = layer.k, lambda n: -(-n // hg.SCALE_BLOCK)
        self.layer, self.x, self.logits = layer, new(tokens, width, dtype=torch.bfloat16).zero_(), new(tokens, experts, dtype=torch.float32).zero_()
        self.route = hg.RoutePlan(tokens, experts, k, "f32", layer.score)
        n = self.route.capacity
        self.quantise_x, self.quantise_a = hg.QuantisePlan(tokens, width, "bf16"), hg.QuantisePlan(n, hidden, "bf16")
        self.up = hg.ScaledPlan(n, hidden, width, c="bf16", groups=experts, a_rows=tokens)
        self.down = hg.ScaledPlan(n, width, hidden, c="bf16", groups=experts)
        self.combine = hg.CombinePlan(tokens, k, width, n, "bf16", "bf16")
        self.weights, self.chosen, self.rows = new(tokens, k, dtype=torch.float32), new(tokens, k, dtype=torch.int32), new(tokens, k, dtype=torch.int32)
        self.offsets, self.tokens = new(experts + 1, dtype=torch.int32), new(n, dtype=torch.int32)
        self.qx, self.sx = new(tokens, width, dtype=torch.uint8), new(blocks(width), tokens, dtype=torch.float32)
        self.h, self.y, self.out = new(n, hidden, dtype=torch.bfloat16), new(n, width, dtype=torch.bfloat16), new(tokens, width, dtype=torch.bfloat16)
        self.qa, self.sa = new(n, hidden, dtype=torch.uint8), new(blocks(hidden), n, dtype=torch.float32)
        self._step()
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._step()

    def _step(self):
        s = torch.cuda.current_stream().cuda_stream
        p = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
        self.route.run(p(self.logits), p(self.layer.bias), p(self.weights), p(self.chosen), p(self.offsets), p(self.rows), p(self.tokens), s)
        self.quantise_x.run(p(self.x), p(self.qx), p(self.sx), stream=s)
        self.up.run(p(self.qx), p(self.sx), p(self.layer.up[0]), p(self.layer.up[1]), p(self.h), s, p(self.offsets), p(self.tokens))
        a = torch.nn.functional.silu(self.h)
        self.quantise_a.run(p(a), p(self.qa), p(self.sa), stream=s)
        self.down.run(p(self.qa), p(self.sa), p(self.layer.down[0]), p(self.layer.down[1]), p(self.y), s, p(self.offsets))
        self.combine.run(p(self.rows), p(self.weights), p(self.y), p(self.out), s)

    def __call__(self, x, logits):
        self.x.copy_(x)
        self.logits.copy_(logits)
        self.graph.replay()
        return self.out


def reference(x, logits, up, down, chosen, dout, score):
    """The layer in 32 bits on the same choice of experts, by autograd: result and gradients."""
    x, logits, up, down = (t.detach().float().requires_grad_() for t in (x, logits, up, down))
    p = torch.sigmoid(logits) if score == "sigmoid" else torch.softmax(logits, 1)
    w = p.gather(1, chosen.long())
    w = w / w.sum(1, keepdim=True)
    out = torch.zeros_like(x)
    for e in range(up.shape[0]):
        t, j = torch.where(chosen == e)
        out = out.index_add(0, t, w[t, j, None] * (torch.nn.functional.silu(x[t] @ up[e].t()) @ down[e].t()))
    out.backward(dout.float())
    return out.detach(), x.grad, logits.grad, up.grad, down.grad


def off(got, want):
    """2-norm of the difference over that of the result."""
    return float((got.double() - want.double()).norm() / want.double().norm())


def compare(tokens, experts, k, width, hidden, score="softmax", seed=0):
    """How far the layer's result, its gradients and a decode step's result are from 32 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    x, logits, dout = new(tokens, width).to(torch.bfloat16), new(tokens, experts), new(tokens, width).to(torch.bfloat16)
    up, down = (new(experts, hidden, width) / width ** 0.5).to(torch.bfloat16), (new(experts, width, hidden) / hidden ** 0.5).to(torch.bfloat16)
    layer = ExpertLayer(up, down, k, score)
    out = layer.forward(x, logits)
    grads = layer.backward(dout)
    want = reference(x, logits, up, down, layer.kept[3], dout, score)
    found = {n: off(a, b) for n, a, b in zip(("out", "dx", "dlogits", "dup", "ddown"), (out, *grads), want)}
    step = DecodeStep(layer, tokens, experts, width, hidden)
    for _ in range(3):
        again = step(x, logits)
        torch.cuda.synchronize()
    found["decode"] = off(again, want[0])
    return found, layer, step, (x, logits, dout)


def milliseconds(f, reps=10):
    f()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(reps):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - began) / reps * 1e3


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 2048), ("experts", 16), ("k", 4), ("width", 2048), ("hidden", 1024)):
        ap.add_argument(f"--{name}", type=int, default=value)
    a = ap.parse_args()
    found, layer, _, (x, logits, dout) = compare(a.tokens, a.experts, a.k, a.width, a.hidden)
    print("distance from 32 bits: " + ", ".join(f"{n} {v:.3f}" for n, v in found.items()), flush=True)
    print(f"forward {milliseconds(lambda: layer.forward(x, logits)):.3f} ms, backward {milliseconds(lambda: layer.backward(dout)):.3f} ms", flush=True)
    few = DecodeStep(layer, 16, a.experts, a.width, a.hidden)
    print(f"step of 16 tokens {milliseconds(lambda: few(x[:16], logits[:16]), 100) * 1e3:.1f} us", flush=True)


if __name__ == "__main__":
    main()
