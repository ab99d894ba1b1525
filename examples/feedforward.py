"""The feed-forward half of a transformer block on 2:4 weights: decoding with 8-bit rows, and a few fine-tuning steps of experts.

    python examples/feedforward.py

``QuantisedBlock``  norm and 8-bit rows in one pass, up-projection with its activation, 8-bit rows again, down-projection onto the residual stream
``Experts``         one projection of every expert: pruned so that the transposed weights satisfy the pattern too, forward, gradients, update
``ExpertBlock``     norm, tokens sorted to their experts, both projections, and back onto the residual stream; its gradients
``RoutedBlock``     the same behind a router of its own, with everything that the gradients need kept in 8 bits
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2104_08378_amd import sp24  # noqa: E402


class QuantisedBlock:
    """Weights as int8 with a scale for each output feature, activations with a scale for each token."""

    def __init__(self, norm, up, down):
        self.norm = norm
        self.up, self.down = self._quantised(up), self._quantised(down)

    @staticmethod
    def _quantised(W):
        codes, scale = sp24.sp24_quantize_rows(sp24.sp24_prune(W), torch.int8)
        return *sp24.sp24_compress(codes, layout="tiled"), scale

    def __call__(self, x, stream):
        """Adds the block to the residual stream in place; x: what the part before it adds."""
        n = sp24.sp24_rmsnorm(x, self.norm, residual=stream, hidden=stream, out_dtype=torch.int8)
        V, meta, scale = self.up
        h = sp24.sp24_linear(V, meta, n.y, torch.bfloat16, w_scale=scale, x_scale=n.scale, act="silu", layout="tiled")
        codes, rows = sp24.sp24_quantize_rows(h, torch.int8)
        V, meta, scale = self.down
        return sp24.sp24_linear(V, meta, codes, torch.bfloat16, w_scale=scale, x_scale=rows, residual=stream, layout="tiled", out=stream)


class Experts:
    """[experts * M, K] weights, one matrix below the other, kept in float32 and used as bfloat16."""

    def __init__(self, weights, experts):
        self.experts = experts
        self.master = sp24.sp24_prune_transposable(weights.to(torch.bfloat16)).float()
        W = self.master.to(torch.bfloat16)
        self.V, self.meta = sp24.sp24_compress(W, layout="tiled")
        self.Vt, self.meta_t = sp24.sp24_compress(self._turned(W), layout="tiled")

    def _turned(self, W):
        M, K = W.shape[0] // self.experts, W.shape[1]
        return W.view(self.experts, M, K).transpose(1, 2).reshape(self.experts * K, M).contiguous()

    def __call__(self, x, offsets, **epilogue):
        return sp24.sp24_linear_grouped(self.V, self.meta, x, offsets, torch.bfloat16, layout="tiled", **epilogue)

    def backward(self, dY, preact, act, x, offsets):
        """(gradient of x, of the weights at their kept positions, of the bias)"""
        dZ, dZt, dbias = sp24.sp24_linear_backward(dY, preact, act, offsets=offsets)
        dx = sp24.sp24_linear_grouped(self.Vt, self.meta_t, dZ, offsets, torch.bfloat16, layout="tiled")
        dW = sp24.sp24_gemm_dense_grouped(dZt, x, offsets, torch.bfloat16).view(self.master.shape)
        return dx, sp24.sp24_mask_apply(dW, self.meta, layout="tiled", out=dW), dbias

    def update(self, dW, rate):
        """A gradient step; the pattern stays, only the values are compressed again."""
        self.master.sub_(dW, alpha=rate)
        W = self.master.to(torch.bfloat16)
        self.V = sp24.sp24_compress_masked(W, self.meta, layout="tiled")
        self.Vt = sp24.sp24_compress_masked(self._turned(W), self.meta_t, layout="tiled")


class ExpertBlock:
    def __init__(self, norm, up, down, bias, experts):
        self.norm, self.bias, self.experts = norm, bias, experts
        self.up, self.down = Experts(up, experts), Experts(down, experts)

    def __call__(self, x, stream, ids, weights):
        """The new residual stream, and what the gradients need.  ids, weights [N, topk]: the router's choices."""
        n = sp24.sp24_rmsnorm(x, self.norm, residual=stream, want_rstd=True)
        offsets, slots, rows = sp24.sp24_moe_sort(ids, self.experts)
        xs = sp24.sp24_moe_gather(n.y, rows, ids.shape[1])
        z = torch.empty(rows.numel(), self.up.V.shape[0] // self.experts, dtype=torch.bfloat16, device=x.device)
        h = self.up(xs, offsets, bias=self.bias, act="gelu", preact=z)
        ys = self.down(h, offsets)
        out = sp24.sp24_moe_combine(ys, slots, weights, residual=n.hidden)
        return out, (n, offsets, slots, rows, xs, z, h, ys, weights)

    def backward(self, dout, kept):
        n, offsets, slots, rows, xs, z, h, ys, weights = kept
        dys, dweights = sp24.sp24_moe_combine_backward(dout, ys, slots, rows, weights)
        dh, ddown, _ = self.down.backward(dys, None, "none", h, offsets)
        dxs, dup, dbias = self.up.backward(dh, z, "gelu", xs, offsets)
        dx, dnorm = sp24.sp24_rmsnorm_backward(sp24.sp24_moe_combine(dxs, slots), n.hidden, self.norm, n.rstd, dhidden=dout)
        return dict(x=dx, norm=dnorm, up=dup, down=ddown, bias=dbias.reshape(-1), weights=dweights)


class RoutedBlock(ExpertBlock):
    """Keeps a byte, not two, for every value of the rows in front of and behind the activation, of the experts' results, and of the normed rows, which are
    kept once a token, whatever the number of its experts."""

    def __init__(self, norm, up, down, bias, router, experts, topk, **routing):
        super().__init__(norm, up, down, bias, experts)
        self.router, self.topk, self.routing = router.to(torch.bfloat16), topk, routing

    def __call__(self, x, stream, balance=None):
        """(the new residual stream, how many choices every expert has, what the gradients need).  balance [experts]: added to the scores for the choice."""
        n = sp24.sp24_rmsnorm(x, self.norm, residual=stream, want_rstd=True)
        logits = sp24.sp24_gemm_dense(n.y, self.router, torch.float32)
        r = sp24.sp24_moe_route(logits, self.topk, bias=balance, want_load=True, **self.routing)
        offsets, slots, rows = sp24.sp24_moe_sort(r.ids, self.experts)
        z = torch.empty(rows.numel(), self.up.V.shape[0] // self.experts, dtype=torch.bfloat16, device=x.device)
        h = self.up(sp24.sp24_moe_gather(n.y, rows, self.topk), offsets, bias=self.bias, act="gelu", preact=z)
        ys = self.down(h, offsets)
        out = sp24.sp24_moe_combine(ys, slots, r.weights, residual=n.hidden)
        return out, r.load, (n.hidden, n.rstd, logits, r, offsets, slots, rows, *(sp24.sp24_checkpoint_rows(t) for t in (n.y, z, h, ys)))

    def backward(self, dout, kept):
        hidden, rstd, logits, r, offsets, slots, rows, y, z, h, ys = kept
        how = {k: v for k, v in self.routing.items() if k in ("score", "renormalise", "scale")}
        dys, dweights = sp24.sp24_moe_combine_backward(dout, sp24.sp24_restore_rows(ys, torch.bfloat16), slots, rows, r.weights)
        ddown = sp24.sp24_gemm_dense_grouped_checkpoint(dys.t(), h, offsets, torch.bfloat16).view(self.down.master.shape)
        dh = sp24.sp24_linear_grouped(self.down.Vt, self.down.meta_t, dys, offsets, torch.bfloat16, layout="tiled")
        dz, dzt, dbias = sp24.sp24_linear_backward_checkpoint(dh, z, "gelu", offsets=offsets)
        dup = sp24.sp24_gemm_dense_grouped_checkpoint(dzt, y, offsets, torch.bfloat16, rows=rows, topk=self.topk).view(self.up.master.shape)
        dxs = sp24.sp24_linear_grouped(self.up.Vt, self.up.meta_t, dz, offsets, torch.bfloat16, layout="tiled")
        # the router's rows are as wide as there are experts; the products ask for whole 16 bytes
        dl = torch.zeros(logits.shape[0], -(-self.experts // 8) * 8, dtype=torch.bfloat16, device=logits.device)[:, :self.experts]
        dl.copy_(sp24.sp24_moe_route_backward(logits, r.ids, dweights, **how))
        drouter = sp24.sp24_gemm_dense_checkpoint(dl.t(), y, torch.float32)
        dy = sp24.sp24_moe_combine(dxs, slots, residual=sp24.sp24_gemm_dense(dl, self.router, torch.bfloat16, b_order="n"))
        dx, dnorm = sp24.sp24_rmsnorm_backward(dy, hidden, self.norm, rstd, dhidden=dout)
        return dict(x=dx, norm=dnorm, up=sp24.sp24_mask_apply(dup, self.up.meta, layout="tiled"), down=sp24.sp24_mask_apply(ddown, self.down.meta, layout="tiled"),
                    bias=dbias.reshape(-1), router=drouter)


def decode(g, H=1024, F=4096, tokens=16):
    """Relative distance of the 8-bit block from the same weights in float32."""
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    norm, up, down = 1 + 0.1 * n(H), (n(F, H) / H ** 0.5).to(torch.bfloat16), (n(H, F) / F ** 0.5).to(torch.bfloat16)
    x, stream = n(tokens, H).to(torch.bfloat16), n(tokens, H).to(torch.bfloat16)
    h = x.float() + stream.float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * norm
    want = h + torch.nn.functional.silu(y @ sp24.sp24_prune(up).float().t()) @ sp24.sp24_prune(down).float().t()
    got = QuantisedBlock(norm, up, down)(x, stream)
    return float((got.float() - want).norm() / want.norm())


def fine_tune(g, H=256, F=512, experts=8, topk=2, tokens=512, steps=12, rate=0.5):
    """Losses of gradient steps towards the outputs of another block of the same kind."""
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    make = lambda: ExpertBlock(1 + 0.1 * n(H), n(experts * F, H) / H ** 0.5, n(experts * H, F) / F ** 0.5, 0.1 * n(experts * F), experts)  # noqa: E731
    teacher, student = make(), make()
    x, stream = n(tokens, H).to(torch.bfloat16), n(tokens, H).to(torch.bfloat16)
    choice = n(tokens, experts).topk(topk, dim=1)
    ids, weights = choice.indices.to(torch.int32), torch.softmax(choice.values, 1)
    target = teacher(x, stream, ids, weights)[0].float()
    losses = []
    for _ in range(steps):
        out, kept = student(x, stream, ids, weights)
        off = out.float() - target
        losses.append(float(off.square().mean()))
        d = student.backward((off / tokens ** 0.5).to(torch.bfloat16), kept)
        student.up.update(d["up"], rate / tokens ** 0.5)
        student.down.update(d["down"], rate / tokens ** 0.5)
        student.norm -= rate / tokens * d["norm"]
        student.bias -= rate / tokens ** 0.5 * d["bias"]
    return losses


def balance(g, H=256, F=512, experts=8, topk=2, tokens=512, steps=8, rate=0.02):
    """The largest share of the choices that one expert has, step by step, while the bias follows the load."""
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    block = RoutedBlock(1 + 0.1 * n(H), n(experts * F, H) / H ** 0.5, n(experts * H, F) / F ** 0.5, 0.1 * n(experts * F), n(experts, H) / H ** 0.5, experts, topk,
                        score="sigmoid", groups=4, groups_kept=2, scale=2.0)
    x, stream = n(tokens, H).to(torch.bfloat16) + 0.5 * n(H).to(torch.bfloat16), n(tokens, H).to(torch.bfloat16)
    bias, shares = torch.zeros(experts, device="cuda"), []
    for _ in range(steps):
        load = block(x, stream, bias)[1].float()
        shares.append(float(load.max() / load.sum()))
        bias += rate * torch.sign(load.mean() - load)
    return shares


if __name__ == "__main__":
    generator = torch.Generator(device="cuda").manual_seed(0)
    print("decoding in 8 bits against float32, relative distance: %.4f" % decode(generator))
    print("fine-tuning experts, loss by step: " + " ".join("%.4f" % v for v in fine_tune(generator)))
    print("balancing experts, largest share by step: " + " ".join("%.3f" % v for v in balance(generator)))
