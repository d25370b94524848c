"""A trainable Transformer block over the dataflow blocks of schedules, from this library's operators.

The cost model's dataflow branch reads the data-movement blocks of a schedule in their order.  Here a small model of that kind (an
embedding, one attention block with a learned relative position bias, one feed-forward block, a pooled score) is trained to rank
candidates, its Siamese copy follows by momentum, and a sequence is scored as it grows, token by token against a cache:

    python examples/flow_block.py [--steps 60] [--candidates 512]

Forward, per block: norm (before) -> projection -> operator -> projection -> norm (after), gate and residual in one call with the next norm
before (`gated_norm`).  What the backward pass needs of activations is put away in 8 bits (`checkpoint=True`, `checkpoint_pack`): linear
layers take their weight gradients from there (`checkpoint_wgrad`) and the norms their block's output (`gated_norm_grad`).  Products that
are one plain matrix product are torch's.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2402_02361_amd as P  # noqa: E402

FEATURES = 23   # of a dataflow block


class FlowModel:
    """Parameters in float32 in one flat tensor (`phi`, as moa_update takes it), used in bfloat16."""

    def __init__(self, dim=64, heads=4, hidden=128, buckets=8, reach=16, seed=0, dtype=torch.bfloat16):
        self.dim, self.heads, self.head_dim, self.dtype = dim, heads, dim // heads, dtype
        self.edges = P.relative_edges(buckets - 1, reach)
        shapes = {"embed": (dim, FEATURES), "qkv": (3 * dim, dim), "out": (dim, dim), "up": (hidden, dim), "down": (dim, hidden), "table": (2 * buckets, heads),
                  "pre1": (dim,), "post1": (dim,), "gate1": (dim,), "pre2": (dim,), "post2": (dim,), "gate2": (dim,), "pre3": (dim,), "score": (dim,)}
        gen = torch.Generator().manual_seed(seed)
        self.phi = torch.zeros(sum(torch.Size(s).numel() for s in shapes.values()), device="cuda")
        self.p, at = {}, 0
        for name, shape in shapes.items():
            n = torch.Size(shape).numel()
            self.p[name] = self.phi[at:at + n].view(shape)
            at += n
            if name.startswith(("pre", "post")):
                self.p[name].fill_(1.0)
            elif name in ("embed", "qkv", "out", "up", "down", "score"):
                self.p[name].copy_(torch.randn(shape, generator=gen) * shape[-1] ** -0.5)

    def weight(self, name):
        return self.p[name].to(self.dtype)

    def forward(self, flow, n_blk):
        """flow [candidates, blocks, 23], n_blk int32 [candidates]: scores [candidates], and what backward needs."""
        batch, tokens, _ = flow.shape
        w, p = self.weight, self.p
        s = {"batch": batch, "tokens": tokens, "n_blk": n_blk, "in": P.checkpoint_pack(flow.to(self.dtype).view(-1, FEATURES))}
        x = s["x"] = flow.to(self.dtype).view(-1, FEATURES) @ w("embed").t()
        _, y, s["y1"] = P.gated_norm(x, None, None, p["pre1"], checkpoint=True)
        qkv = (y @ w("qkv").t()).view(batch, tokens, 3, self.heads, self.head_dim)
        s["q"], s["k"], s["v"] = qkv.unbind(2)
        o, s["lse"] = P.rel_attention(s["q"], s["k"], s["v"], w("table"), self.edges, q_len=n_blk, k_len=n_blk, want_lse=True)
        s["o"] = o
        f = o.view(-1, self.dim) @ w("out").t()
        s["o8"], s["f1"] = P.checkpoint_pack(o.view(-1, self.dim)), P.checkpoint_pack(f)
        h, y, s["y2"] = P.gated_norm(x, f, p["post1"], p["pre2"], gate=p["gate1"], checkpoint=True)
        s["h"] = h
        a = torch.relu(y @ w("up").t())
        f = a @ w("down").t()
        s["a"], s["f2"] = P.checkpoint_pack(a), P.checkpoint_pack(f)
        _, y, _ = P.gated_norm(h, f, p["post2"], p["pre3"], gate=p["gate2"])
        there = torch.arange(tokens, device="cuda")[None, :] < n_blk[:, None]
        s["pool"] = there / n_blk.clamp(min=1)[:, None]
        s["y3"] = y
        return ((y.float() @ p["score"]).view(batch, tokens) * s["pool"]).sum(1), s

    def backward(self, s, dscore):
        """The gradient of every parameter, as `phi` lies."""
        w, p = self.weight, self.p
        g = torch.zeros_like(self.phi)
        at, view = 0, {}
        for name, t in p.items():
            view[name] = g[at:at + t.numel()].view(t.shape)
            at += t.numel()
        each = (dscore[:, None] * s["pool"]).reshape(-1, 1)
        view["score"].copy_((each * s["y3"].float()).sum(0))
        dy = (each * p["score"]).to(self.dtype)
        dh, df, dgate, dpost, dpre = P.gated_norm_grad(None, dy, s["h"], s["f2"], p["post2"], p["pre3"], gate=p["gate2"])
        view["gate2"].copy_(dgate), view["post2"].copy_(dpost), view["pre3"].copy_(dpre)
        P.checkpoint_wgrad(df, s["a"], dw=view["down"])
        da = (df @ w("down")) * (s["a"].codes > 0)   # (a code is 0 where the activation is, or is too small to matter)
        P.checkpoint_wgrad(da, s["y2"], dw=view["up"])
        dx, df, dgate, dpost, dpre = P.gated_norm_grad(dh, da @ w("up"), s["x"], s["f1"], p["post1"], p["pre2"], gate=p["gate1"])
        view["gate1"].copy_(dgate), view["post1"].copy_(dpost), view["pre2"].copy_(dpre)
        P.checkpoint_wgrad(df, s["o8"], dw=view["out"])
        do = (df @ w("out")).view(s["o"].shape)
        dq, dk, dv, dtable = P.rel_attention_grad(do, s["q"], s["k"], s["v"], s["o"], s["lse"], w("table"), self.edges, q_len=s["n_blk"], k_len=s["n_blk"])
        view["table"].copy_(dtable)
        dqkv = torch.stack([dq, dk, dv], 2).view(-1, 3 * self.dim)
        P.checkpoint_wgrad(dqkv, s["y1"], dw=view["qkv"])
        dx, _, _, _, dpre = P.gated_norm_grad(dx, dqkv @ w("qkv"), s["x"], None, None, p["pre1"])
        view["pre1"].copy_(dpre)
        P.checkpoint_wgrad(dx, s["in"], dw=view["embed"])
        return g

    def grow(self, flow):
        """Attention's outputs for one candidate's blocks, [blocks, dim], each block scored when it arrives, against a cache of those before it (one-sided: what
        comes later is not known yet)."""
        w, p = self.weight, self.p
        tokens = flow.shape[0]
        past = w("table")[: len(self.edges) + 1].contiguous()
        cache = torch.zeros(2, 1, tokens, self.heads, self.head_dim, dtype=self.dtype, device="cuda")
        one, out = torch.ones(1, dtype=torch.int32, device="cuda"), []
        for t in range(tokens):
            x = flow[t:t + 1].to(self.dtype) @ w("embed").t()
            _, y, _ = P.gated_norm(x, None, None, p["pre1"])
            q, cache[0, 0, t], cache[1, 0, t] = (y @ w("qkv").t()).view(3, self.heads, self.head_dim).unbind(0)
            out.append(P.rel_attention(q.view(1, 1, self.heads, self.head_dim), cache[0], cache[1], past, self.edges, q_len=one, k_len=one * (t + 1), causal=True).view(1, -1))
        return torch.cat(out)


def rank_loss(score, latency, group):
    """Pairs of one task's candidates: the faster one is to score higher; the mean of log(1 + exp(-(difference))) and its gradient."""
    s, t = score.view(-1, group), latency.view(-1, group)
    faster = (t[:, :, None] < t[:, None, :]).float()
    d = s[:, :, None] - s[:, None, :]
    n = faster.sum().clamp(min=1)
    pull = -faster * torch.sigmoid(-d) / n
    return (faster * torch.nn.functional.softplus(-d)).sum() / n, (pull.sum(2) - pull.sum(1)).reshape(-1)


def synthetic(candidates, tokens, seed):
    """Features of up to `tokens` blocks, and a latency that depends on which blocks are neighbours."""
    gen = torch.Generator().manual_seed(seed)
    flow = torch.randn(candidates, tokens, FEATURES, generator=gen)
    n_blk = torch.randint(1, tokens + 1, (candidates,), generator=gen, dtype=torch.int32)
    there = torch.arange(tokens)[None, :] < n_blk[:, None]
    near = (flow[:, 1:, 0] * flow[:, :-1, 1] * (there[:, 1:] & there[:, :-1])).sum(1) + (flow[:, :, 2] * there).sum(1)
    return flow.cuda(), n_blk.cuda(), (near / n_blk).cuda()


def train(steps, candidates, group=32, tokens=8, lr=3e-3, seed=0, log=None):
    """Fine-tunes the target model by Adam, the Siamese weights following; returns (model, siamese weights, losses)."""
    model = FlowModel(seed=seed)
    siamese = model.phi.clone()
    m, v = torch.zeros_like(model.phi), torch.zeros_like(model.phi)
    flow, n_blk, latency = synthetic(candidates, tokens, seed)
    losses = []
    for step in range(1, steps + 1):
        score, kept = model.forward(flow, n_blk)
        loss, dscore = rank_loss(score, latency, group)
        g = model.backward(kept, dscore)
        m.mul_(0.9).add_(g, alpha=0.1)
        v.mul_(0.99).addcmul_(g, g, value=0.01)
        model.phi.addcdiv_(m / (1 - 0.9 ** step), (v / (1 - 0.99 ** step)).sqrt_().add_(1e-8), value=-lr)
        P.moa_update(siamese, model.phi, 0.99)
        losses.append(loss)
        if log and (step == 1 or step % 20 == 0):
            log(f"step {step}: ranking loss {loss.item():.4f}")
    return model, siamese, [float(x) for x in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--candidates", type=int, default=512)
    a = ap.parse_args()
    model, siamese, losses = train(a.steps, a.candidates, log=print)
    print(f"siamese weights follow at a distance of {(siamese - model.phi).norm().item():.3f}")
    grown = model.grow(synthetic(1, 8, 1)[0][0])
    print(f"one candidate's blocks as they arrive: {grown.shape[0]} outputs of {grown.shape[1]}")


if __name__ == "__main__":
    main()
