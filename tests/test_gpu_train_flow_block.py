"""The example that trains a block from the library's operators: its gradients against torch's own of the same model in binary32, that it learns, and that a
sequence scored as it grows gives what it gives at once."""
import os
import sys

import pytest
import torch

import paper_2402_02361_amd as P

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


def _plain(model, phi, flow, n_blk):
    """The model in binary32, by elementary operations that torch differentiates."""
    p, at = {}, 0
    for name, t in model.p.items():
        p[name] = phi[at:at + t.numel()].view(t.shape)
        at += t.numel()
    batch, tokens, _ = flow.shape
    norm = lambda x: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    x = flow @ p["embed"].t()
    q, k, v = ((norm(x) * p["pre1"]) @ p["qkv"].t()).view(batch, tokens, 3, model.heads, model.head_dim).permute(2, 0, 3, 1, 4)
    r = torch.arange(tokens, device="cuda")[None, :] - torch.arange(tokens, device="cuda")[:, None]
    n = torch.bucketize(r.abs(), torch.from_numpy(model.edges).cuda().long(), right=True) + (r > 0) * (len(model.edges) + 1)
    s = (q[:, :, :, None] * k[:, :, None]).sum(-1) * model.head_dim ** -0.5 + p["table"][n].permute(2, 0, 1)
    there = torch.arange(tokens, device="cuda")[None, :] < n_blk[:, None]
    a = torch.softmax(s.masked_fill(~there[:, None, None], -1e30), -1)
    o = (a[..., None] * v[:, :, None]).sum(3) * there[:, None, :, None]
    f = o.permute(0, 2, 1, 3).reshape(batch, tokens, -1) @ p["out"].t()
    h = x + torch.sigmoid(p["gate1"]) * norm(f) * p["post1"]
    f = torch.relu((norm(h) * p["pre2"]) @ p["up"].t()) @ p["down"].t()
    y = norm(h + torch.sigmoid(p["gate2"]) * norm(f) * p["post2"]) * p["pre3"]
    return ((y @ p["score"]) * there / n_blk.clamp(min=1)[:, None]).sum(1)


def test_gradients_are_those_of_the_model():
    """Activations in 16 bits, and in 8 for the weight gradients: the gradient of every parameter points where that in binary32 points.  A step of 8 bits is
    2^-7 of a group's largest value and of random sign, so a gradient over hundreds of rows is off by far less than a tenth."""
    from flow_block import FlowModel, rank_loss, synthetic
    model = FlowModel(seed=3)
    flow, n_blk, latency = synthetic(256, 8, 5)
    with torch.no_grad():
        for name in ("gate1", "gate2", "table"):
            model.p[name].copy_(torch.randn(model.p[name].shape, generator=torch.Generator().manual_seed(len(name))) * 0.3)
    phi = model.phi.clone().requires_grad_(True)
    want = _plain(model, phi, flow, n_blk)
    score, kept = model.forward(flow, n_blk)
    assert (score - want).abs().max() <= 0.05 * want.abs().max()
    _, dscore = rank_loss(want.detach(), latency, 32)
    (want * dscore).sum().backward()
    got, at = model.backward(kept, dscore), 0
    for name, t in model.p.items():
        a, b = got[at:at + t.numel()], phi.grad[at:at + t.numel()]
        at += t.numel()
        assert (a - b).norm() <= 0.1 * b.norm(), name


def test_it_learns():
    from flow_block import train
    _, siamese, losses = train(40, 256)
    assert losses[-1] < 0.8 * losses[0] and torch.isfinite(siamese).all()


def test_a_growing_sequence():
    from flow_block import FlowModel, synthetic
    model = FlowModel(seed=4)
    flow = synthetic(1, 8, 6)[0]
    grown = model.grow(flow[0])
    x = flow.bfloat16().view(-1, 23) @ model.weight("embed").t()
    _, y, _ = P.gated_norm(x, None, None, model.p["pre1"])
    q, k, v = (y @ model.weight("qkv").t()).view(1, 8, 3, model.heads, model.head_dim).unbind(2)
    whole = P.rel_attention(q, k, v, model.weight("table")[: len(model.edges) + 1].contiguous(), model.edges, causal=True).view(8, -1)
    assert (grown - whole).abs().max() <= 2.0 ** -6 * whole.abs().max()
