"""What a call of the block's operators allocates for itself stays its own while another stream still works with it."""
import pytest
import torch

import paper_2402_02361_amd as P

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _attention():
    gen = torch.Generator().manual_seed(1)
    q, k, v, do = ((torch.randn(1, 1500, 2, 64, generator=gen)).to(BF).cuda() for _ in range(4))
    edges = P.relative_edges(8, 64)
    table = torch.randn(len(edges) + 1, 2, generator=gen).to(BF).cuda()
    o, lse = P.rel_attention(q, k, v, table, edges, causal=True, want_lse=True)
    return lambda stream: (P.rel_attention(q, k, v, table, edges, causal=True, stream=stream), *P.rel_attention_grad(do, q, k, v, o, lse, table, edges, causal=True, stream=stream))


def _norm():
    gen = torch.Generator().manual_seed(2)
    x, f, dy = (torch.randn(2000, 320, generator=gen).to(BF).cuda() for _ in range(3))
    w = torch.rand(320, generator=gen).cuda() + 0.5
    return lambda stream: P.gated_norm_grad(None, dy, x, f, w, w, stream=stream)


def _wgrad():
    gen = torch.Generator().manual_seed(3)
    dy, x = (torch.randn(6000, n, generator=gen).to(BF).cuda() for n in (200, 136))
    kept = P.checkpoint_pack(x)
    return lambda stream: P.checkpoint_wgrad(dy, kept, stream=stream)


@pytest.mark.parametrize("make", [_attention, _norm, _wgrad])
def test_scratch_is_not_given_away(make):
    call = make()
    as_list = lambda r: [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]  # noqa: E731
    want = as_list(call(None))
    a = torch.randn(4096, 4096, device="cuda", dtype=BF)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(60):   # (several milliseconds before the call's first launch)
            a @ a
    got = as_list(call(side))
    # what the current stream makes next must not lie where the call still writes
    junk = [torch.full((1 << n,), float("nan"), device="cuda") for n in range(22, 6, -1) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and all(j.isnan().all() for j in junk)
