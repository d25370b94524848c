"""A call on a given stream takes no memory from work that is still under way on the current one, and what it returned or worked in is not given away while
it is in use: the entry points of the exploration round."""
import numpy as np
import pytest
import torch

import workloads as w
from test_gpu_parity import P, dev, lse_population  # noqa: F401  (P is a fixture)

pytestmark = pytest.mark.gpu

SG = [w.gemm(96, 80, 72, hw=w.toy_device()), w.gemm(60, 90, 64, hw=w.toy_device())]
LENS = [30000, 20000]


def _weights(make):
    return {k: (dev(v) if isinstance(v, np.ndarray) else v) for k, v in make.items()}


def _draft(P, seed):
    seg, tiles = lse_population(SG, LENS, seed=seed)
    tiles = dev(tiles)
    return lambda stream: P.draft_score(SG, seg, tiles, symbols=True, stream=stream)


def _topk(P, seed):
    seg = np.array([0, 30000, 50000], np.int64)
    score = torch.rand(50000, generator=torch.Generator().manual_seed(seed)).cuda()
    return lambda stream: P.topk(score, seg, 500, stream=stream)


def _prior_filter(P, seed):
    seg, tiles = lse_population(SG, LENS, seed=seed)
    tiles = dev(tiles)
    return lambda stream: P.prior_filter(SG, seg, tiles, 500, stream=stream)


def _lse(P, seed):
    seg, tiles = lse_population(SG, LENS, seed=seed)
    populations = {given: dev(tiles) for given in (False, True)}   # (each call moves its population on, which is the caller's to keep until then)
    return lambda stream: P.lse(SG, seg, populations[stream is not None], 100, 3, seed, 52429, stream=stream)


def _random_init(P, seed):
    seg = np.array([0, 30000, 50000], np.int64)
    rows = max(w.n_slots(s) for s in SG)
    return lambda stream: P.random_init(SG, seg, rows, seed, stream=stream)


def _verify(P, seed):
    gen = np.random.default_rng(seed)
    feat, n_stmt = dev(gen.normal(size=(3000, 8, 164)).astype(np.float32)), dev(gen.integers(1, 9, 3000).astype(np.int32))
    m = _weights(w.make_mlp_weights(seed=1))
    return lambda stream: P.verify_score(feat, n_stmt, m, stream=stream)


CALLS = [_draft, _topk, _prior_filter, _random_init, _verify]


def _tensors(r):
    return [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]


def _same(a, b):
    return len(a) == len(b) and all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.fixture(scope="module")
def busy():
    """Several milliseconds of work on the current stream."""
    a, out = (torch.zeros(4096, 4096, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    return lambda: [torch.mm(a, a, out=out) for _ in range(60)]


@pytest.mark.parametrize("make", CALLS)
def test_memory_that_pending_work_uses_is_left_alone(P, make, busy):
    call = make(P, 1)
    want = [t.clone() for t in _tensors(call(None))]
    held, more = _tensors(call(None)), [torch.empty_like(t) for t in want]
    copies = [torch.empty_like(t) for t in held]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy()
    for c, t in zip(copies, held):
        c.copy_(t)
    for t in more:
        t.zero_()
    t = held = more = None
    got = _tensors(call(side))
    torch.cuda.synchronize()
    assert _same(copies, want) and _same(got, want)


@pytest.mark.parametrize("make", CALLS + [_lse])
def test_what_a_call_works_in_stays_its_own(P, make, busy):
    call = make(P, 2)
    want = [t.clone() for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        busy()
    got = _tensors(call(side))
    junk = [torch.full((1 << n,), float("nan"), device="cuda") for n in range(22, 6, -1) for _ in range(3)]
    torch.cuda.synchronize()
    assert _same(got, want) and all(j.isnan().all() for j in junk)
