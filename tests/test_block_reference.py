"""The 64-bit reference of the block's operators against differences, and the host side of the entry points (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import block_reference as ref
import paper_2402_02361_amd as P
from paper_2402_02361_amd import binding as B

EINVAL, EWORKSPACE, OK = -1, -2, 0
FAKE = 0x1000


@pytest.fixture(scope="module")
def lib():
    return P.load_library()


def _difference(fun, at, index, step=1e-5):
    up, down = at.copy(), at.copy()
    up[index] += step
    down[index] -= step
    return (fun(up) - fun(down)) / (2 * step)


@pytest.mark.parametrize("causal,sides,lq,lk", [(False, 2, 5, 5), (True, 1, 4, 7), (True, 0, 6, 3), (False, 1, 3, 6)])
def test_attention_gradients_are_the_differences(causal, sides, lq, lk):
    rng = np.random.default_rng(3)
    q, k, v, do = rng.normal(size=(2, lq, 4, 8)), rng.normal(size=(2, lk, 2, 8)), rng.normal(size=(2, lk, 2, 8)), rng.normal(size=(2, lq, 4, 8))
    edges = [1, 2, 4]
    table = rng.normal(size=(sides * 4, 4)) if sides else None
    kw = dict(edges=edges, q_len=[lq, lq - 1], k_len=[lk, lk - 2], causal=causal)
    got = ref.attention(q, k, v, table, do=do, **kw)
    loss = lambda q=q, k=k, v=v, t=table: (ref.attention(q, k, v, t, **kw)["o"] * do).sum()  # noqa: E731
    for _ in range(6):
        for name, a, f in (("dq", q, lambda x: loss(q=x)), ("dk", k, lambda x: loss(k=x)), ("dv", v, lambda x: loss(v=x)), ("dtable", table, lambda x: loss(t=x))):
            if a is None:
                continue
            i = tuple(int(rng.integers(n)) for n in a.shape)
            assert abs(_difference(f, a, i) - got[name][i]) < 1e-7, (name, i)


@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("gated", [None, "rows", "vector"])
def test_norm_gradients_are_the_differences(center, gated):
    rng = np.random.default_rng(4)
    x, f, dh, dy = (rng.normal(size=(3, 10)) for _ in range(4))
    w1, w2 = 1 + 0.2 * rng.normal(size=10), 1 + 0.2 * rng.normal(size=10)
    gate = None if gated is None else rng.normal(size=(3, 10) if gated == "rows" else 10)

    def loss(x=x, f=f, w1=w1, w2=w2, g=gate):
        o = ref.norm(x, f, w1, w2, g, 0.7, 1e-3, center)
        return (o["h"] * dh).sum() + (o["y"] * dy).sum()

    got = ref.norm(x, f, w1, w2, gate, 0.7, 1e-3, center, dh, dy)
    for _ in range(6):
        for name, a, fun in (("dx", x, lambda t: loss(x=t)), ("df", f, lambda t: loss(f=t)), ("dw_post", w1, lambda t: loss(w1=t)), ("dw_pre", w2, lambda t: loss(w2=t)),
                             ("dgate", gate, lambda t: loss(g=t))):
            if a is None:
                continue
            i = tuple(int(rng.integers(n)) for n in a.shape)
            want = got[name].sum(0) if name == "dgate" and gated == "vector" else got[name]
            assert abs(_difference(fun, a, i) - want[i]) < 1e-7, (name, i)


def test_relative_edges():
    for n in (1, 2, 3, 7, 16, 31, 64):
        for far in {n, n + 1, 128, 1024}:
            if far < n:
                continue
            e = P.relative_edges(n, far)
            assert len(e) == n and e[0] == 1 and np.all(np.diff(e) > 0) and e[-1] == (far if n > 1 else 1)
    with pytest.raises(AssertionError):
        P.relative_edges(65, 128)


def test_buckets_of_hand_made_edges():
    assert ref.buckets([-9, -4, -3, -1, 0, 1, 3, 4, 9], [1, 4], False).tolist() == [2, 2, 1, 1, 0, 0, 0, 0, 0]
    assert ref.buckets([-9, -4, -3, -1, 0, 1, 3, 4, 9], [1, 4], True).tolist() == [2, 2, 1, 1, 0, 4, 4, 5, 5]


def test_struct_sizes_match_the_header():
    assert C.sizeof(B.CCheckpoint) == 16 and C.sizeof(B.CNorm) == 8 + 3 * 4 + 2 * 4 + 4 + 4 * 8
    assert C.sizeof(B.CHeads) == 32 and C.sizeof(B.CAttention) == 8 * 4 + 4 + 4 + 4 * 8 + 8


def _kept(codes=FAKE, exps=FAKE):
    return C.byref(B.CCheckpoint(codes, exps))


def test_checkpoints_refuse(lib):
    f = lib.pruner_checkpoint_pack
    assert f(None, 0, 0, 8, 8, None, None) == OK                             # no rows: nothing to do
    assert f(None, 0, 4, 8, 8, _kept(), None) == EINVAL
    assert f(FAKE, 0, 4, 8, 8, None, None) == EINVAL
    assert f(FAKE + 1, 0, 4, 8, 8, _kept(), None) == EINVAL                  # misaligned
    assert f(FAKE + 2, 2, 4, 8, 8, _kept(), None) == EINVAL
    assert f(FAKE, 3, 4, 8, 8, _kept(), None) == EINVAL                      # unknown type
    assert f(FAKE, 0, 4, 0, 8, _kept(), None) == EINVAL and f(FAKE, 0, -1, 8, 8, _kept(), None) == EINVAL
    assert f(FAKE, 0, 4, 8, 7, _kept(), None) == EINVAL                      # pitch below dim
    assert f(FAKE, 0, 1 << 30, 8, 1 << 12, _kept(), None) == EINVAL          # beyond 2^40 values
    assert f(FAKE, 0, 4, 8, 8, _kept(codes=FAKE + 4), None) == EINVAL and f(FAKE, 0, 4, 8, 8, _kept(exps=None), None) == EINVAL
    g = lib.pruner_checkpoint_restore
    assert g(None, 0, 0, 8, None, 8, None) == OK and g(_kept(), 0, 4, 8, None, 8, None) == EINVAL and g(_kept(), 0, 4, 8, FAKE, 7, None) == EINVAL


def test_weight_gradient_refuses(lib):
    f, need = lib.pruner_checkpoint_wgrad, lib.pruner_checkpoint_wgrad_workspace_bytes
    assert need(65536, 256, 256) > 256 and need(-1, 8, 8) == 0 and need(8, 0, 8) == 0 and need(8, 8, 1 << 21) == 0
    assert np.all(np.diff([need(n, 256, 256) for n in (1, 500, 600, 5000, 100000, 1 << 24)]) >= 0)
    ok = (FAKE, 0, 256, _kept(), 65536, 256, 256, FAKE, 0, FAKE, need(65536, 256, 256) - 1, None)
    assert f(*ok) == EWORKSPACE
    assert f(None, 0, 8, None, 0, 8, 8, FAKE, 1, None, 0, None) == OK          # no rows, added to: nothing to do
    for i, bad in ((0, None), (0, FAKE + 1), (1, 2), (1, -1), (2, 255), (3, None), (4, -1), (5, 0), (6, 0), (7, None), (7, FAKE + 2), (8, 2)):
        assert f(*[bad if j == i else a for j, a in enumerate(ok)]) == EINVAL, (i, bad)


def _norm(rows=4, dim=64, dtype=0, center=0, alpha=1.0, eps=1e-6, w_post=FAKE, w_pre=FAKE, gate=None, pitch=0):
    return C.byref(B.CNorm(rows, dim, dtype, center, alpha, eps, w_post, w_pre, gate, pitch))


def test_norms_refuse(lib):
    f = lib.pruner_gated_norm
    call = lambda p, x=FAKE, xp=64, ff=FAKE, fp=64, h=FAKE, y=FAKE, kept=None: f(p, x, xp, ff, fp, h, y, kept, None)  # noqa: E731
    assert call(_norm(rows=0), x=None) == OK
    for bad in (dict(rows=-1), dict(dim=0), dict(dim=8193), dict(dtype=3), dict(alpha=float("nan")), dict(alpha=float("inf")), dict(eps=-1.0), dict(eps=float("nan")),
                dict(w_post=None), dict(w_pre=None), dict(w_pre=FAKE + 2), dict(gate=FAKE, pitch=63), dict(gate=FAKE + 1, pitch=64), dict(gate=FAKE + 2), dict(pitch=-1)):
        assert call(_norm(**bad)) == EINVAL, bad
    for bad in (dict(x=None), dict(x=FAKE + 1), dict(xp=63), dict(fp=63), dict(ff=FAKE + 1), dict(h=FAKE + 1), dict(y=FAKE + 1), dict(h=None, y=None), dict(kept=_kept(codes=None))):
        assert call(_norm(), **bad) == EINVAL, bad
    g, need = lib.pruner_gated_norm_grad, lib.pruner_gated_norm_grad_workspace_bytes
    names = ("p", "dh", "dhp", "dy", "dyp", "x", "xp", "f", "fp", "kept", "dx", "df", "dgate", "dw1", "dw2", "ws", "wsb", "st")
    ok = dict(zip(names, (_norm(), FAKE, 64, FAKE, 64, FAKE, 64, FAKE, 64, None, FAKE, FAKE, None, FAKE, FAKE, FAKE, need(4, 64), None)))
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(wsb=need(4, 64) - 1)):
        assert g(*{**ok, **bad}.values()) == EWORKSPACE, bad
    for bad in (dict(dy=None), dict(dhp=63), dict(dyp=8), dict(x=None), dict(kept=_kept()), dict(dx=None), dict(df=None), dict(dw1=None), dict(dw2=None), dict(p=_norm(gate=FAKE, pitch=64)),
                dict(p=_norm(w_post=None)), dict(dx=FAKE + 1)):
        assert g(*{**ok, **bad}.values()) == EINVAL, bad


def _attention(**kw):
    f = dict(dtype=0, batch=2, q_tokens=64, k_tokens=64, q_heads=4, kv_heads=2, head_dim=64, flags=0, scale=0.125, q_len=None, k_len=None, table=None, edges=None, n_edges=0)
    f.update(kw)
    return C.byref(B.CAttention(**f))


def _h(p=FAKE, batch=64 * 64, token=64, head=64):
    return C.byref(B.CHeads(p, batch, token, head))


def test_attention_refuses(lib):
    f, need = lib.pruner_rel_attention, lib.pruner_rel_attention_workspace_bytes
    edges = np.array([1, 2, 4], np.int32)
    down, far, zero = (np.array(e, np.int32) for e in ([1, 4, 4], [1, 2, 1025], [0, 1, 2]))
    assert f(_attention(batch=0), None, None, None, None, None, None, 0, None) == OK
    assert f(_attention(q_tokens=0), None, None, None, None, None, None, 0, None) == OK
    for bad in (dict(dtype=2), dict(batch=-1), dict(q_tokens=-1), dict(k_tokens=1 << 30), dict(q_heads=3), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=4), dict(head_dim=132),
                dict(head_dim=136), dict(flags=4), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(n_edges=65), dict(n_edges=-1),
                dict(batch=1 << 24), dict(q_len=FAKE + 2), dict(table=FAKE + 1), dict(table=FAKE, n_edges=3),
                *(dict(table=FAKE, n_edges=3, edges=e.ctypes.data) for e in (down, far, zero))):
        assert f(_attention(**bad), _h(), _h(), _h(), _h(), None, FAKE, 1 << 40, None) == EINVAL, bad
    ok = _attention(table=FAKE, n_edges=3, edges=edges.ctypes.data)
    for bad in (_h(p=None), _h(p=FAKE + 8), _h(token=60), _h(head=4), _h(batch=12), _h(token=(1 << 22) + 8), _h(token=-8), None):
        for i in range(4):
            assert f(ok, *[bad if j == i else _h() for j in range(4)], None, FAKE, 1 << 40, None) == EINVAL, (bad, i)
    assert f(ok, _h(), _h(), _h(), _h(), FAKE + 2, FAKE, 1 << 40, None) == EINVAL
    long = dict(batch=1, q_tokens=1, k_tokens=1 << 20)                        # split over workgroups: needs its workspace
    assert need(_attention(**long)) > 256 and need(_attention(batch=-1)) == 0
    assert f(_attention(**long), _h(), _h(), _h(), _h(), None, FAKE, need(_attention(**long)) - 1, None) == EWORKSPACE
    assert f(_attention(**long), _h(), _h(), _h(), _h(), None, None, 1 << 40, None) == EWORKSPACE
    g, need = lib.pruner_rel_attention_grad, lib.pruner_rel_attention_grad_workspace_bytes
    call = lambda a, lse=FAKE, dtable=None, ws=FAKE, size=1 << 40, **h: g(a, *[h.get(n, _h()) for n in ("do", "q", "k", "v", "o")], lse, *[h.get(n, _h()) for n in ("dq", "dk", "dv")],  # noqa: E731
                                                                         dtable, ws, size, None)
    assert call(_attention(), ws=None) == EWORKSPACE and call(_attention(), size=need(_attention()) - 1) == EWORKSPACE and call(_attention(), ws=FAKE + 128) == EWORKSPACE
    assert call(_attention(), lse=None) == EINVAL and call(_attention(), dtable=FAKE) == EINVAL and call(ok) == EINVAL and call(ok, dtable=FAKE + 1) == EINVAL
    for n in ("do", "q", "k", "v", "o", "dq", "dk", "dv"):
        assert call(_attention(), **{n: _h(p=FAKE + 8)}) == EINVAL and call(_attention(), **{n: None}) == EINVAL, n
