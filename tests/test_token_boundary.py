"""What the calls of a token step refuse: every call below returns from checks on the host, before anything is launched (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import paper_2402_02361_amd as P
import paper_2402_02361_amd.binding as B

OK, EINVAL, EWORKSPACE = 0, -1, -2
FAKE = 0x1000   # aligned, never dereferenced on these paths
FREQS = np.array([1.0, 0.5, 0.25, 0.125])


@pytest.fixture(scope="module")
def lib():
    return P.load_library()


def _heads(p=FAKE, batch=1024, token=256, head=64):
    return C.byref(B.CHeads(p, batch, token, head))


def _rotation(**kw):
    d = dict(dtype=0, batch=2, tokens=3, q_heads=4, kv_heads=2, head_dim=64, rotary_dim=8, flags=0, amplitude=1.0, freqs=FREQS.ctypes.data, positions=0, q_len=0, k_len=0)
    d.update(kw)
    return C.byref(B.CRotation(*d.values()))


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(batch=-1), dict(tokens=-1), dict(tokens=1 << 30), dict(batch=1 << 15, tokens=1 << 15), dict(q_heads=-1), dict(kv_heads=65536),
                                 dict(head_dim=1), dict(head_dim=513), dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=66), dict(head_dim=512, rotary_dim=258), dict(flags=2),
                                 dict(amplitude=float("inf")), dict(amplitude=float("nan")), dict(freqs=0), dict(positions=0x1002), dict(q_len=0x1001), dict(k_len=0x1002)])
def test_rotary_refuses(lib, bad):
    for call in (lib.pruner_rotary, lib.pruner_rotary_grad):
        assert call(_rotation(**bad), _heads(), _heads(), _heads(0x2000), _heads(0x2000), None) == EINVAL


def test_rotary_refuses_frequencies_and_rows(lib):
    for f in (65.0, -65.0, float("nan"), float("inf")):
        freqs = np.array([1.0, f, 1.0, 1.0])
        assert lib.pruner_rotary(_rotation(freqs=freqs.ctypes.data), _heads(), _heads(), _heads(), _heads(), None) == EINVAL
    far = _heads(0x2000)
    for q, k, qo, ko in ((None, _heads(), far, far), (_heads(), None, far, far), (_heads(), _heads(), None, far), (_heads(), _heads(), far, None), (_heads(0), _heads(), far, far),
                         (_heads(0x1001), _heads(), far, far), (_heads(token=-8), _heads(), far, far), (_heads(), _heads(), _heads(token=128), _heads()), (_heads(), _heads(), _heads(head=8), _heads())):
        assert lib.pruner_rotary(_rotation(), q, k, qo, ko, None) == EINVAL
    assert lib.pruner_rotary(_rotation(dtype=2), _heads(0x1002), _heads(), far, far, None) == EINVAL
    assert lib.pruner_rotary(None, _heads(), _heads(), far, far, None) == EINVAL
    # nothing to do
    assert lib.pruner_rotary(_rotation(batch=0), None, None, None, None, None) == OK
    assert lib.pruner_rotary(_rotation(tokens=0), None, None, None, None, None) == OK
    assert lib.pruner_rotary(_rotation(q_heads=0, kv_heads=0), None, None, None, None, None) == OK


def _cache(**kw):
    d = dict(k_codes=FAKE, v_codes=FAKE, k_exps=FAKE, v_exps=FAKE, table=FAKE, pages=10, page_tokens=64, kv_heads=2, head_dim=64, seq_pages=4)
    d.update(kw)
    return C.byref(B.CCache(*d.values()))


BAD_CACHES = [dict(k_codes=0), dict(v_codes=0), dict(k_exps=0), dict(v_exps=0), dict(k_codes=0x1008), dict(v_codes=0x1004), dict(table=0x1002), dict(pages=-1), dict(page_tokens=0), dict(page_tokens=8),
              dict(page_tokens=48), dict(page_tokens=512), dict(kv_heads=0), dict(kv_heads=65536), dict(head_dim=0), dict(head_dim=24), dict(head_dim=144), dict(seq_pages=-1), dict(seq_pages=1 << 24),
              dict(table=0, pages=7)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_every_call_refuses(lib, bad):
    assert lib.pruner_cache_append(_cache(**bad), 0, 2, 3, _heads(), _heads(), None, None, None) == EINVAL
    assert lib.pruner_cache_restore(_cache(**bad), 0, 2, 3, None, _heads(), _heads(), None) == EINVAL
    a = _attention(**{k: v for k, v in bad.items() if k in ("kv_heads", "head_dim")})
    assert lib.pruner_cache_attention(a, _cache(**bad), _heads(), _heads(), None, None, 0, None) == EINVAL


def test_append_and_restore_refuse(lib):
    for bad in (dict(dtype=3), dict(dtype=-1), dict(batch=-1), dict(tokens=-1), dict(tokens=1 << 30), dict(k=None), dict(v=None), dict(k=_heads(0)), dict(v=_heads(0x1001)), dict(k=_heads(token=-8)),
                dict(k_len=0x1002)):
        d = dict(dtype=0, batch=2, tokens=3, k=_heads(), v=_heads(), k_len=None)
        d.update(bad)
        assert lib.pruner_cache_append(_cache(), d["dtype"], d["batch"], d["tokens"], d["k"], d["v"], None, d["k_len"], None) == EINVAL
        assert lib.pruner_cache_restore(_cache(), d["dtype"], d["batch"], d["tokens"], d["k_len"], d["k"], d["v"], None) == EINVAL
    assert lib.pruner_cache_append(_cache(), 0, 2, 3, _heads(), _heads(), 0x1002, None, None) == EINVAL
    assert lib.pruner_cache_restore(_cache(), 0, 2, 4 * 64 + 1, None, _heads(), _heads(), None) == EINVAL            # more than a sequence has room for
    assert lib.pruner_cache_append(_cache(kv_heads=60000), 0, 1000, 64, _heads(), _heads(), None, None, None) == EINVAL   # too many workgroups
    assert lib.pruner_cache_append(None, 0, 2, 3, _heads(), _heads(), None, None, None) == EINVAL
    for c in (lib.pruner_cache_append(_cache(), 0, 0, 3, None, None, None, None, None), lib.pruner_cache_append(_cache(), 0, 2, 0, None, None, None, None, None),
              lib.pruner_cache_append(_cache(pages=0, k_codes=0, v_codes=0, k_exps=0, v_exps=0), 0, 2, 3, _heads(), _heads(), None, None, None),
              lib.pruner_cache_restore(_cache(), 0, 0, 3, None, None, None, None), lib.pruner_cache_restore(_cache(), 0, 2, 0, None, None, None, None)):
        assert c == OK


def _attention(**kw):
    d = dict(dtype=0, batch=2, q_tokens=1, k_tokens=256, q_heads=4, kv_heads=2, head_dim=64, flags=1, scale=0.125, q_len=0, k_len=0, table=0, edges=0, n_edges=0)
    d.update(kw)
    return C.byref(B.CAttention(*d.values()))


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(batch=-1), dict(q_tokens=-1), dict(k_tokens=-1), dict(k_tokens=257), dict(q_heads=3), dict(kv_heads=4), dict(head_dim=32), dict(flags=4), dict(scale=0.0),
                                 dict(scale=float("nan")), dict(q_len=0x1002), dict(k_len=0x1001), dict(table=0x1001), dict(table=FAKE, n_edges=2), dict(n_edges=65)])
def test_attention_refuses(lib, bad):
    assert lib.pruner_cache_attention(_attention(**bad), _cache(), _heads(), _heads(), None, None, 0, None) == EINVAL


def test_attention_refuses_pointers_and_workspaces(lib):
    a = _attention()
    for q, o, lse in ((None, _heads(), None), (_heads(), None, None), (_heads(0x1008), _heads(), None), (_heads(), _heads(0x1002), None), (_heads(token=12), _heads(), None), (_heads(), _heads(), 0x1002)):
        assert lib.pruner_cache_attention(a, _cache(), q, o, lse, None, 0, None) == EINVAL
    assert lib.pruner_cache_attention(None, _cache(), _heads(), _heads(), None, None, 0, None) == EINVAL
    assert lib.pruner_cache_attention(a, None, _heads(), _heads(), None, None, 0, None) == EINVAL
    long = _attention(k_tokens=1 << 16)
    room = _cache(seq_pages=1 << 10, pages=1 << 12)
    need = lib.pruner_cache_attention_workspace_bytes(long)
    assert need > 0
    for ws, size in ((None, need), (FAKE, need - 1), (FAKE + 16, need)):
        assert lib.pruner_cache_attention(long, room, _heads(), _heads(), None, ws, size, None) == EWORKSPACE
    assert lib.pruner_cache_attention(_attention(batch=0), _cache(), None, None, None, None, 0, None) == OK
    assert lib.pruner_cache_attention(_attention(q_tokens=0), _cache(), None, None, None, None, 0, None) == OK
    assert lib.pruner_cache_attention_workspace_bytes(_attention(head_dim=24)) == 0 and lib.pruner_cache_attention_workspace_bytes(None) == 0


def test_edges_that_do_not_ascend_are_refused(lib):
    for edges in ([3, 3], [0, 1], [2, 2000]):
        e = np.array(edges, np.int32)
        assert lib.pruner_cache_attention(_attention(table=FAKE, edges=e.ctypes.data, n_edges=2), _cache(), _heads(), _heads(), None, None, 0, None) == EINVAL


def _weights(**kw):
    d = dict(codes=FAKE, scales=FAKE, n_out=100, dim=200, group=32)
    d.update(kw)
    return C.byref(B.CWeights(*d.values()))


@pytest.mark.parametrize("bad", [dict(codes=0), dict(scales=0), dict(codes=0x1008), dict(scales=0x1004), dict(n_out=0), dict(dim=0), dict(n_out=(1 << 24) + 1), dict(dim=(1 << 24) + 1), dict(group=16),
                                 dict(group=48), dict(group=0)])
def test_weights_that_every_call_refuses(lib, bad):
    w = _weights(**bad)
    assert lib.pruner_weights_pack(FAKE, 0, 200, w, None) == EINVAL
    assert lib.pruner_weights_restore(w, 0, FAKE, 200, None) == EINVAL
    assert lib.pruner_weights_linear(w, FAKE, 0, 1, 200, None, FAKE, 100, None) == EINVAL


def test_weights_refuse(lib):
    w = _weights()
    for p, dtype, pitch in ((None, 0, 200), (0x1001, 0, 200), (0x1002, 2, 200), (FAKE, 3, 200), (FAKE, -1, 200), (FAKE, 0, 199)):
        assert lib.pruner_weights_pack(p, dtype, pitch, w, None) == EINVAL
        assert lib.pruner_weights_restore(w, dtype, p, pitch, None) == EINVAL
    assert lib.pruner_weights_pack(FAKE, 0, 1 << 24, _weights(n_out=1 << 24, dim=1 << 24), None) == EINVAL   # too many workgroups
    for x, dtype, rows, x_pitch, bias, y, y_pitch in ((None, 0, 1, 200, None, FAKE, 100), (FAKE, 0, 1, 200, None, None, 100), (0x1001, 0, 1, 200, None, FAKE, 100), (FAKE, 0, 1, 200, None, 0x1001, 100),
                                                      (FAKE, 2, 1, 200, None, FAKE, 100), (FAKE, 0, -1, 200, None, FAKE, 100), (FAKE, 0, (1 << 20) + 1, 200, None, FAKE, 100),
                                                      (FAKE, 0, 1, 199, None, FAKE, 100), (FAKE, 0, 1, 200, None, FAKE, 99), (FAKE, 0, 1, 200, 0x1002, FAKE, 100)):
        assert lib.pruner_weights_linear(w, x, dtype, rows, x_pitch, bias, y, y_pitch, None) == EINVAL
    assert lib.pruner_weights_linear(w, None, 0, 0, 200, None, None, 100, None) == OK


def test_every_call_is_exported(lib):
    for name in ("rotary", "rotary_grad", "cache_append", "cache_restore", "cache_attention", "cache_attention_workspace_bytes", "weights_pack", "weights_restore", "weights_linear"):
        assert hasattr(lib, "pruner_" + name)
