"""What pruner_gated_norm_grad refuses where the forward pass formed no y (no GPU)."""
from test_block_reference import EINVAL, EWORKSPACE, FAKE, _kept, _norm, lib  # noqa: F401  (lib is a fixture)


def test_gradients_without_a_norm_after(lib):
    names = ("p", "dh", "dhp", "dy", "dyp", "x", "xp", "f", "fp", "kept", "dx", "df", "dgate", "dw1", "dw2", "ws", "wsb", "st")
    bare = _norm(w_pre=None)
    need = lib.pruner_gated_norm_grad_workspace_bytes(4, 64)
    ok = dict(zip(names, (bare, FAKE, 64, None, 0, FAKE, 64, FAKE, 64, None, FAKE, FAKE, None, FAKE, None, FAKE, need - 1, None)))
    assert lib.pruner_gated_norm_grad(*ok.values()) == EWORKSPACE            # all else is in order
    for bad in (dict(dy=FAKE, dyp=64), dict(dw2=FAKE), dict(dh=None), dict(dh=FAKE + 1), dict(dhp=63), dict(p=_norm()), dict(x=None), dict(dw1=None), dict(kept=_kept()),
                dict(p=_norm(w_pre=None, gate=FAKE, pitch=64))):
        assert lib.pruner_gated_norm_grad(*{**ok, "wsb": need, **bad}.values()) == EINVAL, bad
