"""The structs of the block's operators as the binding packs them lie as the C structs do (no GPU)."""
import paper_2402_02361_amd.binding as B


def test_packed_structs_are_the_structs():
    assert B._PACK_CHECKPOINT.pack(0x1234, 0x5678) == bytes(B.CCheckpoint(0x1234, 0x5678))
    assert B._PACK_HEADS.pack(0x1234, 5, 6, -7) == bytes(B.CHeads(0x1234, 5, 6, -7))
    norm = (1 << 33, 2, 1, 1, 0.5, 0.25, 0x10, 0x20, 0x30, 1 << 34)
    assert B._PACK_NORM.pack(*norm) == bytes(B.CNorm(*norm))
    attention = (1, 2, 3, 4, 5, 6, 7, 3, 0.125, 0x10, 0x20, 0x30, 0x40, 9)
    assert B._PACK_ATTENTION.pack(*attention) == bytes(B.CAttention(*attention))
