"""What the calls with low-rank adapters turn away, before any device call (pointers here are never dereferenced)."""
import ctypes
import os
import re

import paper_2502_01681_amd as dg4

P = 4096
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -6, -8
BIG = 1 << 40


def cfg(hidden=256, dtype="bf16", heads=None):
    return dg4.LayerConfig(hidden, hidden // 32 if heads is None else heads, 2, 1, dtype)


def pack(c=None, W=P, n=4, rank=8, down=P, up=P, gain=P, packed=P, size=BIG):
    c = (c or cfg()).c()
    return dg4.lib().dg4_lora_pack(ctypes.byref(c), W, n, rank, down, up, gain, packed, size, None)


def proj(c=None, packed=P, size=BIG, n=4, rank=8, S=P, lo=0, hi=0, adapter=P, Q=P, K=P, V=P):
    c = (c or cfg()).c()
    return dg4.lib().dg4_qkv_proj_lora(ctypes.byref(c), packed, size, n, rank, S, lo, hi, adapter, Q, K, V, None)


def test_library_exports_what_the_header_declares():
    hdr = open(os.path.join(os.path.dirname(__file__), "..", "include", "dg4_serving.h")).read()
    names = set(re.findall(r"^(?:int|int64_t)\s+(dg4_[a-z0-9_]+)\s*\(", hdr, flags=re.M))
    assert names == {"dg4_kv8_write", "dg4_kv8_read", "dg4_sparse_attn_kv8_fwd", "dg4_lora_packed_bytes", "dg4_lora_pack", "dg4_qkv_proj_lora"}
    for n in names:
        assert hasattr(dg4.lib(), n) and hasattr(dg4, n), n


def test_pack():
    for bad in (dict(W=None), dict(W=P + 8), dict(n=-1), dict(rank=0), dict(rank=-3), dict(down=None), dict(up=None), dict(down=P + 8),
                dict(up=P + 8), dict(gain=P + 2)):
        assert pack(**bad) == EINVAL, bad
    for bad in (dict(rank=65), dict(c=cfg(512)), dict(c=cfg(256, heads=4))):
        assert pack(**bad) == EUNSUPPORTED, bad
    need = dg4.dg4_lora_packed_bytes(cfg(), 4, 8)
    for bad in (dict(packed=None), dict(packed=P + 16), dict(size=need - 1), dict(size=0)):
        assert pack(**bad) == EWORKSPACE, bad


def test_proj():
    for bad in (dict(S=None), dict(Q=None), dict(K=None), dict(V=None), dict(S=P + 8), dict(Q=P + 4), dict(K=P + 8), dict(V=P + 8),
                dict(adapter=P + 2), dict(lo=-1), dict(lo=3, hi=2), dict(n=-1), dict(rank=0)):
        assert proj(**bad) == EINVAL, bad
    assert proj(rank=65) == EUNSUPPORTED
    need = dg4.dg4_lora_packed_bytes(cfg(), 4, 8)
    for bad in (dict(packed=None), dict(packed=P + 128), dict(size=need - 1)):
        assert proj(**bad) == EWORKSPACE, bad
    assert proj() == 0 and proj(adapter=None) == 0 and proj(lo=7, hi=7) == 0
    apart = dict(S=P, Q=2 * P, K=3 * P, V=4 * P)   # rows of 512 bytes
    for bad in (dict(Q=P), dict(K=P + 4080), dict(V=2 * P + 16), dict(K=4 * P - 4080), dict(S=4 * P), dict(Q=3 * P + 512)):
        assert proj(**{**apart, **bad}, hi=8) == EINVAL and proj(**{**apart, **bad}, lo=6, hi=14) == EINVAL, bad
    # no adapters: the rank is not looked at
    assert proj(n=0, rank=0, adapter=None) == 0 and proj(n=0, rank=900) == 0


def test_packed_bytes():
    for hidden in (128, 256):
        for dtype, es in (("f32", 4), ("bf16", 2)):
            for n, rank in ((1, 1), (3, 8), (64, 27), (1000, 64)):
                r8 = (rank + 7) // 8 * 8
                want = 3 * hidden * hidden * es + n * hidden * (rank + 3 * r8) * es + (4 * n + 255) // 256 * 256
                assert dg4.dg4_lora_packed_bytes(cfg(hidden, dtype), n, rank) == want
            assert dg4.dg4_lora_packed_bytes(cfg(hidden, dtype), 0, 0) == 3 * hidden * hidden * es
    for n, rank, status in ((-1, 8, "EINVAL"), (2, 0, "EINVAL"), (2, 65, "EUNSUPPORTED")):
        try:
            dg4.dg4_lora_packed_bytes(cfg(), n, rank)
            assert False
        except dg4.DG4Error as e:
            assert e.name == status
    # far more adapters than 32 bits of bytes hold
    assert dg4.dg4_lora_packed_bytes(cfg(), 100_000, 64) > 1 << 33
