"""What the calls in 4 bits turn away, before any device call (pointers here are never dereferenced), and the plain forms by hand."""
import ctypes
import os
import re

import numpy as np
import pytest

import fp4_ref as ref
import paper_2502_01681_amd as dg4

P = 1 << 20
FAR = 1 << 30
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -6, -8


def cfg(hidden=128, heads=None, dtype="f32", **kw):
    return dg4.LayerConfig(hidden, heads or hidden // 32, kw.pop("hops", 2), 1, dtype, **kw)


def write(c=None, K=P, V=P, lo=0, hi=4, ids=None, codes=P, scales=P, n=8):
    return dg4.lib().dg4_kv4_write(ctypes.byref((c or cfg()).c()), K, V, lo, hi, ids, codes, scales, n, None)


def read(c=None, K=P, V=P, lo=0, hi=4, ids=None, codes=P, scales=P, n=8):
    return dg4.lib().dg4_kv4_read(ctypes.byref((c or cfg()).c()), codes, scales, n, ids, lo, hi, K, V, None)


def test_library_exports_what_the_header_declares():
    hdr = open(os.path.join(os.path.dirname(__file__), "..", "include", "dg4_mx4.h")).read()
    names = set(re.findall(r"^(?:int|int64_t)\s+(dg4_[a-z0-9_]+)\s*\(", hdr, flags=re.M))
    assert names == {"dg4_kv4_write", "dg4_kv4_read", "dg4_sparse_attn_kv4_fwd", "dg4_mx4_packed_bytes", "dg4_mx4_pack", "dg4_qkv_proj_mx4",
                     "dg4_qkv_proj_kv4", "dg4_ffn_mx4_fwd"}
    for n in names:
        assert hasattr(dg4.lib(), n) and hasattr(dg4, n), n


@pytest.mark.parametrize("call", [write, read])
def test_store_calls(call):
    for bad in (dict(K=None), dict(V=None), dict(codes=None), dict(scales=None), dict(K=P + 8), dict(V=P + 2), dict(codes=P + 4),
                dict(scales=P + 1), dict(ids=P + 2), dict(lo=-1), dict(lo=3, hi=2), dict(hi=9), dict(n=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(c=cfg(64, 2)) == EUNSUPPORTED and call(c=cfg(128, 8)) == EUNSUPPORTED
    if call is read:                               # rows of 512 bytes, four of them
        assert call() == EINVAL and call(V=P + 2032) == EINVAL and call(K=P + 16) == EINVAL
    # nothing to do: fine, and nothing is looked at
    assert call(lo=2, hi=2) == 0 and call(lo=8, hi=8) == 0 and call(n=0, hi=0) == 0 and call(n=0, hi=5, ids=P) == 0


def test_attention():
    g = dg4.dg4_build_levels(5, [0, 1], [2, 2], [0, 1], 2)

    def call(c=cfg(dtype="bf16"), graph=g.handle, lo=0, hi=5, ids=None, Q=P, codes=P, scales=P, bias=P, A=P):
        return dg4.lib().dg4_sparse_attn_kv4_fwd(ctypes.byref(c.c()), graph, lo, hi, ids, Q, codes, scales, bias, A, None)
    for bad in (dict(graph=None), dict(Q=None), dict(codes=None), dict(scales=None), dict(bias=None), dict(A=None), dict(Q=P + 8),
                dict(A=P + 8), dict(codes=P + 8), dict(scales=P + 8), dict(bias=P + 2), dict(ids=P + 1), dict(lo=-1),
                dict(hi=6), dict(lo=3, hi=1), dict(c=cfg(dtype="bf16", hops=3))):
        assert call(**bad) == EINVAL, bad
    assert call(c=cfg(96, 3, "bf16")) == EUNSUPPORTED
    assert call(A=P + 256) == EINVAL and call(Q=P + 1264) == EINVAL           # (in place, or apart)
    assert call(lo=5, hi=5) == 0


def test_pack():
    size = lambda k, n, c=None: dg4.lib().dg4_mx4_packed_bytes(ctypes.byref((c or cfg()).c()), k, n)
    for k, n in ((128, 384), (128, 512), (512, 128)):
        assert k * n * 17 // 32 <= size(k, n) < k * n * 17 // 32 + n * 4 + 256 and size(k, n) % 256 == 0
    for k, n in ((128, 128), (384, 128), (256, 768), (0, 0), (-128, 384), (128, 383)):
        assert size(k, n) == EUNSUPPORTED
    assert size(64, 192, cfg(64, 2)) == EUNSUPPORTED and size(128, 384, cfg(ln_eps=-1.0)) == EINVAL

    def pack(c=None, W=P, k=128, n=384, packed=P, room=None):
        return dg4.lib().dg4_mx4_pack(ctypes.byref((c or cfg()).c()), W, k, n, packed, size(128, 384) if room is None else room, None)
    assert pack(W=None) == EINVAL and pack(W=P + 4) == EINVAL
    assert pack(packed=None) == EWORKSPACE and pack(packed=P + 128) == EWORKSPACE and pack(room=size(128, 384) - 1) == EWORKSPACE
    assert pack(n=256) == EUNSUPPORTED and pack(c=cfg(256)) == EUNSUPPORTED


def test_products():
    room = dg4.dg4_mx4_packed_bytes(cfg(), 128, 384)
    room1, room2 = dg4.dg4_mx4_packed_bytes(cfg(), 128, 512), dg4.dg4_mx4_packed_bytes(cfg(), 512, 128)
    L = dg4.lib()

    def proj(c=None, packed=FAR, size=room, S=P, lo=0, hi=4, Q=2 * P, K=3 * P, V=4 * P):
        return L.dg4_qkv_proj_mx4(ctypes.byref((c or cfg()).c()), packed, size, S, lo, hi, Q, K, V, None)

    def into(c=None, packed=FAR, size=room, S=P, lo=0, hi=4, ids=None, Q=2 * P, codes=3 * P, scales=4 * P, n=8):
        return L.dg4_qkv_proj_kv4(ctypes.byref((c or cfg()).c()), packed, size, S, lo, hi, ids, Q, codes, scales, n, None)

    def ffn(c=None, w1=FAR, s1=room1, w2=FAR, s2=room2, S=P, lo=0, hi=4, Out=2 * P):
        return L.dg4_ffn_mx4_fwd(ctypes.byref((c or cfg()).c()), w1, s1, w2, s2, S, lo, hi, Out, None)
    for call, outs in ((proj, "QKV"), (into, "Q"), (ffn, ("Out",))):
        for bad in (dict(S=None), dict(S=P + 8), dict(lo=-1), dict(lo=3, hi=2), dict(c=cfg(ln_eps=float("nan")))):
            assert call(**bad) == EINVAL, bad
        for name in outs:                          # rows of 512 bytes, four of them
            for at in (None, 2 * P + 4, P, P + 2032, P - 2032):
                assert call(**{name: at}) == EINVAL, (name, at)
        assert call(c=cfg(64, 2)) == EUNSUPPORTED
        assert call(lo=7, hi=7) == 0
    for call in (proj, into):
        assert call(packed=None) == EWORKSPACE and call(packed=FAR + 64) == EWORKSPACE and call(size=room - 1) == EWORKSPACE
    assert ffn(w1=None) == EWORKSPACE and ffn(w2=FAR + 16) == EWORKSPACE and ffn(s1=room1 - 1) == EWORKSPACE and ffn(s2=room2 - 1) == EWORKSPACE
    assert proj(Q=3 * P) == EINVAL and proj(K=4 * P + 16) == EINVAL and proj(V=2 * P - 16) == EINVAL
    for bad in (dict(codes=None), dict(scales=None), dict(codes=P + 4), dict(scales=P + 1), dict(ids=P + 2), dict(hi=9), dict(n=-1)):
        assert into(**bad) == EINVAL, bad


def test_reference_quantiser():
    """The plain form that the device is held to, by hand."""
    x = np.zeros((1, 32))
    x[0, :8] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]        # ties go to 0, 1, 1, 2, 2, 4, 4: codes with a last bit of zero
    code, byte = ref.quantise(x)
    assert byte[0, 0] == 127 and list(code[0, :8]) == [7, 0, 2, 2, 4, 4, 6, 6]
    x[0, 0] = 7.0                                  # the largest magnitude at a scale of one
    code, byte = ref.quantise(x)
    assert byte[0, 0] == 127 and list(code[0, :2]) == [7, 0]
    x[0, 0] = 7.0001
    code, byte = ref.quantise(x)
    assert byte[0, 0] == 128 and list(code[0, :4]) == [6, 0, 1, 1]
    x[0, :3] = [-7.0, -0.25, -0.0]
    assert list(ref.quantise(x)[0][0, :3]) == [15, 8, 8]
    assert ref.quantise(np.zeros((1, 32)))[1][0, 0] == 0
    x[0, 1] = np.inf
    assert ref.quantise(x)[1][0, 0] == 255 and np.isnan(ref.rounded(x)).all()
    codes, scales = ref.store(np.ones((2, 128)), -np.full((2, 128), 3.0))
    assert codes.shape == (2, 128) and (codes[:, :64] == 0x66).all() and (codes[:, 64:] == 0xFF).all()        # 4 * 2^-2, -6 * 2^-1
    K, V = ref.values(codes, scales)
    assert (K == 1).all() and (V == -3).all()


def test_reference_quantiser_error():
    """What the header says of the error: a fifth of the value, or a fourteenth of the block's largest magnitude; a ninth over a block."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4000, 32)) * np.exp2(rng.uniform(-3, 3, (4000, 1)))
    err = np.abs(ref.rounded(x) - x)
    assert (err <= np.maximum(np.abs(x) / 5, np.abs(x).max(1, keepdims=True) / 14) * (1 + 1e-12)).all()
    assert 0.105 < np.linalg.norm(err) / np.linalg.norm(x) < 0.12


def test_binding_turns_away_what_is_not_on_the_device():
    import torch
    x, codes, scales = torch.zeros((3, 128)), torch.zeros((3, 128), dtype=torch.uint8), torch.zeros((3, 4, 2), dtype=torch.uint8)
    g = dg4.dg4_build_levels(3, [0, 1], [2, 2], [0, 1], 2)
    w = dg4.Mx4Weights(torch.zeros(1 << 16, dtype=torch.uint8), 128, 384, 128)
    for call in (lambda: dg4.dg4_kv4_write(cfg(), x, x, codes, scales), lambda: dg4.dg4_kv4_read(cfg(), codes, scales, x, x),
                 lambda: dg4.dg4_sparse_attn_kv4_fwd(cfg(), g, x, codes, scales, torch.zeros((4, 4)), x),
                 lambda: dg4.dg4_mx4_pack(cfg(), torch.zeros((128, 384))), lambda: dg4.dg4_qkv_proj_mx4(cfg(), w, x, x, x, x),
                 lambda: dg4.dg4_qkv_proj_kv4(cfg(), w, x, x, codes, scales), lambda: dg4.dg4_ffn_mx4_fwd(cfg(), w, w, x, x)):
        with pytest.raises(dg4.DG4Error):
            call()


def test_binding_turns_away_what_is_no_tensor_or_no_configuration():
    import torch
    x, codes, scales = torch.zeros((3, 128)), torch.zeros((3, 128), dtype=torch.uint8), torch.zeros((3, 4, 2), dtype=torch.uint8)
    for call in (lambda: dg4.dg4_kv4_write(cfg(), None, x, codes, scales), lambda: dg4.dg4_kv4_read(cfg(), np.zeros(3), scales, x, x),
                 lambda: dg4.dg4_kv4_write(cfg(dtype=1), x, x, codes, scales), lambda: dg4.dg4_kv4_write(cfg(dtype="f16"), x, x, codes, scales),
                 lambda: dg4.dg4_kv4_write(cfg(), torch.zeros(()), x, codes, scales), lambda: dg4.dg4_ffn_mx4_fwd(cfg(), None, None, "S", x)):
        with pytest.raises(dg4.DG4Error):
            call()
    for call in (lambda: dg4.dg4_kv4_write(None, x, x, codes, scales), lambda: dg4.dg4_kv4_write(cfg(), x, x, codes), lambda: dg4.dg4_kv4_write(cfg(), x, x, codes, scales, row=3)):
        with pytest.raises((AttributeError, TypeError)):
            call()


def test_two_threads_make_the_first_call_of_a_process():
    """In a process of its own: the binding's native part is loaded by whoever comes first, and both calls get their answer."""
    import subprocess
    import sys
    code = """
import threading
import torch
import paper_2502_01681_amd as dg4
cfg = dg4.LayerConfig(128, 4, 2, 1, "f32")
x, codes, scales = torch.zeros((3, 128)), torch.zeros((3, 128), dtype=torch.uint8), torch.zeros((3, 4, 2), dtype=torch.uint8)
got, go = [], threading.Barrier(4)
def run():
    go.wait()
    try:
        dg4.dg4_kv4_write(cfg, x, x, codes, scales)
    except dg4.DG4Error as e:
        got.append(e.name)
threads = [threading.Thread(target=run) for _ in range(4)]
[t.start() for t in threads]
[t.join() for t in threads]
assert got == ["EINVAL"] * 4, got
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.join(os.path.dirname(__file__), ".."), timeout=120)
