"""What the calls on a K|V store in 8 bits turn away, before any device call (pointers here are never dereferenced)."""
import ctypes

import numpy as np
import pytest

import kv8_ref as ref
import paper_2502_01681_amd as dg4

P = 4096
EINVAL, EUNSUPPORTED = -1, -6


def write(cfg=None, fmt=0, K=P, V=P, lo=0, hi=4, ids=None, codes=P, scales=P, n=8):
    c = (cfg or dg4.LayerConfig(128, 4, 2, 1, "f32")).c()
    return dg4.lib().dg4_kv8_write(ctypes.byref(c), fmt, K, V, lo, hi, ids, codes, scales, n, None)


def read(cfg=None, fmt=0, K=P, V=P, lo=0, hi=4, ids=None, codes=P, scales=P, n=8):
    c = (cfg or dg4.LayerConfig(128, 4, 2, 1, "f32")).c()
    return dg4.lib().dg4_kv8_read(ctypes.byref(c), fmt, codes, scales, n, ids, lo, hi, K, V, None)


@pytest.mark.parametrize("call", [write, read])
def test_store_calls(call):
    for bad in (dict(K=None), dict(V=None), dict(codes=None), dict(scales=None), dict(K=P + 8), dict(V=P + 2), dict(codes=P + 4),
                dict(scales=P + 1), dict(ids=P + 2), dict(fmt=2), dict(fmt=-1), dict(lo=-1), dict(lo=3, hi=2), dict(hi=9), dict(n=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(cfg=dg4.LayerConfig(64, 2, 2, 1, "f32")) == EUNSUPPORTED
    assert call(cfg=dg4.LayerConfig(128, 8, 2, 1, "f32")) == EUNSUPPORTED
    if call is read:                               # rows of 512 bytes, four of them
        assert call() == EINVAL and call(V=P + 2032) == EINVAL and call(K=P + 16) == EINVAL
    # nothing to do: fine, and nothing is looked at
    assert call(lo=2, hi=2) == 0
    assert call(lo=8, hi=8) == 0
    assert call(n=0, hi=0) == 0
    assert call(n=0, hi=5, ids=P) == 0


def test_attention():
    g = dg4.dg4_build_levels(5, [0, 1], [2, 2], [0, 1], 2)
    cfg = dg4.LayerConfig(128, 4, 2, 1, "bf16")

    def call(cfg=cfg, fmt=0, graph=g.handle, lo=0, hi=5, ids=None, Q=P, codes=P, scales=P, bias=P, A=P):
        c = cfg.c()
        return dg4.lib().dg4_sparse_attn_kv8_fwd(ctypes.byref(c), fmt, graph, lo, hi, ids, Q, codes, scales, bias, A, None)
    for bad in (dict(graph=None), dict(Q=None), dict(codes=None), dict(scales=None), dict(bias=None), dict(A=None), dict(Q=P + 8),
                dict(A=P + 8), dict(codes=P + 8), dict(scales=P + 8), dict(bias=P + 2), dict(ids=P + 1), dict(fmt=7), dict(lo=-1),
                dict(hi=6), dict(lo=3, hi=1), dict(cfg=dg4.LayerConfig(128, 4, 3, 1, "bf16"))):
        assert call(**bad) == EINVAL, bad
    assert call(cfg=dg4.LayerConfig(96, 3, 2, 1, "bf16")) == EUNSUPPORTED
    assert call(A=P + 256) == EINVAL and call(Q=P + 1264) == EINVAL           # (in place, or apart)
    assert call(lo=5, hi=5) == 0


def test_reference_quantiser():
    """The plain form that the device is held to, by hand."""
    x = np.zeros((1, 32))
    x[0, :4] = [448.0, 1.0, 17.0, -18.0]           # e4m3 steps of 2 between 16 and 32: 17 is a tie (to 16), 18 a code
    y, byte = ref.quantise(x, "e4m3")
    assert byte[0, 0] == 127 and list(y[0, :4]) == [448.0, 1.0, 16.0, -18.0]
    x[0, 0] = 449.0
    y, byte = ref.quantise(x, "e4m3")
    assert byte[0, 0] == 128 and list(y[0, :4]) == [224.0, 0.5, 8.0, -9.0]     # 224.5: step 16
    x[0, :4] = [127.0, 2.5, 3.5, -0.5]
    y, byte = ref.quantise(x, "int8")
    assert byte[0, 0] == 127 and list(y[0, :4]) == [127.0, 2.0, 4.0, 0.0]
    x[0, 0] = 127.5
    y, byte = ref.quantise(x, "int8")
    assert byte[0, 0] == 128 and y[0, 0] == 64.0
    assert ref.quantise(np.zeros((1, 32)), "int8")[1][0, 0] == 0
    x[0, 1] = np.inf
    assert ref.quantise(x, "int8")[1][0, 0] == 255
    assert ref.VALUES["e4m3"][0x7E] == 448.0 and ref.VALUES["e4m3"][1] == 2.0 ** -9 and ref.VALUES["int8"][0x80] == -128


def test_binding_turns_away_what_is_not_on_the_device():
    import torch
    cfg = dg4.LayerConfig(128, 4, 2, 1, "f32")
    x, codes, scales = torch.zeros((3, 128)), torch.zeros((3, 256), dtype=torch.uint8), torch.zeros((3, 4, 2), dtype=torch.uint8)
    g = dg4.dg4_build_levels(3, [0, 1], [2, 2], [0, 1], 2)
    for call in (lambda: dg4.dg4_kv8_write(cfg, "e4m3", x, x, codes, scales), lambda: dg4.dg4_kv8_read(cfg, "e4m3", codes, scales, x, x),
                 lambda: dg4.dg4_sparse_attn_kv8_fwd(cfg, "e4m3", g, x, codes, scales, torch.zeros((4, 4)), x),
                 lambda: dg4.dg4_lora_pack(cfg, torch.zeros((128, 384)))):
        with pytest.raises(dg4.DG4Error):
            call()
