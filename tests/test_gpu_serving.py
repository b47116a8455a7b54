"""Serving calls where they meet the rest: attention over the rows of a partitioned circuit, the gates of a level written by number."""
import numpy as np
import pytest
import torch

import dg4_synth as synth
import kv8_ref as ref
import paper_2502_01681_amd as dg4
from gpu_utils import tdtype, to_np
from test_gpu_kv8 import cfg, reference, store
from test_gpu_lora import project, rows_of, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden,dtype,fmt", [(128, "f32", "int8"), (256, "bf16", "e4m3"), (128, "bf16", "e4m3"), (256, "f32", "int8")])
@pytest.mark.parametrize("k,stride,batch,marks,where", [(2, 1, 16, True, "host"), (3, 2, 7, True, "host"), (3, 2, 16, False, "host"), (8, 6, 32, True, "host"),
                                                        (8, 6, 32, True, "device"), (5, 3, 4, False, "host")])
def test_attention_on_a_partitioned_circuit(hidden, dtype, fmt, k, stride, batch, marks, where):
    """Rows of the updating strategy (Section 3.4): parts of cones; without marks a gate is there once for every mini-batch that holds it."""
    c = synth.Config("part", 9, 20, 400, 40, 0.9, 0, hidden, hidden // 32, k, 1, dtype)
    w = synth.make(c)
    if where == "host":
        g = dg4.dg4_build_partitioned(c.n_nodes, w.edge_src, w.edge_dst, w.edge_inv, k, stride, batch, marks=marks)
    else:
        g = dg4.dg4_build_partitioned_device(c.n_nodes, *(torch.from_numpy(a).cuda() for a in (w.edge_src, w.edge_dst, w.edge_inv)), k, stride, batch)
    assert (g.n == c.n_nodes) == marks
    print(f"kv8 attention on a partition k={k} stride={stride} B={batch} marks={marks} {where} {fmt} {hidden} {dtype}: {g.n} rows", flush=True)
    codes, scales = store(3, g.n, hidden, fmt)
    Q = rows_of(4, g.n, hidden, dtype)
    bias = torch.from_numpy(np.random.default_rng(5).standard_normal((hidden // 32, 4)).astype(np.float32)).cuda()
    bias[1, 3] = -np.inf
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, k), fmt, g, Q, codes, scales, bias, A)
    want, bound = reference(g, range(g.n), Q, codes, scales, fmt, bias, dtype)
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()
    ids = torch.from_numpy(np.random.default_rng(6).permutation(g.n)[:97].astype(np.int32)).cuda()
    B = torch.zeros((97, hidden), dtype=Q.dtype, device="cuda")
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, k), fmt, g, Q[ids.long()].contiguous(), codes, scales, bias, B, ids=ids)
    assert torch.equal(B, A[ids.long()])


@pytest.mark.parametrize("hidden,dtype,fmt", [(128, "f32", "int8"), (256, "bf16", "e4m3"), (256, "f32", "e4m3"), (128, "bf16", "int8")])
def test_the_gates_of_a_level_by_number(hidden, dtype, fmt):
    """Projected in any order and written by number into a store that holds something else: the rows that the whole batch gives."""
    n, heads = 325, hidden // 32
    rng = np.random.default_rng(9)
    packed = dg4.dg4_lora_pack(cfg(hidden, dtype), *weights(5, hidden, 3, 8, dtype))
    adapter = torch.from_numpy(rng.integers(-1, 3, n).astype(np.int32)).cuda()
    S = rows_of(6, n, hidden, dtype)
    _, K, V = project(cfg(hidden, dtype), packed, S, adapter)
    codes = torch.zeros((n, 2 * hidden), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n, heads, 2), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, K, V, codes, scales)
    for part, x in enumerate((K, V)):
        code, byte = ref.quantise(to_np(x), fmt)
        assert np.array_equal(ref.VALUES[fmt][codes[:, part * hidden:(part + 1) * hidden].cpu().numpy()], code)
        assert np.array_equal(scales[:, :, part].cpu().numpy(), byte)
    other, byte = torch.full_like(codes, 0x55), torch.full_like(scales, 0x66)
    for lo, hi in ((0, 40), (40, n)):
        ids = torch.from_numpy(rng.permutation(np.arange(lo, hi)).astype(np.int32)).cuda()
        at = ids.long()
        _, k, v = project(cfg(hidden, dtype), packed, S[at].contiguous(), adapter[at].contiguous())
        dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, k, v, other, byte, ids=ids)
        assert torch.equal(other[:hi], codes[:hi]) and torch.equal(byte[:hi], scales[:hi])
        assert (other[hi:] == 0x55).all() and (byte[hi:] == 0x66).all()
