"""Attention over the 8-bit store where rows of Q or values of the store are at the end of their type's range."""
import numpy as np
import pytest
import torch

import kv8_ref as ref
import paper_2502_01681_amd as dg4
from gpu_utils import tdtype, to_np
from test_gpu_kv8 import HALF_STEP, cfg, circuit, reference, store

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "bf16"), (256, "f32"), (128, "bf16")])
@pytest.mark.parametrize("hops", [1, 3, 5, 8])
def test_a_head_without_sources_gives_zeros_whatever_q_holds(fmt, hidden, dtype, hops):
    """Head 0 leaves everything out, head 1 the gate itself (all that a primary input has). Rows of Q in turn: finite, with a
    NaN, an infinity, a negative infinity in every head."""
    n = 120
    print(f"kv8 Q that is not finite {fmt} {hidden} {dtype} hops={hops}", flush=True)
    g = circuit(n, 60, hops, seed=2)
    codes, scales = store(6, n, hidden, fmt)
    rng = np.random.default_rng(7)
    finite = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.zeros((hidden // 32, 4), device="cuda")
    bias[0] = -np.inf
    bias[1, 0] = -np.inf
    Q = finite.clone().view(n, -1, 32)
    for kind, x in ((1, "nan"), (2, "inf"), (3, "-inf")):
        Q[kind::4, :, 5 + kind] = float(x)
    Q = Q.view(n, hidden)
    A, B = torch.full_like(Q, 7.0), torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, finite, codes, scales, bias, A)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q, codes, scales, bias, B)
    assert torch.equal(A[::4], B[::4])             # (a row does not see its neighbours)
    single = torch.from_numpy(np.diff(g.array("nbr_ptr")) == 1).cuda()
    assert int(single[1::4].sum()) and int(single[2::4].sum()) and int(single[3::4].sum())
    assert (B[:, :32] == 0).all()
    assert (B[single][:, 32:64] == 0).all()
    # with a source left, a NaN in Q is a NaN in the head
    assert B[1::4, 64:].isnan().all() and B[1::4][~single[1::4]][:, 32:64].isnan().all()
    want, bound = reference(g, range(0, n, 4), finite[::4], codes, scales, fmt, bias, dtype)
    assert (np.abs(to_np(B[::4]) - want) <= bound).all()
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hops", [2, 5])
@pytest.mark.parametrize("small", [-118, -124, -127, -131])
def test_large_q_against_the_smallest_values(fmt, dtype, hops, small):
    """K of 2^small, at the end of a float's range, against Q of about its reciprocal: ordinary scores."""
    n, hidden = 90, 128
    print(f"kv8 large Q {fmt} {dtype} hops={hops} K about 2^{small}", flush=True)
    g = circuit(n, 30, hops, seed=4)
    codes, scales = store(6, n, hidden, fmt)
    rng = np.random.default_rng(11)
    K = torch.from_numpy((rng.standard_normal((n, hidden)) * 2.0 ** small).astype(np.float32)).cuda()
    V = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).cuda()
    dg4.dg4_kv8_write(cfg(hidden, "f32"), fmt, K, V, codes, scales)
    Q = torch.from_numpy(rng.standard_normal((n, hidden)) * 2.0 ** min(-small, 125)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((4, 4)).astype(np.float32)).cuda()
    want, bound = reference(g, range(n), Q, codes, scales, fmt, bias, dtype)
    # (what a product below 2^-126 may lose against a score: 32 times 2^-149, nothing)
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q, codes, scales, bias, A)
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "bf16")])
def test_a_store_row_named_twice_harms_no_other(fmt, hidden, dtype):
    """What it holds itself is of the two rows that name it, byte by byte; written again, it is right."""
    n, rows = 60, 50
    rng = np.random.default_rng(3)
    ids = rng.permutation(n)[:rows].astype(np.int32)
    ids[[7, 30, 41]] = ids[[8, 12, 49]]
    K, V = (torch.from_numpy(rng.standard_normal((rows, hidden)).astype(np.float32) * np.exp2(rng.integers(-9, 9, (rows, 1)))).to(tdtype(dtype)).cuda() for _ in range(2))

    def written(k, v, at):
        codes = torch.full((n, 2 * hidden), 0x55, dtype=torch.uint8, device="cuda")
        scales = torch.full((n, hidden // 32, 2), 0x66, dtype=torch.uint8, device="cuda")
        dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, k, v, codes, scales, ids=torch.from_numpy(at).cuda())
        return codes, scales
    both = written(K, V, ids)
    keep = np.ones(rows, dtype=bool)
    keep[[7, 30, 41]] = False
    last = written(K[torch.from_numpy(keep).cuda()].contiguous(), V[torch.from_numpy(keep).cuda()].contiguous(), ids[keep])
    twice = ids[[8, 12, 49]]
    keep[[7, 30, 41]], keep[[8, 12, 49]] = True, False
    first = written(K[torch.from_numpy(keep).cuda()].contiguous(), V[torch.from_numpy(keep).cuda()].contiguous(), ids[keep])
    others = torch.from_numpy(np.setdiff1d(np.arange(n), twice)).cuda()
    for x, y, z in zip(both, last, first):
        assert torch.equal(x[others], y[others])
        assert ((x == y) | (x == z)).all()
    again = torch.tensor([8, 12, 49], device="cuda")
    dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, K[again].contiguous(), V[again].contiguous(), *both, ids=torch.from_numpy(twice).cuda())
    assert all(torch.equal(x, y) for x, y in zip(both, last))
