"""The calls in 4 bits at the ends of their ranges: calls of several launches, keys, rows and weights at the smallest scales, subnormal
queries, magnitudes that the type's largest number is below."""
import ctypes
import re

import numpy as np
import pytest
import torch

import fp4_ref as ref
import kv8_ref
import paper_2502_01681_amd as dg4
from fp4_ref import HALF_STEP
from gpu_utils import tdtype, to_np

pytestmark = pytest.mark.gpu

SHAPES = [(128, "f32"), (256, "bf16"), (256, "f32"), (128, "bf16")]


def cfg(hidden, dtype, hops=2, **kw):
    return dg4.LayerConfig(hidden, hidden // 32, hops, 1, dtype, **kw)


def table(rng, shape, size, dtype):
    """Normal numbers times size, rounded to the type, on the host."""
    return torch.from_numpy((rng.standard_normal(shape).clip(-3.5, 3.5) * size).astype(np.float32)).to(tdtype(dtype))


def close(got, want, bound):
    err = np.abs(got - want)
    assert (err <= bound).all(), (err / bound).max()


def launches(call):
    """How many kernels a call launches: what a capture of it holds (nothing is run)."""
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    path = re.search(r"\S*libamdhip64\.so\S*", open("/proc/self/maps").read()).group(0)
    nodes = ctypes.c_size_t(0)
    assert ctypes.CDLL(path).hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(nodes)) == 0
    return nodes.value


def around(limit, rows):
    return torch.tensor([0, 3, limit - 2, limit - 1, limit, limit + 1, limit + 3, rows - 1], device="cuda")


def test_attention_in_several_launches():
    """Rows of eight hops at hidden 128, four of them to a workgroup: 2^25 to a launch."""
    hidden, n, limit = 128, 400, 2 ** 25
    rows = limit + 5
    c = cfg(hidden, "bf16", 8)
    print(f"kv4 attention over {rows} rows, nearly all padding", flush=True)
    rng = np.random.default_rng(1)
    fan = [(u, v, int(rng.integers(0, 2))) for v in range(30, n) for u in rng.choice(np.arange(max(0, v - 40), v), 2, replace=False)]
    g = dg4.dg4_build_levels(n, *(np.array(x) for x in zip(*fan)), 8)
    g.upload()
    codes = torch.zeros((n, hidden), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n, hidden // 32, 2), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv4_write(c, *(table(rng, (n, hidden), 1.0, "bf16").cuda() for _ in range(2)), codes, scales)
    bias = torch.zeros((hidden // 32, 4), device="cuda")
    gates = torch.tensor([5, 399, 0, 17, 398, 5, 100, 250], dtype=torch.int32, device="cuda")
    few, want = table(rng, (8, hidden), 1.0, "bf16").cuda(), torch.empty((8, hidden), dtype=torch.bfloat16, device="cuda")
    dg4.dg4_sparse_attn_kv4_fwd(c, g, few, codes, scales, bias, want, ids=gates)
    at = around(limit, rows)
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    Q = torch.full((rows, hidden), 7.0, dtype=torch.bfloat16, device="cuda")
    ids[at], Q[at] = gates, few
    A = torch.full_like(Q, 7.0)
    call = lambda end: dg4.dg4_sparse_attn_kv4_fwd(c, g, Q, codes, scales, bias, A, ids=ids, row_end=end)
    assert launches(lambda: call(limit)) == 1 and launches(lambda: call(limit + 1)) == 2
    call(rows)
    assert torch.equal(A[at], want)
    A[at] = 7.0
    assert torch.equal(A, A[1:2].expand_as(A))
    # from a row that is not the first, in place
    Q[at], A = few, None
    dg4.dg4_sparse_attn_kv4_fwd(c, g, Q, codes, scales, bias, Q, ids=ids, row_begin=1)
    assert torch.equal(Q[at[1:]], want[1:]) and torch.equal(Q[0], few[0])


def test_write_and_read_in_several_launches():
    """Rows of float at hidden 256, four of them to a workgroup: 2^25 to a launch."""
    hidden, n, limit = 256, 64, 2 ** 25
    rows = limit + 5
    c = cfg(hidden, "f32")
    print(f"kv4 write and read of {rows} rows, nearly all padding", flush=True)
    at, gates = around(limit, rows), torch.tensor([5, 63, 0, 17, 31, 6, 40, 25], dtype=torch.int32, device="cuda")
    few = table(np.random.default_rng(2), (8, hidden), 1.0, "f32")
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    K = torch.full((rows, hidden), 7.0, device="cuda")
    ids[at], K[at] = gates, few.cuda()
    codes = torch.full((n, hidden), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, hidden // 32, 2), 0x66, dtype=torch.uint8, device="cuda")
    write = lambda end: dg4.dg4_kv4_write(c, K, K, codes, scales, ids=ids, row_end=end)
    assert launches(lambda: write(limit)) == 1 and launches(lambda: write(limit + 1)) == 2
    write(rows)
    code, byte = ref.store(to_np(few), to_np(few))
    named = gates.cpu().numpy()
    others = np.setdiff1d(np.arange(n), named)
    got, at_scale = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(got[named], code) and np.array_equal(at_scale[named], byte)
    assert (got[others] == 0x55).all() and (at_scale[others] == 0x66).all()
    K.fill_(7.0)
    V = torch.full_like(K, 7.0)
    read = lambda end: dg4.dg4_kv4_read(c, codes, scales, K, V, ids=ids, row_end=end)
    assert launches(lambda: read(limit)) == 1 and launches(lambda: read(limit + 1)) == 2
    read(rows)
    for x, want in zip((K, V), ref.values(code, byte)):
        assert torch.equal(x[at].cpu(), torch.from_numpy(want).float())
        x[at] = 7.0
        assert torch.equal(x, x[1:2].expand_as(x))


def circuit(n, hops):
    rng = np.random.default_rng(4)
    fan = [(u, v, int(rng.integers(0, 2))) for v in range(8, n) for u in rng.choice(np.arange(max(0, v - 30), v), 2, replace=False)]
    return dg4.dg4_build_levels(n, *(np.array(x) for x in zip(*fan)), hops)


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("hops", [2, 5])
@pytest.mark.parametrize("byte", [0, 252])
def test_scores_of_the_smallest_and_the_largest_keys(hidden, dtype, hops, byte):
    """Keys under the scale 2^-127 (subnormal in float) against Q about 2^125; keys under 2^125 against Q of normal numbers about 2^-125,
    of these and one subnormal number to a head, and of subnormal numbers and zeros alone: ordinary scores, to which all of them count."""
    n = 90
    print(f"kv4 keys under 2^{byte - 127} {hidden} {dtype} hops={hops}", flush=True)
    g = circuit(n, hops)
    rng = np.random.default_rng(5)
    codes = rng.integers(0, 256, (n, hidden)).astype(np.uint8)
    scales = np.full((n, hidden // 32, 2), 126, dtype=np.uint8)
    scales[:, :, 0] = byte
    K, V = ref.values(codes, scales)
    assert (K != 0).mean() > 0.8
    if byte == 0:
        q = rng.standard_normal((n, hidden)).clip(-3.5, 3.5) * 2.0 ** 125
    else:
        sign = np.where(rng.random((n, hidden)) < 0.5, 1.0, -1.0)
        q = sign * (1 + rng.random((n, hidden))) * 2.0 ** -125
        q[1::3, 9::32] = 3 * 2.0 ** -128
        q[2::3] = sign[2::3] * rng.integers(0, 8, q[2::3].shape) * 2.0 ** -129
    Q = torch.from_numpy(q).to(torch.float32).to(tdtype(dtype))
    assert (Q != 0).float().mean() > 0.8
    bias = rng.standard_normal((hidden // 32, 4)).astype(np.float32)
    want, bound = kv8_ref.attention(g.array("nbr_ptr"), g.array("nbr_idx"), g.array("nbr_rel"), range(n), to_np(Q), K, V, bias, HALF_STEP[dtype])
    A = torch.zeros((n, hidden), dtype=tdtype(dtype), device="cuda")
    dev = lambda x: torch.from_numpy(x).cuda()
    dg4.dg4_sparse_attn_kv4_fwd(cfg(hidden, dtype, hops), g, Q.cuda(), dev(codes), dev(scales), dev(bias), A)
    close(to_np(A), want, bound)


def lowest(x, axis):
    """Whether all blocks of x along an axis are under 2^-127, and most of their codes are no zero."""
    code, byte = ref.quantise(np.moveaxis(to_np(x).astype(np.float64), axis, -1))
    return (byte == 0).all() and (code & 7 != 0).mean() > 0.6


# Sizes of rows and weights: one of them is under the scale 2^-127 whole, the other brings the products back
LOW = 2.0 ** -127


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("which", ["rows", "weights"])
def test_projection_at_the_lowest_scales(hidden, dtype, which):
    rows, d = 70, hidden
    print(f"mx4 projection, {which} under 2^-127 {hidden} {dtype}", flush=True)
    rng = np.random.default_rng(6)
    S = table(rng, (rows, d), LOW if which == "rows" else 2.0 ** 100, dtype)
    W = table(rng, (d, 3 * d), LOW if which == "weights" else 2.0 ** 100, dtype)
    assert lowest(S, 1) if which == "rows" else lowest(W, 0)
    assert ref.exact_sums(to_np(S), to_np(W))
    c = cfg(d, dtype)
    packed, x = dg4.dg4_mx4_pack(c, W.cuda()), S.cuda()
    out = [torch.zeros_like(x) for _ in range(3)]
    dg4.dg4_qkv_proj_mx4(c, packed, x, *out)
    y, bound = ref.proj(to_np(S), to_np(W), HALF_STEP[dtype])
    close(np.concatenate([to_np(t) for t in out], 1), y, bound)
    codes, scales = torch.zeros((rows, d), dtype=torch.uint8, device="cuda"), torch.zeros((rows, d // 32, 2), dtype=torch.uint8, device="cuda")
    Q = torch.zeros_like(x)
    dg4.dg4_qkv_proj_kv4(c, packed, x, Q, codes, scales)
    code, byte = ref.store(y[:, d:2 * d], y[:, 2 * d:])
    assert torch.equal(Q, out[0]) and np.array_equal(scales.cpu().numpy(), byte)
    assert all(np.array_equal(a, b) for a, b in zip(ref.values(codes.cpu().numpy(), byte), ref.values(code, byte)))


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("which,sizes", [("rows", (LOW, 2.0 ** 100, 1.0)), ("first weights", (2.0 ** 50, LOW, 2.0 ** 118)), ("second weights", (1.0, 2.0 ** 118, LOW))])
def test_feed_forward_at_the_lowest_scales(hidden, dtype, which, sizes):
    """Sums in which the product counts at least as much as a tenth of the row does, and a row's variance without an epsilon."""
    rows, d = 50, hidden
    print(f"mx4 feed-forward, {which} under 2^-127 {hidden} {dtype}", flush=True)
    rng = np.random.default_rng(7)
    S, W1, W2 = (table(rng, shape, size, dtype) for shape, size in zip(((rows, d), (d, 4 * d), (4 * d, d)), sizes))
    assert lowest(S, 1) if which == "rows" else lowest(W1 if which == "first weights" else W2, 0)
    h = np.maximum(ref.rounded(to_np(S)) @ ref.across(to_np(W1)), 0)
    assert ref.exact_sums(to_np(S), to_np(W1)) and ref.exact_sums(h, to_np(W2))
    assert np.linalg.norm(ref.rounded(h) @ ref.across(to_np(W2))) > 0.1 * np.linalg.norm(to_np(S).astype(np.float64))
    c = cfg(d, dtype, ln_eps=0.0)
    x = S.cuda()
    out = torch.zeros_like(x)
    dg4.dg4_ffn_mx4_fwd(c, dg4.dg4_mx4_pack(c, W1.cuda()), dg4.dg4_mx4_pack(c, W2.cuda()), x, out)
    close(to_np(out), *ref.ffn(to_np(S), to_np(W1), to_np(W2), 0.0, HALF_STEP[dtype]))


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_magnitudes_that_the_type_does_not_reach(hidden, dtype):
    """From 1.75 * 2^127 on a block's largest magnitudes go to 4 * 2^126, which float and bfloat16 read as an infinity; up to there to
    6 * 2^125. The rest of the block reads as it is."""
    x = torch.zeros((2, hidden))
    x[0, 0], x[1, 0] = torch.finfo(tdtype(dtype)).max, 1.75 * 2.0 ** 127
    x[:, 1], x[:, 40] = -2.0 ** 126, 3.0
    x = x.to(tdtype(dtype)).cuda()
    codes, scales = torch.zeros((2, hidden), dtype=torch.uint8, device="cuda"), torch.zeros((2, hidden // 32, 2), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv4_write(cfg(hidden, dtype), x, -x, codes, scales)
    K, V = torch.ones_like(x), torch.ones_like(x)
    dg4.dg4_kv4_read(cfg(hidden, dtype), codes, scales, K, V)
    assert scales[:, 0, 0].tolist() == [253, 252] and torch.equal(K, -V)
    assert K[0, 0] == np.inf and K[1, 0].float() == 1.5 * 2.0 ** 127
    assert torch.equal(K[:, 1:], x[:, 1:])
