"""The K|V store in 4 bits: written, read back and attended over, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import fp4_ref as ref
import kv8_ref
import paper_2502_01681_amd as dg4
from fp4_ref import HALF_STEP
from gpu_utils import tdtype, to_np
from test_gpu_kv8 import cfg, circuit

pytestmark = pytest.mark.gpu

SHAPES = [(128, "f32"), (256, "bf16"), (256, "f32"), (128, "bf16")]


def rows_of(seed, rows, hidden, dtype):
    """Rows with every kind of block: ordinary, tiny, huge, zero, one value only, largest magnitudes at and beside 6 and 7 codes,
    values half way between codes."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, hidden // 32, 32)) * np.exp2(rng.integers(-6, 7, (rows, hidden // 32, 1)))
    kind = rng.integers(0, 12, (rows, hidden // 32))
    x[kind == 0] = 0.0
    x[kind == 1] *= 2.0 ** -130                    # around the smallest normal numbers
    x[kind == 2] *= 2.0 ** 110
    x[kind == 3, 1:] = 0.0
    top = np.array([6.0, 6.5, 7.0, 7.03125, 8.0, 3.5, 3.515625, 12.0])
    at = np.nonzero(kind == 4)
    x[at[0], at[1]] = np.rint(x[at[0], at[1]] * 4) / 8
    x[at[0], at[1], 5] = top[rng.integers(0, len(top), len(at[0]))]
    at = np.nonzero(kind == 5)                     # ties
    x[at[0], at[1]] = (np.rint(rng.standard_normal((len(at[0]), 32)) * 6) + 0.5) * 0.5
    x[at[0], at[1], 7] = 7.0
    x[kind == 6] *= -1e-3
    return torch.from_numpy(x.reshape(rows, hidden).astype(np.float32)).to(tdtype(dtype)).cuda()


def blank(n, hidden):
    return (torch.full((n, hidden), 0x55, dtype=torch.uint8, device="cuda"), torch.full((n, hidden // 32, 2), 0x66, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("hidden", [128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 3, 17, 260])
def test_write_and_read_every_row(hidden, dtype, rows):
    print(f"kv4 {hidden} {dtype} rows={rows}", flush=True)
    K, V = rows_of(rows, rows, hidden, dtype), rows_of(rows + 1, rows, hidden, dtype)
    codes, scales = blank(rows + 2, hidden)
    dg4.dg4_kv4_write(cfg(hidden, dtype), K, V, codes, scales)
    want, byte = ref.store(to_np(K), to_np(V))
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    assert (c[rows:] == 0x55).all() and (s[rows:] == 0x66).all()
    assert np.array_equal(s[:rows], byte) and np.array_equal(c[:rows], want)
    K2, V2 = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    dg4.dg4_kv4_read(cfg(hidden, dtype), codes, scales, K2, V2)
    for got, want in zip((K2, V2), ref.values(c[:rows], s[:rows])):
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(tdtype(dtype)))
    # within the format's error of what was written; scales end at 2^-127, where half a step is 2^-129
    for got, x in zip((K2, V2), (K, V)):
        x, got = to_np(x).astype(np.float64).reshape(rows, -1, 32), to_np(got).astype(np.float64).reshape(rows, -1, 32)
        bound = np.maximum(np.abs(x) / 5, np.abs(x).max(axis=2, keepdims=True) / 14)
        assert (np.abs(got - x) - bound * (1 + 1e-12)).max() <= 2.0 ** -129


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_every_code_reads_as_its_number(hidden, dtype):
    """All 256 bytes under all 256 scales (a scale of 255 is NaN whatever the codes)."""
    n = 256
    rng = np.random.default_rng(0)
    codes = np.stack([np.roll(np.tile(np.arange(256, dtype=np.uint8), hidden // 128), i)[:hidden] for i in range(n)])
    scales = np.repeat(np.arange(n, dtype=np.uint8), hidden // 32 * 2).reshape(n, hidden // 32, 2)
    scales = scales + rng.integers(0, 2, scales.shape).astype(np.uint8)
    K, V = (torch.zeros((n, hidden), dtype=tdtype(dtype), device="cuda") for _ in range(2))
    dg4.dg4_kv4_read(cfg(hidden, dtype), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K, V)
    for got, want in zip((K, V), ref.values(codes, scales)):
        want = torch.from_numpy(want).to(tdtype(dtype))
        assert torch.equal(got.cpu().isnan(), want.isnan()) and torch.equal(got.cpu().nan_to_num(0.0, 1e38, -1e38), want.nan_to_num(0.0, 1e38, -1e38))


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_listed_rows(hidden, dtype):
    print(f"kv4 listed {hidden} {dtype}", flush=True)
    n, rows = 300, 77
    rng = np.random.default_rng(5)
    ids = rng.permutation(n)[:rows].astype(np.int32)
    ids[[0, 13, 40, 76]] = [-1, n, 2 ** 31 - 1, -2 ** 31]          # no row of the store
    named = (ids >= 0) & (ids < n)
    K, V = rows_of(1, rows, hidden, dtype), rows_of(2, rows, hidden, dtype)
    codes, scales = blank(n, hidden)
    lo, hi = 3, 75
    dg4.dg4_kv4_write(cfg(hidden, dtype), K, V, codes, scales, ids=torch.from_numpy(ids).cuda(), row_begin=lo, row_end=hi)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    used = np.nonzero(named & (np.arange(rows) >= lo) & (np.arange(rows) < hi))[0]
    others = np.setdiff1d(np.arange(n), ids[used])
    assert (c[others] == 0x55).all() and (s[others] == 0x66).all()
    want, byte = ref.store(to_np(K)[used], to_np(V)[used])
    assert np.array_equal(c[ids[used]], want) and np.array_equal(s[ids[used]], byte)
    # read back in another order, rows twice, rows that are none
    back = np.concatenate([ids[used][::-1], ids[used][:5], [-1, n, -2 ** 31]]).astype(np.int32)
    out = [torch.full((len(back), hidden), 7.0, dtype=tdtype(dtype), device="cuda") for _ in range(2)]
    dg4.dg4_kv4_read(cfg(hidden, dtype), codes, scales, *out, ids=torch.from_numpy(back).cuda())
    for got, want in zip(out, ref.values(c, s)):
        assert torch.equal(got[:-3].cpu(), torch.from_numpy(want[back[:-3]]).to(tdtype(dtype))) and (got[-3:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_that_are_not_finite_read_as_nan(dtype):
    x = torch.ones((5, 128), device="cuda")
    x[0, 3], x[1, 40], x[2, 127], x[4, 64] = float("nan"), float("inf"), float("-inf"), -float("nan")
    x[3, 0] = torch.finfo(torch.bfloat16).max
    x = x.to(tdtype(dtype))
    codes, scales = blank(5, 128)
    dg4.dg4_kv4_write(cfg(128, dtype), x, torch.ones_like(x), codes, scales)
    want, byte = ref.store(to_np(x), np.ones((5, 128)))
    assert np.array_equal(codes.cpu().numpy(), want) and np.array_equal(scales.cpu().numpy(), byte)
    K, V = torch.zeros_like(x), torch.zeros_like(x)
    dg4.dg4_kv4_read(cfg(128, dtype), codes, scales, K, V)
    bad = torch.zeros((5, 4), dtype=torch.bool)
    bad[0, 0] = bad[1, 1] = bad[2, 3] = bad[4, 2] = True
    assert torch.equal(K.view(5, 4, 32).isnan().all(2).cpu(), bad) and torch.equal(K.view(5, 4, 32).isnan().any(2).cpu(), bad)
    assert (V == 1).all() and (K[3, 32:] == 1).all()


def store(seed, n, hidden):
    rng = np.random.default_rng(seed)
    codes, scales = blank(n, hidden)
    kv = [torch.from_numpy((rng.standard_normal((n, hidden)) * np.exp2(rng.integers(-2, 2, (n, 1)))).astype(np.float32)).cuda() for _ in range(2)]
    dg4.dg4_kv4_write(cfg(hidden, "f32"), *kv, codes, scales)
    return codes, scales


def reference(g, gates, Q, codes, scales, bias, dtype):
    """(A, bound): the bound of kv8_ref.attention."""
    K, V = ref.values(codes.cpu().numpy(), scales.cpu().numpy())
    return kv8_ref.attention(g.array("nbr_ptr"), g.array("nbr_idx"), g.array("nbr_rel"), gates, to_np(Q), K, V, bias.cpu().numpy(), HALF_STEP[dtype])


def attend(c, g, Q, codes, scales, bias, **kw):
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv4_fwd(c, g, Q, codes, scales, bias, A, **kw)
    return A


def close(A, want, bound):
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("hidden", [128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,hops", [(230, 1), (230, 2), (230, 3), (150, 4), (200, 5), (260, 6), (300, 7), (330, 8)])
def test_attention(hidden, dtype, n, hops):
    g = circuit(n, 24 if hops < 6 else 330, hops)
    print(f"kv4 attention {hidden} {dtype} n={n} hops={hops} longest row {int(np.diff(g.array('nbr_ptr')).max())}", flush=True)
    codes, scales = store(3, n, hidden)
    rng = np.random.default_rng(4)
    Q = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((hidden // 32, 4)).astype(np.float32)).cuda()
    c = cfg(hidden, dtype, hops)
    A = attend(c, g, Q, codes, scales, bias)
    close(A, *reference(g, range(n), Q, codes, scales, bias, dtype))
    # a gate alone in its row copies its values exactly
    single = np.nonzero(np.diff(g.array("nbr_ptr")) == 1)[0]
    V = ref.values(codes.cpu().numpy(), scales.cpu().numpy())[1]
    assert len(single) and torch.equal(A[single].cpu(), torch.from_numpy(V[single]).to(tdtype(dtype)))
    # the same bits for parts of the rows, for listed gates and in place; other rows stay
    for lo, hi in ((0, 1), (5, 6), (n - 1, n), (3, n - 7), (9, 9)):
        B = attend(c, g, Q, codes, scales, bias, row_begin=lo, row_end=hi)
        assert torch.equal(B[lo:hi], A[lo:hi]) and (B[:lo] == 7.0).all() and (B[hi:] == 7.0).all()
    ids = rng.permutation(n)[:61].astype(np.int32)
    ids[[0, 9, 60]] = [-1, n, 2 ** 31 - 1]
    ids[20] = ids[21]
    ok = torch.from_numpy((ids >= 0) & (ids < n)).cuda()
    pick = torch.from_numpy(np.where((ids >= 0) & (ids < n), ids, 0).astype(np.int64)).cuda()
    B = attend(c, g, Q[pick].contiguous(), codes, scales, bias, ids=torch.from_numpy(ids).cuda())
    assert torch.equal(B[ok], A[pick][ok]) and (B[~ok] == 7.0).all()
    dg4.dg4_sparse_attn_kv4_fwd(c, g, Q, codes, scales, bias, Q)
    assert torch.equal(Q, A)


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("hops", [1, 3, 5, 8])
def test_relations_left_out(hidden, dtype, hops):
    """Heads: 0 without any relation, 1 without the gate itself, 2 without what lies further up, 3 with the type's lowest value. Rows of
    Q in turn: finite, with a NaN, an infinity, a negative infinity in every head."""
    n = 120
    print(f"kv4 relations left out {hidden} {dtype} hops={hops}", flush=True)
    g = circuit(n, 60, hops, seed=2)
    codes, scales = store(6, n, hidden)
    rng = np.random.default_rng(7)
    finite = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((hidden // 32, 4)).astype(np.float32))
    bias[0] = bias[1, 0] = bias[2, 3] = -np.inf
    bias[3] = torch.finfo(torch.float32).min
    bias = bias.cuda()
    want, bound = reference(g, range(n), finite, codes, scales, bias, dtype)
    # the lowest value swallows the score: every source counts the same there
    ptr, V = g.array("nbr_ptr"), ref.values(codes.cpu().numpy(), scales.cpu().numpy())[1]
    for v in range(n):
        src = g.array("nbr_idx")[ptr[v]:ptr[v + 1]]
        want[v, 96:128] = V[src, 96:128].mean(axis=0)
        bound[v, 96:128] = (2 * len(src) + 4) * 2.0 ** -24 * np.abs(V[src, 96:128]).mean(axis=0) + HALF_STEP[dtype] * np.abs(want[v, 96:128]) + 1e-37
    A = attend(cfg(hidden, dtype, hops), g, finite, codes, scales, bias)
    close(A, want, bound)
    Q = finite.clone().view(n, -1, 32)
    for kind, x in ((1, "nan"), (2, "inf"), (3, "-inf")):
        Q[kind::4, :, 5 + kind] = float(x)
    B = attend(cfg(hidden, dtype, hops), g, Q.view(n, hidden), codes, scales, bias)
    close(B[::4], want[::4], bound[::4])           # (a row does not see its neighbours)
    single = torch.from_numpy(np.diff(ptr) == 1).cuda()
    assert int(single[1::4].sum()) and int(single[2::4].sum()) and int(single[3::4].sum())
    assert (B[:, :32] == 0).all() and (B[single][:, 32:64] == 0).all()
    # with a source left, a NaN in Q is a NaN in the head
    assert B[1::4, 64:].isnan().all() and B[1::4][~single[1::4]][:, 32:64].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hops", [2, 5])
def test_any_scale_and_code(dtype, hops):
    """Stores as a caller may fill them: every code, scales from the smallest on."""
    n, hidden = 90, 128
    g = circuit(n, 30, hops, seed=4)
    rng = np.random.default_rng(8)
    codes = rng.integers(0, 256, (n, hidden)).astype(np.uint8)
    scales = rng.integers(110, 126, (n, 4, 2))
    scales[rng.random(scales.shape) < 0.2] = 0
    scales[rng.random(scales.shape) < 0.1] = 1
    scales[:, :, 1] += rng.integers(0, 3, (n, 4)) * 30         # (values far apart in size)
    codes, scales = torch.from_numpy(codes).cuda(), torch.from_numpy(scales.astype(np.uint8)).cuda()
    Q = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((4, 4)).astype(np.float32)).cuda()
    close(attend(cfg(hidden, dtype, hops), g, Q, codes, scales, bias), *reference(g, range(n), Q, codes, scales, bias, dtype))
    # a scale of 255 is NaN, whatever the codes
    g1 = dg4.dg4_build_levels(4, [0, 1, 2], [2, 2, 3], [0, 0, 0], 1)
    codes, scales = codes[:4].contiguous(), torch.full((4, 4, 2), 120, dtype=torch.uint8, device="cuda")
    codes[0], codes[1] = 0, 1
    scales[0, 1, 0] = scales[1, 2, 1] = 255
    nan = attend(cfg(hidden, dtype, 1), g1, Q[:4].contiguous(), codes, scales, bias).isnan().view(4, 4, 32)
    assert nan[0, 1].all() and nan[1, 2].all() and nan[2, 1].all() and nan[2, 2].all() and int(nan.sum()) == 4 * 32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hops", [2, 5])
@pytest.mark.parametrize("size", [-131, -127, -124, -90, 90, 100, 125])
def test_q_at_the_ends_of_its_range(dtype, hops, size):
    """K of 2^size against Q of about its reciprocal: ordinary scores, whichever of the two is at an end. (Rows of Q in turn also with
    a zero, and all zero but one.)"""
    n, hidden = 90, 128
    print(f"kv4 Q against K about 2^{size} {dtype} hops={hops}", flush=True)
    g = circuit(n, 30, hops, seed=4)
    rng = np.random.default_rng(11)
    K = torch.from_numpy((rng.standard_normal((n, hidden)).clip(-3, 3) * 2.0 ** size).astype(np.float32)).cuda()
    V = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).cuda()
    codes, scales = blank(n, hidden)
    dg4.dg4_kv4_write(cfg(hidden, "f32"), K, V, codes, scales)
    q = rng.standard_normal((n, hidden)) * 2.0 ** min(-size, 125)
    q[1::3, 9::32] = 0
    q[2::3, 1:] = 0
    Q = torch.from_numpy(q).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((4, 4)).astype(np.float32)).cuda()
    want, bound = reference(g, range(n), Q, codes, scales, bias, dtype)
    # A product of fp32 with fp32 may be below 2^-126 and lose up to 2^-149, against scores 32 of them: nothing.
    close(attend(cfg(hidden, dtype, hops), g, Q, codes, scales, bias), want, bound)


def test_what_is_left_out_may_hold_anything():
    n, hidden = 40, 256
    g = dg4.dg4_build_levels(n, [0, 1, 2, 3], [10, 10, 11, 11], [0, 1, 0, 1], 2)
    codes, scales = store(1, n, hidden)
    Q = torch.randn((n, hidden), generator=torch.Generator().manual_seed(1)).cuda()
    bias = torch.zeros((8, 4), device="cuda")
    bias[:, 2] = -np.inf                           # inverted fanins: gates 1 and 3
    A = attend(cfg(hidden, "f32"), g, Q, codes, scales, bias)
    codes[1], scales[1] = 0x77, 255
    codes[3], scales[3] = 0x77, 254
    B = attend(cfg(hidden, "f32"), g, Q, codes, scales, bias)
    rest = [v for v in range(n) if v not in (1, 3)]
    assert torch.equal(A[rest], B[rest]) and not A.isnan().any()
    assert B[1].isnan().all()                      # (its own row is not left out)
    bias[:, 2] = 0
    assert attend(cfg(hidden, "f32"), g, Q, codes, scales, bias)[10].isnan().all()


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("span", [-300.0, -40.0, 9.0, 40.0, 300.0])
def test_scores_that_rise_or_fall_along_a_row(hidden, dtype, span):
    """Long rows in ascending id: the maximum moves on in every step, in a few, or stays with the first; V up to 2^118."""
    n, hops = 1200, 8
    g = circuit(n, 200, hops)
    assert np.diff(g.array("nbr_ptr")).max() > 96               # (several steps)
    rise = torch.linspace(0, 1, n, device="cuda")[:, None] * (span / 32 * np.sqrt(32)) + torch.zeros((n, hidden), device="cuda")
    V = rows_of(13, n, hidden, "f32")
    codes, scales = blank(n, hidden)
    dg4.dg4_kv4_write(cfg(hidden, "f32"), rise, V, codes, scales)
    Q = torch.ones((n, hidden), device="cuda").to(tdtype(dtype))
    bias = torch.zeros((hidden // 32, 4), device="cuda")
    want, bound = reference(g, range(n), Q, codes, scales, bias, dtype)
    # Powers below 2^-126, the smallest normal number, may count as zero, those of weights (relative to a base that is at most 4 below
    # the maximum, e^4 < 2^6) and those that join two bases: a source loses at most 2^-126 * 2^6 of the largest weight.
    V = ref.values(codes.cpu().numpy(), scales.cpu().numpy())[1]
    ptr, idx = g.array("nbr_ptr"), g.array("nbr_idx")
    bound = bound + 2.0 ** -120 * np.stack([np.abs(V[idx[ptr[v]:ptr[v + 1]]]).sum(0) for v in range(n)])
    close(attend(cfg(hidden, dtype, hops), g, Q, codes, scales, bias), want, bound)


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_a_store_row_named_twice_harms_no_other(hidden, dtype):
    """What it holds itself is of the two rows that name it, byte by byte; written again, it is right."""
    n, rows = 60, 50
    rng = np.random.default_rng(3)
    ids = rng.permutation(n)[:rows].astype(np.int32)
    ids[[7, 30, 41]] = ids[[8, 12, 49]]
    K, V = (torch.from_numpy(rng.standard_normal((rows, hidden)).astype(np.float32) * np.exp2(rng.integers(-9, 9, (rows, 1)))).to(tdtype(dtype)).cuda() for _ in range(2))

    def written(keep):
        codes, scales = blank(n, hidden)
        at = torch.from_numpy(np.nonzero(keep)[0]).cuda()
        dg4.dg4_kv4_write(cfg(hidden, dtype), K[at].contiguous(), V[at].contiguous(), codes, scales, ids=torch.from_numpy(ids[keep]).cuda())
        return codes, scales
    keep = np.ones(rows, dtype=bool)
    both = written(keep)
    keep[[7, 30, 41]] = False
    last = written(keep)
    keep[[7, 30, 41]], keep[[8, 12, 49]] = True, False
    first = written(keep)
    twice = ids[[8, 12, 49]]
    others = torch.from_numpy(np.setdiff1d(np.arange(n), twice)).cuda()
    for x, y, z in zip(both, last, first):
        assert torch.equal(x[others], y[others]) and ((x == y) | (x == z)).all()
    again = torch.tensor([8, 12, 49], device="cuda")
    dg4.dg4_kv4_write(cfg(hidden, dtype), K[again].contiguous(), V[again].contiguous(), *both, ids=torch.from_numpy(twice).cuda())
    assert all(torch.equal(x, y) for x, y in zip(both, last))


# n rows of the store: offsets above 2^31 in the form that buffer addressing reaches (up to 3 GiB of codes), and past that form
@pytest.mark.parametrize("hidden,n,hops,dtype", [(256, 9_000_000, 2, "bf16"), (128, 18_000_000, 4, "f32"), (256, 13_200_000, 2, "f32"),
                                                 (256, 17_000_000, 4, "bf16"), (128, 26_000_000, 3, "bf16")])
def test_attention_over_a_large_store(hidden, n, hops, dtype):
    """A circuit whose gates lie on both sides of every power of two of bytes; all other rows of the store are NaN."""
    marks = [b // hidden for b in (2 ** 31, 0xC0000000, 2 ** 32) if b // hidden + 8 < n]
    places = np.unique(np.concatenate([[0, 1, 7, 100], [x + d for x in marks for d in (-3, -2, -1, 0, 1, 2)], np.linspace(1000, n - 40, 48), n - 1 - np.arange(6)]).astype(np.int64))
    m = len(places)
    print(f"kv4 attention over {n} rows of {hidden} bytes {dtype} hops={hops}, {m} gates in use", flush=True)
    rng = np.random.default_rng(hops)
    src, dst, inv = [], [], []
    for v in range(4, m):
        for u in rng.choice(np.arange(max(0, v - 12), v), 2, replace=False):
            src.append(u); dst.append(v); inv.append(int(rng.integers(0, 2)))
    src, dst, inv = np.array(src), np.array(dst), np.array(inv, dtype=np.uint8)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()
    g = dg4.dg4_build_levels_device(n, dev(places[src], torch.int32), dev(places[dst], torch.int32), dev(inv, torch.uint8), hops)
    local = dg4.dg4_build_levels(m, src, dst, inv, hops)
    assert np.diff(local.array("nbr_ptr")).max() > {2: 4, 3: 8, 4: 16}[hops]
    codes = torch.full((n, hidden), 0x77, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, hidden // 32, 2), 255, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda: torch.randn((m, hidden), generator=gen, device="cuda").to(tdtype(dtype))
    K, V, Q = rnd(), rnd(), rnd()
    ids = dev(places, torch.int32)
    dg4.dg4_kv4_write(cfg(hidden, dtype), K, V, codes, scales, ids=ids)
    c, s = ref.store(to_np(K), to_np(V))
    assert np.array_equal(codes[ids.long()].cpu().numpy(), c) and np.array_equal(scales[ids.long()].cpu().numpy(), s)
    assert int((scales != 255).flatten(1).any(1).sum()) == m
    K2, V2 = torch.zeros_like(K), torch.zeros_like(V)
    dg4.dg4_kv4_read(cfg(hidden, dtype), codes, scales, K2, V2, ids=ids)
    kv = ref.values(c, s)
    assert torch.equal(K2.cpu(), torch.from_numpy(kv[0]).to(tdtype(dtype))) and torch.equal(V2.cpu(), torch.from_numpy(kv[1]).to(tdtype(dtype)))
    bias = torch.randn((hidden // 32, 4), generator=gen, device="cuda")
    bias[0, 2] = bias[1, 3] = bias[2, 0] = -np.inf
    bias[3] = -np.inf
    A = attend(cfg(hidden, dtype, hops), g, Q, codes, scales, bias, ids=ids)
    close(A, *kv8_ref.attention(local.array("nbr_ptr"), local.array("nbr_idx"), local.array("nbr_rel"), range(m), to_np(Q), *kv, bias.cpu().numpy(), HALF_STEP[dtype]))
    # one of the other rows is what the store holds for it: NaN, and a gate by itself
    lone = torch.tensor([int(places[10]) + 5], dtype=torch.int32, device="cuda")
    assert attend(cfg(hidden, dtype, hops), g, Q[:1].contiguous(), codes, scales, torch.zeros_like(bias), ids=lone).isnan().all()


def test_more_rows_than_a_launch_holds():
    c, n, rows = cfg(128, "bf16", 5), 400, 2 ** 26 + 5
    print(f"kv4 attention over {rows} rows, nearly all padding", flush=True)
    g = circuit(n, 24, 5)
    codes, scales = store(2, n, 128)
    bias = torch.zeros((4, 4), device="cuda")
    at = torch.tensor([0, 3, 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 6, 2 ** 26 - 1, 2 ** 26, rows - 1], device="cuda")
    gates = torch.tensor([5, 399, 0, 17, 398, 5, 100, 250], dtype=torch.int32, device="cuda")
    few = rows_of(1, 8, 128, "bf16")
    want = attend(c, g, few, codes, scales, bias, ids=gates)
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    Q = torch.full((rows, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ids[at], Q[at] = gates, few
    A = attend(c, g, Q, codes, scales, bias, ids=ids)
    assert torch.equal(A[at], want)
    A[at] = 7.0
    assert torch.equal(A, A[1:2].expand_as(A))


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("how,hops", [("device", 2), ("device", 6), ("partitioned", 2), ("partitioned", 3), ("partitioned", 8), ("copies", 2), ("copies", 5)])
def test_attention_over_other_graphs(hidden, dtype, how, hops):
    """Rows of graphs that the device analysed, rows that a partition restricts, rows of its copies of gates."""
    n = 260
    rng = np.random.default_rng(hops)
    src, dst, inv = [], [], []
    for v in range(12, n):
        a, b = rng.choice(np.arange(max(0, v - 40), v), 2, replace=False)
        for u in ([a] if rng.random() < 0.1 else [a, b]):
            src.append(u); dst.append(v); inv.append(int(rng.random() < 0.4))
    if how == "device":
        up = lambda x, t: torch.tensor(x, dtype=t, device="cuda")
        g = dg4.dg4_build_levels_device(n, up(src, torch.int32), up(dst, torch.int32), up(inv, torch.uint8), hops)
    else:
        g = dg4.dg4_build_partitioned(n, src, dst, inv, hops, hops - 1, 16, marks=how == "partitioned")
    print(f"kv4 attention, {how}, {hidden} {dtype} hops={hops} rows={g.n}", flush=True)
    codes, scales = store(5, g.n, hidden)
    Q = torch.from_numpy(rng.standard_normal((g.n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((hidden // 32, 4)).astype(np.float32)).cuda()
    A = attend(cfg(hidden, dtype, hops), g, Q, codes, scales, bias)
    close(A, *reference(g, range(g.n), Q, codes, scales, bias, dtype))


def test_a_graph_that_is_closed_and_a_configuration_past_32_bits():
    n, hidden = 4, 128
    x, (codes, scales), bias = torch.zeros((n, hidden), device="cuda"), blank(n, hidden), torch.zeros((4, 4), device="cuda")
    g = dg4.dg4_build_levels(n, [0, 1], [2, 2], [0, 1], 2)
    dg4.dg4_sparse_attn_kv4_fwd(cfg(hidden, "f32"), g, x, codes, scales, bias, x)
    far = [dg4.LayerConfig(2 ** 32 + hidden, 4, 2, 1, "f32"), dg4.LayerConfig(hidden, 2 ** 32 + 4, 2, 1, "f32"), dg4.LayerConfig(hidden, 4, 2 ** 32 + 2, 1, "f32")]
    for c in far:
        with pytest.raises(dg4.DG4Error):
            dg4.dg4_sparse_attn_kv4_fwd(c, g, x, codes, scales, bias, x)
    g.close()
    with pytest.raises(dg4.DG4Error):
        dg4.dg4_sparse_attn_kv4_fwd(cfg(hidden, "f32"), g, x, codes, scales, bias, x)


def test_binding_checks():
    """Shapes, types and places that do not fit are turned away before anything is queued; nothing to do is fine."""
    n, hidden = 6, 128
    c = cfg(hidden, "f32")
    g = dg4.dg4_build_levels(n, [0, 1], [2, 2], [0, 1], 2)
    f = lambda *shape: torch.zeros(shape, device="cuda")
    b = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device="cuda")
    i = lambda k, t=torch.int32: torch.zeros(k, dtype=t, device="cuda")
    good = dict(x=f(n, hidden), y=f(n, hidden), codes=b(n, 128), scales=b(n, 4, 2), ids=i(n), cfg=c, bias=f(4, 4))
    bad = [dict(x=f(n, hidden).double()), dict(x=f(n, hidden).cpu()), dict(y=f(n - 1, hidden)), dict(x=f(hidden, n).t()), dict(codes=b(n, 127)),
           dict(codes=b(n, 256)), dict(codes=b(n, 128).float()), dict(scales=b(n, 8, 2)), dict(scales=b(n - 1, 4, 2)), dict(scales=b(n, 2, 4)),
           dict(scales=b(n, 8)), dict(ids=i(n - 1)), dict(ids=i(n, torch.int64)), dict(ids=i(n).cpu()), dict(cfg=cfg(hidden, "bf16")),
           dict(cfg=dg4.LayerConfig(256, 8, 2, 1, "f32")), dict(cfg=dg4.LayerConfig(hidden, 4, 2, 1, "f16")), dict(y=f(2 * n, hidden)[::2])]

    def calls(x, y, codes, scales, ids, cfg, bias, **kw):
        yield lambda: dg4.dg4_sparse_attn_kv4_fwd(cfg, g, x, codes, scales, bias, y, ids=ids, **kw)
        yield lambda: dg4.dg4_kv4_write(cfg, x, y, codes, scales, ids=ids, **kw)
        yield lambda: dg4.dg4_kv4_read(cfg, codes, scales, x, y, ids=ids, **kw)
    for change in bad:
        for call in calls(**{**good, **change}):
            with pytest.raises(dg4.DG4Error):
                call()
    for change in (dict(bias=f(3, 4)), dict(bias=f(4, 4).double()), dict(cfg=cfg(hidden, "f32", 3)), dict(codes=b(n - 1, 128), scales=b(n - 1, 4, 2))):
        with pytest.raises(dg4.DG4Error):
            next(calls(**{**good, **change}))()
    for rng in (dict(row_begin=-1), dict(row_end=n + 1), dict(row_begin=3, row_end=2)):
        for call in calls(**good, **rng):
            with pytest.raises(dg4.DG4Error):
                call()
    empty = dict(good, x=f(0, hidden), y=f(0, hidden), ids=i(0))
    none = dict(good, codes=b(0, 128), scales=b(0, 4, 2))
    for call in [*calls(**empty), *calls(**{**empty, "ids": None}), *calls(**good, row_begin=4, row_end=4), *list(calls(**none))[1:]]:
        call()
    with pytest.raises(dg4.DG4Error):
        list(calls(**{**none, "ids": None}))[1]()
    with pytest.raises(dg4.DG4Error):              # (a format of the store in 8 bits only)
        dg4.dg4_kv8_write(c, "fp4", good["x"], good["y"], good["codes"], good["scales"])
    torch.cuda.synchronize()
