"""The K|V store in 8 bits: written, read back and attended over, against plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import dg4_synth as synth
import kv8_ref as ref
import paper_2502_01681_amd as dg4
from gpu_utils import tdtype, to_np

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def cfg(hidden, dtype, hops=2):
    return dg4.LayerConfig(hidden, hidden // 32, hops, 1, dtype)


def rows_of(seed, rows, hidden, dtype):
    """Rows with every kind of block: ordinary, tiny, huge, zero, one value only, largest magnitudes at and beside the format's
    largest code, values half way between codes."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, hidden // 32, 32)) * np.exp2(rng.integers(-6, 7, (rows, hidden // 32, 1)))
    kind = rng.integers(0, 12, (rows, hidden // 32))
    x[kind == 0] = 0.0
    x[kind == 1] *= 2.0 ** -130                    # around the smallest normal numbers
    x[kind == 2] *= 2.0 ** 110
    x[kind == 3, 1:] = 0.0
    top = np.array([448.0, 127.0, 127.5, 464.0, 240.0, 1.0, 1.75, 255.0])
    at = np.nonzero(kind == 4)
    x[at[0], at[1]] = np.rint(x[at[0], at[1]] * 4) / 2
    x[at[0], at[1], 5] = top[rng.integers(0, len(top), len(at[0]))]
    at = np.nonzero(kind == 5)                     # ties of either format
    x[at[0], at[1]] = (np.rint(rng.standard_normal((len(at[0]), 32)) * 30) + 0.5) * 0.25
    x[at[0], at[1], 7] = 31.75
    x[kind == 6] *= -1e-3
    x = x.reshape(rows, hidden).astype(np.float32)
    t = torch.from_numpy(x).to(tdtype(dtype)).cuda()
    return t


def same_codes(got, want, fmt):
    return np.array_equal(ref.VALUES[fmt][got], want)      # (by number: a negative zero is a zero)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hidden", [128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 3, 17, 260])
def test_write_and_read_every_row(fmt, hidden, dtype, rows):
    print(f"kv8 {fmt} {hidden} {dtype} rows={rows}", flush=True)
    K, V = rows_of(rows, rows, hidden, dtype), rows_of(rows + 1, rows, hidden, dtype)
    n = rows + 2
    codes = torch.full((n, 2 * hidden), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, hidden // 32, 2), 0x66, dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, K, V, codes, scales)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    assert (c[rows:] == 0x55).all() and (s[rows:] == 0x66).all()
    for part, x in enumerate((K, V)):
        want, byte = ref.quantise(to_np(x), fmt)
        assert np.array_equal(s[:rows, :, part], byte)
        assert same_codes(c[:rows, part * hidden:(part + 1) * hidden], want, fmt)
    K2, V2 = torch.full_like(K, 7.0), torch.full_like(V, 7.0)
    dg4.dg4_kv8_read(cfg(hidden, dtype), fmt, codes, scales, K2, V2)
    for got, want in zip((K2, V2), ref.values(c[:rows], s[:rows], fmt)):
        exact = torch.from_numpy(want).to(tdtype(dtype))           # (subnormal bfloat16 numbers and overflow round)
        assert torch.equal(got.cpu(), exact)
    # within the format's error of what was written: a code is off by half a step at most
    for got, x in zip((K2, V2), (K, V)):
        x, got = to_np(x).astype(np.float64).reshape(rows, -1, 32), to_np(got).astype(np.float64).reshape(rows, -1, 32)
        top = np.abs(x).max(axis=2, keepdims=True)
        if fmt == "int8":
            bound = top / 127 * np.ones_like(x)
        else:
            bound = np.maximum(np.abs(x) * 2.0 ** -4, top * 2.0 ** -17)
        # Scales end at 2^-127: there a code's step is 2^-127 in int8 and 2^-9 of that in e4m3, whatever the block's largest
        # magnitude, so half a step is 2^-128 and 2^-137 (bfloat16's own smallest step is 2^-133)
        worst = (np.abs(got - x) - bound).max()
        assert worst <= (2.0 ** -128 if fmt == "int8" else 2.0 ** -133)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "bf16"), (256, "f32"), (128, "bf16")])
def test_listed_rows(fmt, hidden, dtype):
    print(f"kv8 listed {fmt} {hidden} {dtype}", flush=True)
    n, rows = 300, 77
    rng = np.random.default_rng(5)
    ids = rng.permutation(n)[:rows].astype(np.int32)
    ids[[0, 13, 40, 76]] = [-1, n, 2 ** 31 - 1, -2 ** 31]          # no row of the store
    named = (ids >= 0) & (ids < n)
    K, V = rows_of(1, rows, hidden, dtype), rows_of(2, rows, hidden, dtype)
    codes = torch.full((n, 2 * hidden), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, hidden // 32, 2), 0x66, dtype=torch.uint8, device="cuda")
    lo, hi = 3, 75
    idt = torch.from_numpy(ids).cuda()
    dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, K, V, codes, scales, ids=idt, row_begin=lo, row_end=hi)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    used = np.nonzero(named & (np.arange(rows) >= lo) & (np.arange(rows) < hi))[0]
    others = np.setdiff1d(np.arange(n), ids[used])
    assert (c[others] == 0x55).all() and (s[others] == 0x66).all()
    for part, x in enumerate((K, V)):
        want, byte = ref.quantise(to_np(x)[used], fmt)
        assert np.array_equal(s[ids[used], :, part], byte)
        assert same_codes(c[ids[used], part * hidden:(part + 1) * hidden], want, fmt)
    # read back in another order, rows twice, rows that are none
    back = np.concatenate([ids[used][::-1], ids[used][:5], [-1, n, -2 ** 31]]).astype(np.int32)
    out = [torch.full((len(back), hidden), 7.0, dtype=tdtype(dtype), device="cuda") for _ in range(2)]
    dg4.dg4_kv8_read(cfg(hidden, dtype), fmt, codes, scales, *out, ids=torch.from_numpy(back).cuda())
    for got, want in zip(out, ref.values(c, s, fmt)):
        assert torch.equal(got[:-3].cpu(), torch.from_numpy(want[back[:-3]]).to(tdtype(dtype)))
        assert (got[-3:] == 7.0).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_blocks_that_are_not_finite_read_as_nan(fmt):
    x = torch.ones((4, 128), device="cuda")
    x[0, 3], x[1, 40], x[2, 127] = float("nan"), float("inf"), float("-inf")
    x[3, 0] = torch.finfo(torch.float32).max
    codes, scales = torch.zeros((4, 256), dtype=torch.uint8, device="cuda"), torch.zeros((4, 4, 2), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(cfg(128, "f32"), fmt, x, torch.ones_like(x), codes, scales)
    K, V = torch.zeros_like(x), torch.zeros_like(x)
    dg4.dg4_kv8_read(cfg(128, "f32"), fmt, codes, scales, K, V)
    bad = torch.zeros((4, 4), dtype=torch.bool)
    bad[0, 0] = bad[1, 1] = bad[2, 3] = True
    assert torch.equal(K.view(4, 4, 32).isnan().all(2).cpu(), bad) and torch.equal(K.view(4, 4, 32).isnan().any(2).cpu(), bad)
    assert (V == 1).all() and (K[3, 32:] == 1).all()


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("f32", "int8")])
def test_store_past_four_gigabytes(dtype, fmt):
    n = 8_700_000
    print(f"kv8 far rows {dtype} {fmt}", flush=True)
    codes = torch.zeros((n, 512), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n, 8, 2), dtype=torch.uint8, device="cuda")
    ids = torch.tensor([n - 1, 0, 2 ** 23 + 1, 2 ** 23 - 1, 2 ** 22, n - 2], dtype=torch.int32, device="cuda")
    K, V = rows_of(8, 6, 256, dtype), rows_of(9, 6, 256, dtype)
    dg4.dg4_kv8_write(cfg(256, dtype), fmt, K, V, codes, scales, ids=ids)
    assert int((codes.view(torch.int64).ne(0).any(1)).sum()) == 6
    for part, x in enumerate((K, V)):
        want, byte = ref.quantise(to_np(x), fmt)
        assert same_codes(codes[ids.long(), part * 256:(part + 1) * 256].cpu().numpy(), want, fmt)
        assert np.array_equal(scales[ids.long(), :, part].cpu().numpy(), byte)
    K2, V2 = torch.zeros_like(K), torch.zeros_like(V)
    dg4.dg4_kv8_read(cfg(256, dtype), fmt, codes, scales, K2, V2, ids=ids)
    kv = ref.values(codes[ids.long()].cpu().numpy(), scales[ids.long()].cpu().numpy(), fmt)
    assert torch.equal(K2.cpu(), torch.from_numpy(kv[0]).to(tdtype(dtype))) and torch.equal(V2.cpu(), torch.from_numpy(kv[1]).to(tdtype(dtype)))
    # a circuit of that many gates, nearly all primary inputs: the last gate reads the first and the last ones
    src = np.array([n - 3, 0, n - 2, 2 ** 23 + 1], dtype=np.int32)
    dst = np.array([n - 2, n - 2, n - 1, n - 1], dtype=np.int32)
    dev = lambda a, t: torch.from_numpy(a).to(t).cuda()
    g = dg4.dg4_build_levels_device(n, dev(src, torch.int32), dev(dst, torch.int32), torch.zeros(4, dtype=torch.uint8, device="cuda"), 2)
    row = np.array([0, 2 ** 23 + 1, n - 3, n - 2, n - 1])
    rel = np.array([3, 1, 3, 1, 0])
    dg4.dg4_kv8_write(cfg(256, dtype), fmt, K[:1] * 0 + 1, V[5:] * 0 + 2, codes, scales, ids=ids[:1] * 0 + (n - 3))
    Q = torch.from_numpy(np.random.default_rng(3).standard_normal((1, 256)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.zeros((8, 4), device="cuda")
    A = torch.zeros_like(Q)
    # (blocks far beyond ordinary size would make the softmax a choice of one: halve their exponents)
    scales.clamp_(110, 128)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(256, dtype), fmt, g, Q, codes, scales, bias, A, ids=ids[:1])
    kv = ref.values(codes[torch.from_numpy(row).cuda()].cpu().numpy(), scales[torch.from_numpy(row).cuda()].cpu().numpy(), fmt)
    want, bound = ref.attention(np.array([0, 5]), np.arange(5), rel, [0], to_np(Q), kv[0], kv[1], np.zeros((8, 4)), HALF_STEP[dtype])
    assert (np.abs(to_np(A) - want) <= bound).all()


def circuit(n, window, hops, seed=0, chain=False):
    """A graph with single-source rows (inputs), inverters and AND gates; with `chain`, every gate reads the two before it."""
    rng = np.random.default_rng(seed)
    src, dst, inv = [], [], []
    for v in range(max(2, n // 20), n):
        a, b = (v - 1, v - 2) if chain else rng.choice(np.arange(max(0, v - window), v), 2, replace=False)
        for u in ([a] if not chain and rng.random() < 0.1 else [a, b]):
            src.append(u); dst.append(v); inv.append(int(rng.random() < 0.4))
    return dg4.dg4_build_levels(n, src, dst, inv, hops)


def store(seed, n, hidden, fmt):
    rng = np.random.default_rng(seed)
    codes = torch.zeros((n, 2 * hidden), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n, hidden // 32, 2), dtype=torch.uint8, device="cuda")
    kv = [torch.from_numpy((rng.standard_normal((n, hidden)) * np.exp2(rng.integers(-2, 2, (n, 1)))).astype(np.float32)).cuda() for _ in range(2)]
    dg4.dg4_kv8_write(cfg(hidden, "f32"), fmt, *kv, codes, scales)
    return codes, scales


def reference(g, gates, Q, codes, scales, fmt, bias, dtype):
    K, V = ref.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
    return ref.attention(g.array("nbr_ptr"), g.array("nbr_idx"), g.array("nbr_rel"), gates, to_np(Q), K, V, bias.cpu().numpy(), HALF_STEP[dtype])


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hidden", [128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,hops", [(230, 1), (230, 2), (230, 3), (150, 4), (200, 5), (330, 8)])
def test_attention(fmt, hidden, dtype, n, hops):
    g = circuit(n, 24 if hops < 8 else 330, hops)
    longest = int(np.diff(g.array("nbr_ptr")).max())
    print(f"kv8 attention {fmt} {hidden} {dtype} n={n} hops={hops} longest row {longest}", flush=True)
    codes, scales = store(3, n, hidden, fmt)
    rng = np.random.default_rng(4)
    Q = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((hidden // 32, 4)).astype(np.float32)).cuda()
    want, bound = reference(g, range(n), Q, codes, scales, fmt, bias, dtype)
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q, codes, scales, bias, A)
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()
    # a gate alone in its row copies its values exactly
    single = np.nonzero(np.diff(g.array("nbr_ptr")) == 1)[0]
    V = ref.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)[1]
    assert len(single) and torch.equal(A[single].cpu(), torch.from_numpy(V[single]).to(tdtype(dtype)))
    # the same bits for parts of the rows, and for listed gates; other rows stay
    for lo, hi in ((0, 1), (5, 6), (n - 1, n), (3, n - 7), (9, 9)):
        B = torch.full_like(Q, 7.0)
        dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q, codes, scales, bias, B, row_begin=lo, row_end=hi)
        assert torch.equal(B[lo:hi], A[lo:hi]) and (B[:lo] == 7.0).all() and (B[hi:] == 7.0).all()
    ids = rng.permutation(n)[:61].astype(np.int32)
    ids[[0, 9, 60]] = [-1, n, 2 ** 31 - 1]
    ids[20] = ids[21]
    ok = (ids >= 0) & (ids < n)
    pick = torch.from_numpy(np.where(ok, ids, 0).astype(np.int64)).cuda()
    B = torch.full((61, hidden), 7.0, dtype=Q.dtype, device="cuda")
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q[pick].contiguous(), codes, scales, bias, B, ids=torch.from_numpy(ids).cuda())
    assert torch.equal(B[torch.from_numpy(ok).cuda()], A[pick][torch.from_numpy(ok).cuda()]) and (B[torch.from_numpy(~ok).cuda()] == 7.0).all()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("hops", [2, 3, 5, 8])
def test_relations_left_out(fmt, hops):
    """Heads: 0 without the gate itself, 1 without any relation, 2 without what lies further up, 3 with the type's lowest value."""
    n, hidden = 120, 128
    g = circuit(n, 60, hops, seed=2)
    codes, scales = store(6, n, hidden, fmt)
    rng = np.random.default_rng(7)
    Q = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).cuda()
    bias = torch.from_numpy(rng.standard_normal((4, 4)).astype(np.float32))
    bias[0, 0] = -np.inf
    bias[1] = -np.inf
    bias[2, 3] = -np.inf
    bias[3] = torch.finfo(torch.float32).min
    bias = bias.cuda()
    # the lowest value swallows the score: every source counts the same there
    want, bound = reference(g, range(n), Q, codes, scales, fmt, bias, "f32")
    rows = g.array("nbr_ptr")
    V = ref.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)[1]
    for v in range(n):
        src = g.array("nbr_idx")[rows[v]:rows[v + 1]]
        want[v, 96:] = V[src, 96:].mean(axis=0)
        bound[v, 96:] = (2 * len(src) + 4) * 2.0 ** -24 * np.abs(V[src, 96:]).mean(axis=0) + 1e-37
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, "f32", hops), fmt, g, Q, codes, scales, bias, A)
    assert (A[:, 32:64] == 0).all()
    single = np.diff(rows) == 1
    assert (A[torch.from_numpy(single).cuda()][:, :32] == 0).all()
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hops", [2, 5])
def test_any_scale_and_code(fmt, dtype, hops):
    """Stores as a caller may fill them: every code that is a number, scales from the smallest on."""
    n, hidden = 90, 128
    g = circuit(n, 30, hops, seed=4)
    rng = np.random.default_rng(8)
    codes = rng.integers(0, 256, (n, 2 * hidden)).astype(np.uint8)
    if fmt == "e4m3":
        codes[(codes & 127) == 127] = 0x7E
    scales = rng.integers(105, 121, (n, 4, 2))
    scales[rng.random(scales.shape) < 0.2] = 0
    scales[rng.random(scales.shape) < 0.1] = 1
    scales[:, :, 1] += rng.integers(0, 3, (n, 4)) * 30         # (values far apart in size)
    codes, scales = torch.from_numpy(codes).cuda(), torch.from_numpy(scales.astype(np.uint8)).cuda()
    Q = torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    bias = torch.from_numpy(rng.standard_normal((4, 4)).astype(np.float32)).cuda()
    want, bound = reference(g, range(n), Q, codes, scales, fmt, bias, dtype)
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q, codes, scales, bias, A)
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()
    # a scale of 255 is NaN, whatever the codes
    g1 = dg4.dg4_build_levels(4, [0, 1, 2], [2, 2, 3], [0, 0, 0], 1)
    codes, scales = codes[:4].contiguous(), torch.full((4, 4, 2), 120, dtype=torch.uint8, device="cuda")
    codes[0], codes[1] = 0, 1
    scales[0, 1, 0] = scales[1, 2, 1] = 255
    A = torch.zeros((4, hidden), dtype=Q.dtype, device="cuda")
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, 1), fmt, g1, Q[:4].contiguous(), codes, scales, bias, A)
    nan = A.isnan().view(4, 4, 32)
    assert nan[0, 1].all() and nan[1, 2].all() and nan[2, 1].all() and nan[2, 2].all() and int(nan.sum()) == 4 * 32


def test_what_is_left_out_may_hold_anything():
    n, hidden = 40, 256
    src, dst = [0, 1, 2, 3], [10, 10, 11, 11]
    g = dg4.dg4_build_levels(n, src, dst, [0, 1, 0, 1], 2)
    for fmt in ("e4m3", "int8"):
        codes, scales = store(1, n, hidden, fmt)
        Q = torch.randn((n, hidden), generator=torch.Generator().manual_seed(1)).cuda()
        bias = torch.zeros((8, 4), device="cuda")
        bias[:, 2] = -np.inf                       # inverted fanins: gates 1 and 3
        A, B = torch.zeros_like(Q), torch.zeros_like(Q)
        dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, "f32"), fmt, g, Q, codes, scales, bias, A)
        codes[1], scales[1] = 0x7F, 255            # NaN of either kind
        codes[3], scales[3] = 0x7F, 254
        dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, "f32"), fmt, g, Q, codes, scales, bias, B)
        rest = [v for v in range(n) if v not in (1, 3)]
        assert torch.equal(A[rest], B[rest]) and not A.isnan().any()
        assert B[1].isnan().all()                  # (its own row is not left out)
        bias[:, 2] = 0
        dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, "f32"), fmt, g, Q, codes, scales, bias, B)
        assert B[10].isnan().all()


@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "bf16")])
def test_captured_and_on_other_streams(hidden, dtype):
    """Write, attend, read back on a stream of their own, then captured and replayed with other inputs."""
    n = 200
    g = circuit(n, 20, 2)
    g.upload()
    c = cfg(hidden, dtype)
    rng = np.random.default_rng(1)
    rnd = lambda: torch.from_numpy(rng.standard_normal((n, hidden)).astype(np.float32)).to(tdtype(dtype)).cuda()
    K, V, Q = rnd(), rnd(), rnd()
    bias = torch.zeros((hidden // 32, 4), device="cuda")
    codes = torch.zeros((n, 2 * hidden), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n, hidden // 32, 2), dtype=torch.uint8, device="cuda")
    out = [torch.zeros_like(Q) for _ in range(3)]

    def calls():
        dg4.dg4_kv8_write(c, "int8", K, V, codes, scales)
        dg4.dg4_sparse_attn_kv8_fwd(c, "int8", g, Q, codes, scales, bias, out[0])
        dg4.dg4_kv8_read(c, "int8", codes, scales, out[1], out[2])
    calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    for t in out:
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        K.copy_(rnd()); V.copy_(rnd()); Q.copy_(rnd())
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out] + [codes.clone(), scales.clone()]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, out + [codes, scales])), step


@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "bf16"), (256, "f32"), (128, "bf16")])
@pytest.mark.parametrize("span", [-300.0, -40.0, 9.0, 40.0, 300.0])
def test_scores_that_rise_or_fall_along_a_row(hidden, dtype, span):
    """Long rows in ascending id: the maximum moves on in every step, in a few, or stays with the first; V up to 2^118."""
    n, hops = 1200, 8
    g = circuit(n, 200, hops)
    assert np.diff(g.array("nbr_ptr")).max() > 96               # (more than three steps)
    codes, scales = store(12, n, hidden, "int8")
    rise = torch.linspace(0, 1, n, device="cuda")[:, None] * (span / 32 * np.sqrt(32)) + torch.zeros((n, hidden), device="cuda")
    V = rows_of(13, n, hidden, "f32")
    dg4.dg4_kv8_write(cfg(hidden, "f32"), "int8", rise, V, codes, scales)
    Q = torch.ones((n, hidden), device="cuda").to(tdtype(dtype))
    bias = torch.zeros((hidden // 32, 4), device="cuda")
    want, bound = reference(g, range(n), Q, codes, scales, "int8", bias, dtype)
    # Powers below 2^-126, the smallest normal number, may count as zero, those of weights (relative to a base that is at most 4
    # below the maximum, e^4 < 2^6, and divided by 2^6) and those that join two bases: a source loses at most 2^-126 * 2^6 of the
    # largest weight, and the sum of weights is at least that. Blocks of 2^110 show it: with weights below 2^-126 taken out, the
    # 64-bit result itself is 1413 times the bound above away (row 1153, span -300).
    V = ref.values(codes.cpu().numpy(), scales.cpu().numpy(), "int8")[1]
    ptr, idx = g.array("nbr_ptr"), g.array("nbr_idx")
    bound = bound + 2.0 ** -120 * np.stack([np.abs(V[idx[ptr[v]:ptr[v + 1]]]).sum(0) for v in range(n)])
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), "int8", g, Q, codes, scales, bias, A)
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "bf16")])
@pytest.mark.parametrize("hops", [2, 3, 6])
def test_attention_in_place(hidden, dtype, hops):
    n = 3000 if hops < 6 else 500
    g = circuit(n, 60, hops)
    codes, scales = store(5, n, hidden, "e4m3")
    Q = rows_of(6, n, hidden, dtype)
    A, bias = torch.zeros_like(Q), torch.zeros((hidden // 32, 4), device="cuda")
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), "e4m3", g, Q, codes, scales, bias, A)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), "e4m3", g, Q, codes, scales, bias, Q)
    assert torch.equal(Q, A)


def test_more_rows_than_a_launch_holds():
    c, n, rows = cfg(128, "bf16", 5), 400, 2 ** 26 + 5
    print(f"kv8 attention over {rows} rows, nearly all padding", flush=True)
    g = circuit(n, 24, 5)
    assert np.diff(g.array("nbr_ptr")).max() > 16              # (four rows to a workgroup)
    codes, scales = store(2, n, 128, "int8")
    bias = torch.zeros((4, 4), device="cuda")
    at = torch.tensor([0, 3, 2 ** 25 - 1, 2 ** 25, 2 ** 25 + 6, 2 ** 26 - 1, 2 ** 26, rows - 1], device="cuda")
    gates = torch.tensor([5, 399, 0, 17, 398, 5, 100, 250], dtype=torch.int32, device="cuda")
    few = rows_of(1, 8, 128, "bf16")
    want = torch.zeros_like(few)
    dg4.dg4_sparse_attn_kv8_fwd(c, "int8", g, few, codes, scales, bias, want, ids=gates)
    ids = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    Q, A = (torch.full((rows, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ids[at], Q[at] = gates, few
    dg4.dg4_sparse_attn_kv8_fwd(c, "int8", g, Q, codes, scales, bias, A, ids=ids)
    assert torch.equal(A[at], want)
    A[at] = 7.0
    assert torch.equal(A, A[:1].expand_as(A))


def test_binding_checks():
    """Shapes, types, formats and places that do not fit are turned away before anything is queued; nothing to do is fine."""
    n, hidden = 6, 128
    c = cfg(hidden, "f32")
    g = dg4.dg4_build_levels(n, [0, 1], [2, 2], [0, 1], 2)
    f = lambda *shape: torch.zeros(shape, device="cuda")
    b = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device="cuda")
    i = lambda k, t=torch.int32: torch.zeros(k, dtype=t, device="cuda")
    good = dict(x=f(n, hidden), y=f(n, hidden), codes=b(n, 256), scales=b(n, 4, 2), ids=i(n), fmt="int8", cfg=c, bias=f(4, 4))
    bad = [dict(x=f(n, hidden).double()), dict(x=f(n, hidden).cpu()), dict(y=f(n - 1, hidden)), dict(x=f(hidden, n).t()), dict(codes=b(n, 255)),
           dict(codes=b(n, 256).float()), dict(scales=b(n, 8, 2)), dict(scales=b(n - 1, 4, 2)), dict(scales=b(n, 2, 4)), dict(scales=b(n, 8)), dict(ids=i(n - 1)), dict(ids=i(n, torch.int64)),
           dict(ids=i(n).cpu()), dict(fmt="fp8"), dict(cfg=cfg(hidden, "bf16")), dict(cfg=dg4.LayerConfig(256, 8, 2, 1, "f32")),
           dict(cfg=dg4.LayerConfig(hidden, 4, 2, 1, "f16")), dict(y=f(2 * n, hidden)[::2])]
    attn_only = [dict(bias=f(3, 4)), dict(bias=f(4, 4).double()), dict(cfg=cfg(hidden, "f32", 3))]

    def calls(x, y, codes, scales, ids, fmt, cfg, bias, **kw):
        yield lambda: dg4.dg4_sparse_attn_kv8_fwd(cfg, fmt, g, x, codes, scales, bias, y, ids=ids, **kw)
        yield lambda: dg4.dg4_kv8_write(cfg, fmt, x, y, codes, scales, ids=ids, **kw)
        yield lambda: dg4.dg4_kv8_read(cfg, fmt, codes, scales, x, y, ids=ids, **kw)
    for change in bad:
        for call in calls(**{**good, **change}):
            with pytest.raises(dg4.DG4Error):
                call()
    for change in attn_only:
        with pytest.raises(dg4.DG4Error):
            next(calls(**{**good, **change}))()
    for rng in (dict(row_begin=-1), dict(row_end=n + 1), dict(row_begin=3, row_end=2)):
        for call in calls(**good, **rng):
            with pytest.raises(dg4.DG4Error):
                call()
    with pytest.raises(dg4.DG4Error):              # a store with fewer rows than the graph has gates
        next(calls(**{**good, "codes": b(n - 1, 256), "scales": b(n - 1, 4, 2)}))()
    empty = dict(good, x=f(0, hidden), y=f(0, hidden), ids=i(0))
    for call in calls(**empty):
        call()
    for call in list(calls(**{**empty, "ids": None})) + list(calls(**good, row_begin=4, row_end=4)):
        call()
    none = dict(good, codes=b(0, 256), scales=b(0, 4, 2))
    for call in list(calls(**none))[1:]:
        call()
    with pytest.raises(dg4.DG4Error):
        list(calls(**{**none, "ids": None}))[1]()
    torch.cuda.synchronize()
    # rows given head by head are the same rows
    a, z = f(n, 4, 32).normal_(), f(n, 4, 32)
    dg4.dg4_kv8_write(c, "int8", a, a, good["codes"], good["scales"])
    dg4.dg4_kv8_read(c, "int8", good["codes"], good["scales"], z, z.clone())
    assert float((z - a).abs().max()) < 0.05
