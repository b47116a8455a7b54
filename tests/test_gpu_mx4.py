"""Products of rows and weights in 4 bits: projection to rows and into the store, feed-forward sub-block, and a run of them with the
attention between, against plain forms in 64 bits."""
import threading

import numpy as np
import pytest
import torch

import fp4_ref as ref
import kv8_ref
import paper_2502_01681_amd as dg4
from fp4_ref import HALF_STEP
from gpu_utils import tdtype, to_np
from test_gpu_kv4 import SHAPES, blank
from test_gpu_kv8 import circuit

pytestmark = pytest.mark.gpu


def cfg(hidden, dtype, hops=2, **kw):
    return dg4.LayerConfig(hidden, hidden // 32, hops, 1, dtype, **kw)


def states(seed, rows, hidden, dtype, size=None):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, hidden)) * (np.exp(0.4 * rng.standard_normal(hidden)) if size is None else size)
    return torch.from_numpy(x.astype(np.float32)).to(tdtype(dtype)).cuda()


def matrix(seed, k, n, dtype, size=None):
    return states(seed, k, n, dtype, k ** -0.5 if size is None else size)


def project(c, packed, S, **kw):
    out = [torch.full_like(S, 7.0) for _ in range(3)]
    dg4.dg4_qkv_proj_mx4(c, packed, S, *out, **kw)
    return out


def feed(c, w1, w2, S, **kw):
    Out = torch.full_like(S, 7.0)
    dg4.dg4_ffn_mx4_fwd(c, w1, w2, S, Out, **kw)
    return Out


def close(got, want, bound):
    err = np.abs(got - want)
    assert (err <= bound).all(), (err / bound).max()


ROWS = [1, 2, 31, 32, 33, 64, 65, 97, 263, 1030]


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("rows", ROWS)
def test_projection(hidden, dtype, rows):
    print(f"mx4 projection {hidden} {dtype} rows={rows}", flush=True)
    S, W = states(rows, rows, hidden, dtype), matrix(1, hidden, 3 * hidden, dtype)
    c, d = cfg(hidden, dtype), hidden
    packed = dg4.dg4_mx4_pack(c, W)
    got = project(c, packed, S)
    y, bound = ref.proj(to_np(S), to_np(W), HALF_STEP[dtype])
    for i, x in enumerate(got):
        close(to_np(x), y[:, i * d:(i + 1) * d], bound[:, i * d:(i + 1) * d])
    # the same bits for parts of the rows; the others stay
    for lo, hi in ((0, 1), (rows - 1, rows), (rows // 3, rows - rows // 4), (rows // 2, rows // 2)):
        for x, full in zip(project(c, packed, S, row_begin=lo, row_end=hi), got):
            assert torch.equal(x[lo:hi], full[lo:hi]) and (x[:lo] == 7.0).all() and (x[hi:] == 7.0).all()
    # into the store: the sums, rounded once
    assert ref.exact_sums(to_np(S), to_np(W))
    rng = np.random.default_rng(3)
    n = rows + 5
    for ids in (None, rng.permutation(n)[:rows].astype(np.int32)):
        if ids is not None:
            ids[::7] = rng.choice([-1, n, 2 ** 31 - 1, -2 ** 31], len(ids[::7]))
        codes, scales = blank(n, d)
        Q = torch.full_like(S, 7.0)
        dg4.dg4_qkv_proj_kv4(c, packed, S, Q, codes, scales, ids=None if ids is None else torch.from_numpy(ids).cuda())
        assert torch.equal(Q, got[0])
        at = np.arange(rows) if ids is None else ids
        named = (at >= 0) & (at < n)
        code, byte = ref.store(y[:, d:2 * d], y[:, 2 * d:])
        others = np.setdiff1d(np.arange(n), at[named])
        k, s = codes.cpu().numpy(), scales.cpu().numpy()
        # (a zero may have either sign: sums of zeros)
        assert np.array_equal(s[at[named]], byte[named]) and all(np.array_equal(a, b) for a, b in zip(ref.values(k[at[named]], s[at[named]]), ref.values(code[named], byte[named])))
        assert (k[others] == 0x55).all() and (s[others] == 0x66).all()
    lo, hi = rows // 3, rows - rows // 4
    part, Q = blank(n, d), torch.full_like(S, 7.0)
    dg4.dg4_qkv_proj_kv4(c, packed, S, Q, *part, row_begin=lo, row_end=hi)
    full = blank(n, d)
    dg4.dg4_qkv_proj_kv4(c, packed, S, torch.empty_like(S), *full)
    assert all(torch.equal(a[lo:hi], b[lo:hi]) and torch.equal(a[:lo], z[:lo]) and torch.equal(a[hi:], z[hi:]) for a, b, z in zip(part, full, blank(n, d)))
    assert torch.equal(Q[lo:hi], got[0][lo:hi]) and (Q[:lo] == 7.0).all() and (Q[hi:] == 7.0).all()


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_projection_of_rows_far_apart_in_size(hidden, dtype):
    """Blocks of a row and of a column between 2^-20 and 2^20 of each other: sums that are not exact in 32 bits."""
    rng = np.random.default_rng(0)
    S = states(2, 70, hidden, dtype, np.repeat(np.exp2(rng.integers(-20, 20, hidden // 32)), 32))
    S[3], S[4, 40:], S[5, :100] = 0, 0, 0
    W = matrix(3, hidden, 3 * hidden, dtype, 0.1)
    W *= torch.from_numpy(np.repeat(np.exp2(rng.integers(-15, 15, (hidden // 32, 3 * hidden))), 32, axis=0)).to(W)
    W[:, 5], W[32:64, 9] = 0, 0
    assert not ref.exact_sums(to_np(S), to_np(W))
    got = project(cfg(hidden, dtype), dg4.dg4_mx4_pack(cfg(hidden, dtype), W), S)
    close(np.concatenate([to_np(x) for x in got], 1), *ref.proj(to_np(S), to_np(W), HALF_STEP[dtype]))
    assert (got[0][3] == 0).all() and (got[0][:, 5] == 0).all()


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_blocks_that_are_not_finite(hidden, dtype):
    """Of a row: NaN for the whole row, and for no other. Of the weights: NaN for the column, of every row."""
    c, rows = cfg(hidden, dtype), 40
    S, W = states(4, rows, hidden, dtype), matrix(5, hidden, 3 * hidden, dtype)
    W1, W2 = matrix(6, hidden, 4 * hidden, dtype), matrix(7, 4 * hidden, hidden, dtype)
    clean = project(c, dg4.dg4_mx4_pack(c, W), S)
    out = feed(c, dg4.dg4_mx4_pack(c, W1), dg4.dg4_mx4_pack(c, W2), S)
    T = S.clone()
    T[3, 7], T[20, 100], T[33, hidden - 1] = float("nan"), float("inf"), -float("inf")
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
    bad[[3, 20, 33]] = True
    for x, y in zip([*project(c, dg4.dg4_mx4_pack(c, W), T), feed(c, dg4.dg4_mx4_pack(c, W1), dg4.dg4_mx4_pack(c, W2), T)], [*clean, out]):
        assert x[bad].isnan().all() and torch.equal(x[~bad], y[~bad])
    codes, scales = blank(rows, hidden)
    dg4.dg4_qkv_proj_kv4(c, dg4.dg4_mx4_pack(c, W), T, torch.empty_like(T), codes, scales)
    assert (scales[bad] == 255).all() and (scales[~bad] != 255).all()
    V = W.clone()
    V[9, 4], V[hidden - 1, hidden + 40] = float("nan"), float("inf")
    for i, (x, y) in enumerate(zip(project(c, dg4.dg4_mx4_pack(c, V), S), clean)):
        col = torch.zeros(hidden, dtype=torch.bool, device="cuda")
        col[[[4], [40], []][i]] = True
        assert x[:, col].isnan().all() and torch.equal(x[:, ~col], y[:, ~col])
    # an activation that is NaN is not one that the maximum with zero takes away
    for w1, w2 in ((V[:, :4 * hidden], None), (None, 1)):
        A, B = W1.clone(), W2.clone()
        if w2 is None:
            A[9, 4] = float("nan")
        else:
            B[70, 3] = -float("inf")
        assert feed(c, dg4.dg4_mx4_pack(c, A), dg4.dg4_mx4_pack(c, B), S).isnan().all()


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("rows", ROWS)
def test_feed_forward(hidden, dtype, rows):
    print(f"mx4 feed-forward {hidden} {dtype} rows={rows}", flush=True)
    S = states(rows, rows, hidden, dtype)
    S[rows // 2] = 0                               # a row of zeros: LayerNorm of nothing
    W1, W2 = matrix(11, hidden, 4 * hidden, dtype), matrix(12, 4 * hidden, hidden, dtype)
    assert ref.exact_sums(to_np(S), to_np(W1))
    h = np.maximum(ref.rounded(to_np(S)) @ ref.across(to_np(W1)), 0)
    assert ref.exact_sums(h, to_np(W2))
    c = cfg(hidden, dtype)
    w1, w2 = dg4.dg4_mx4_pack(c, W1), dg4.dg4_mx4_pack(c, W2)
    got = feed(c, w1, w2, S)
    close(to_np(got), *ref.ffn(to_np(S), to_np(W1), to_np(W2), c.ln_eps, HALF_STEP[dtype]))
    assert (got[rows // 2] == 0).all()
    for lo, hi in ((0, 1), (rows - 1, rows), (rows // 3, rows - rows // 4), (rows // 2, rows // 2)):
        x = feed(c, w1, w2, S, row_begin=lo, row_end=hi)
        assert torch.equal(x[lo:hi], got[lo:hi]) and (x[:lo] == 7.0).all() and (x[hi:] == 7.0).all()


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("eps,shift", [(0.0, 0.0), (1e-5, 300.0), (0.5, -20.0)])
def test_feed_forward_of_rows_off_zero(hidden, dtype, eps, shift):
    """Rows with a mean far from zero (a difference of large sums would lose their variance), and another epsilon."""
    S = (states(3, 50, hidden, "f32").float() + shift).to(tdtype(dtype))
    W1, W2 = matrix(13, hidden, 4 * hidden, dtype, 2.0 ** -9), matrix(14, 4 * hidden, hidden, dtype)
    h = np.maximum(ref.rounded(to_np(S)) @ ref.across(to_np(W1)), 0)
    assert ref.exact_sums(to_np(S), to_np(W1)) and ref.exact_sums(h, to_np(W2))
    c = cfg(hidden, dtype, ln_eps=eps)
    got = feed(c, dg4.dg4_mx4_pack(c, W1), dg4.dg4_mx4_pack(c, W2), S)
    close(to_np(got), *ref.ffn(to_np(S), to_np(W1), to_np(W2), eps, HALF_STEP[dtype]))


@pytest.mark.parametrize("hidden,dtype", SHAPES)
def test_near_the_products_in_full(hidden, dtype):
    """What 4 bits cost: the block error of rows and weights, 11 % each for normal numbers, and of the activations. Independent errors
    of products add in squares: sqrt(2) * 0.1125 = 0.16 for the projection, with a tenth of room; the sub-block's second term is off by
    up to sqrt(4) * 0.1125 and is half the sum, before a LayerNorm that keeps relative errors."""
    S, W = states(8, 500, hidden, dtype, 1.0), matrix(9, hidden, 3 * hidden, dtype)
    c = cfg(hidden, dtype)
    got = torch.cat(project(c, dg4.dg4_mx4_pack(c, W), S), 1).double()
    full = S.double() @ W.double()
    assert 0.1 < float((got - full).norm() / full.norm()) < 0.176
    W1, W2 = matrix(11, hidden, 4 * hidden, dtype), matrix(12, 4 * hidden, hidden, dtype)
    got = feed(c, dg4.dg4_mx4_pack(c, W1), dg4.dg4_mx4_pack(c, W2), S).double()
    full = torch.nn.functional.layer_norm(S.double() + (S.double() @ W1.double()).relu() @ W2.double(), (hidden,))
    assert float((got - full).norm() / full.norm()) < 0.225 * 0.75


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("hops", [2, 5])
def test_a_layer_as_it_would_be_served(hidden, dtype, hops):
    """Level by level: the gates of a level projected into the store by number, their attention over it, feed-forward; then captured
    into a graph and replayed on other inputs, with eager work between; and the whole against the plain forms."""
    n = 300
    g = circuit(n, 40, hops, seed=1)
    g.upload()
    c = cfg(hidden, dtype, hops)
    S, W = states(21, n, hidden, dtype), matrix(22, hidden, 3 * hidden, dtype)
    W1, W2 = matrix(23, hidden, 4 * hidden, dtype), matrix(24, 4 * hidden, hidden, dtype)
    packed, w1, w2 = (dg4.dg4_mx4_pack(c, w) for w in (W, W1, W2))
    bias = torch.from_numpy(np.random.default_rng(5).standard_normal((hidden // 32, 4)).astype(np.float32)).cuda()
    order, ptr = g.array("order"), g.array("level_ptr")
    level = [torch.from_numpy(order[a:b].astype(np.int32)).cuda() for a, b in zip(ptr[:-1], ptr[1:])]
    gather = [x.long() for x in level]
    codes, scales = blank(n, hidden)
    A, Out = torch.full_like(S, 7.0), torch.full_like(S, 7.0)

    def calls():
        for ids, at in zip(level, gather):
            s = S[at]
            Q, a, o = torch.empty_like(s), torch.empty_like(s), torch.empty_like(s)
            dg4.dg4_qkv_proj_kv4(c, packed, s, Q, codes, scales, ids=ids)
            dg4.dg4_sparse_attn_kv4_fwd(c, g, Q, codes, scales, bias, a, ids=ids)
            dg4.dg4_ffn_mx4_fwd(c, w1, w2, a, o)
            A[at], Out[at] = a, o
    calls()
    assert ref.exact_sums(to_np(S), to_np(W))
    y, _ = ref.proj(to_np(S), to_np(W), 0)
    code, byte = ref.store(y[:, hidden:2 * hidden], y[:, 2 * hidden:])
    kv = ref.values(code, byte)
    got = ref.values(codes.cpu().numpy(), scales.cpu().numpy())
    assert np.array_equal(kv[0], got[0]) and np.array_equal(kv[1], got[1])
    Q = torch.from_numpy(y[:, :hidden]).to(tdtype(dtype))      # (exact sums: Q is their rounding)
    close(to_np(A), *kv8_ref.attention(g.array("nbr_ptr"), g.array("nbr_idx"), g.array("nbr_rel"), range(n), to_np(Q), *kv, bias.cpu().numpy(), HALF_STEP[dtype]))
    close(to_np(Out), *ref.ffn(to_np(A), to_np(W1), to_np(W2), c.ln_eps, HALF_STEP[dtype]))
    # the same on another stream, whole at once, and captured
    whole = [torch.empty_like(S) for _ in range(3)]
    other = blank(n, hidden)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        dg4.dg4_qkv_proj_kv4(c, packed, S, whole[0], *other)
        dg4.dg4_sparse_attn_kv4_fwd(c, g, whole[0], *other, bias, whole[1])
        dg4.dg4_ffn_mx4_fwd(c, w1, w2, whole[1], whole[2])
    side.synchronize()
    assert torch.equal(codes, other[0]) and torch.equal(scales, other[1]) and torch.equal(whole[1], A) and torch.equal(whole[2], Out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        S.copy_(states(30 + step, n, hidden, dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (codes, scales, A, Out)]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (codes, scales, A, Out))), step


def test_two_threads_share_weights():
    """Calls of two threads on streams of their own, the weights read by both."""
    hidden, rows = 256, 3000
    c = cfg(hidden, "bf16")
    W1, W2, W = matrix(1, hidden, 4 * hidden, "bf16"), matrix(2, 4 * hidden, hidden, "bf16"), matrix(3, hidden, 3 * hidden, "bf16")
    packed, w1, w2 = (dg4.dg4_mx4_pack(c, w) for w in (W, W1, W2))
    S = [states(i, rows + 100 * i, hidden, "bf16") for i in range(2)]
    want = [(feed(c, w1, w2, s), *project(c, packed, s)) for s in S]
    torch.cuda.synchronize()
    got, failed = [None, None], []

    def run(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i] = (feed(c, w1, w2, S[i]), *project(c, packed, S[i]))
                torch.cuda.current_stream().synchronize()
        except Exception as e:                     # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed and all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


@pytest.mark.parametrize("hidden,dtype", SHAPES)
@pytest.mark.parametrize("rows", [8160, 8192, 8193, 16385, 24576, 24609, 33000])
def test_rows_around_what_workgroups_take_at_once(hidden, dtype, rows):
    """One tile, two, three and four to a workgroup, whole and not, against calls of few rows (a row's result depends on nothing else)."""
    print(f"mx4 {rows} rows of {hidden} {dtype}", flush=True)
    c = cfg(hidden, dtype)
    S = torch.empty((rows, hidden), dtype=tdtype(dtype), device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(rows))
    packed, w1, w2 = (dg4.dg4_mx4_pack(c, matrix(i, k, m, dtype)) for i, (k, m) in enumerate(((hidden, 3 * hidden), (hidden, 4 * hidden), (4 * hidden, hidden))))
    whole, parts = [*project(c, packed, S), feed(c, w1, w2, S)], [torch.empty_like(S) for _ in range(4)]
    store = blank(rows, hidden), blank(rows, hidden)
    Q = torch.empty_like(S)
    dg4.dg4_qkv_proj_kv4(c, packed, S, Q, *store[0])
    assert torch.equal(Q, whole[0])
    for lo in range(0, rows, 3000):
        kw = dict(row_begin=lo, row_end=min(rows, lo + 3000))
        dg4.dg4_qkv_proj_mx4(c, packed, S, *parts[:3], **kw)
        dg4.dg4_ffn_mx4_fwd(c, w1, w2, S, parts[3], **kw)
        dg4.dg4_qkv_proj_kv4(c, packed, S, Q, *store[1], **kw)
    assert all(torch.equal(a, b) for a, b in zip(whole, parts)) and torch.equal(Q, whole[0])
    assert all(torch.equal(a, b) for a, b in zip(*store))


def test_packed_weights_that_are_not_whole_are_refused():
    c = cfg(128, "f32")
    w = dg4.dg4_mx4_pack(c, torch.zeros((128, 384), device="cuda"))
    x = [torch.zeros((3, 128), device="cuda") for _ in range(4)]
    for packed in (w.packed[:1].expand(w.packed.numel()), w.packed.view(torch.int32), w.packed[:-256], w.packed[16:], w.packed.cpu()):
        with pytest.raises(dg4.DG4Error):
            dg4.dg4_qkv_proj_mx4(c, dg4.Mx4Weights(packed, 128, 384, 128), *x)


@pytest.mark.parametrize("hidden,dtype", [(256, "bf16"), (128, "f32")])
def test_rows_past_four_gigabytes(hidden, dtype):
    """Rows on both sides of every mark of 4.4 GB arrays against calls of those rows alone (a row's result depends on nothing else)."""
    rows = 8_600_000
    print(f"mx4 {rows} rows of {hidden} {dtype}", flush=True)
    S = torch.empty((rows, hidden), dtype=tdtype(dtype), device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    c = cfg(hidden, dtype)
    packed, w1, w2 = (dg4.dg4_mx4_pack(c, matrix(i, k, m, dtype)) for i, (k, m) in enumerate(((hidden, 3 * hidden), (hidden, 4 * hidden), (4 * hidden, hidden))))
    mark = [2 ** 31 // (hidden * S.element_size()), 2 ** 32 // (hidden * S.element_size())]
    some = torch.cat([torch.arange(100), *(torch.arange(x - 80, x + 80) for x in mark), torch.arange(rows - 100, rows),
                      torch.randint(0, rows, (3000,), generator=torch.Generator().manual_seed(2))]).cuda()
    few = S[some].contiguous()
    for got, want in zip([*project(c, packed, S), feed(c, w1, w2, S)], [*project(c, packed, few), feed(c, w1, w2, few)]):
        assert torch.equal(got[some], want)
        del got
    codes, scales = (torch.zeros((rows, hidden), dtype=torch.uint8, device="cuda"), torch.zeros((rows, hidden // 32, 2), dtype=torch.uint8, device="cuda"))
    dg4.dg4_qkv_proj_kv4(c, packed, S, torch.empty_like(S), codes, scales)
    code, byte = blank(len(some), hidden)
    dg4.dg4_qkv_proj_kv4(c, packed, few, torch.empty_like(few), code, byte)
    assert torch.equal(codes[some], code) and torch.equal(scales[some], byte)


def test_binding_checks():
    n, hidden = 6, 128
    c = cfg(hidden, "f32")
    f = lambda *shape: torch.zeros(shape, device="cuda")
    b = lambda *shape: torch.zeros(shape, dtype=torch.uint8, device="cuda")
    W, w1, w2 = (dg4.dg4_mx4_pack(c, f(*s)) for s in ((128, 384), (128, 512), (512, 128)))
    for bad in (f(128, 128), f(384, 128), f(256, 768), f(128, 384).double(), f(128, 384).cpu(), f(384, 128).t(), f(128 * 384), f(128, 384).bfloat16()):
        with pytest.raises(dg4.DG4Error):
            dg4.dg4_mx4_pack(c, bad)

    def proj(cfg=c, w=W, x=f(n, hidden), y=f(n, hidden), **kw):
        dg4.dg4_qkv_proj_mx4(cfg, w, x, y, kw.pop("k", f(n, hidden)), f(n, hidden), **kw)

    def into(cfg=c, w=W, x=f(n, hidden), y=f(n, hidden), codes=b(n, hidden), scales=b(n, 4, 2), **kw):
        dg4.dg4_qkv_proj_kv4(cfg, w, x, y, codes, scales, **kw)

    def ffn(cfg=c, w=w1, x=f(n, hidden), y=f(n, hidden), second=w2, **kw):
        dg4.dg4_ffn_mx4_fwd(cfg, w, second, x, y, **kw)
    for call in (proj, into, ffn):
        for bad in (dict(x=f(n, hidden).double()), dict(x=f(n, hidden).cpu()), dict(y=f(n - 1, hidden)), dict(x=f(hidden, n).t()), dict(y=f(2 * n, hidden)[::2]),
                    dict(w=w2), dict(w=w1 if call is not ffn else W), dict(cfg=cfg(hidden, "bf16")), dict(cfg=cfg(256, "f32")),
                    dict(cfg=dg4.LayerConfig(hidden, 4, 2, 1, "f16")), dict(row_begin=-1), dict(row_end=n + 1), dict(row_begin=3, row_end=2)):
            with pytest.raises(dg4.DG4Error):
                call(**bad)
        same = f(n, hidden)
        with pytest.raises(dg4.DG4Error):          # (not in place)
            call(x=same, y=same)
        call()
        call(row_begin=4, row_end=4)
    with pytest.raises(dg4.DG4Error):
        ffn(second=w1)
    with pytest.raises(dg4.DG4Error):
        proj(k=f(n, hidden).cpu())
    ffn(x=f(0, hidden), y=f(0, hidden))
    into(x=f(0, hidden), y=f(0, hidden))
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    for bad in (dict(codes=b(n, 2 * hidden)), dict(scales=b(n, 8, 2)), dict(ids=ids.long()), dict(ids=ids[:3]), dict(codes=b(n - 1, hidden), scales=b(n - 1, 4, 2)),
                dict(codes=b(0, hidden), scales=b(0, 4, 2), ids=ids)):
        with pytest.raises(dg4.DG4Error):
            into(**bad)
    torch.cuda.synchronize()
    # weights packed from one type serve rows of the other
    S = states(1, 40, hidden, "bf16")
    V = matrix(2, hidden, 3 * hidden, "bf16")
    a = project(cfg(hidden, "f32"), dg4.dg4_mx4_pack(cfg(hidden, "bf16"), V), S.float())
    z = project(cfg(hidden, "f32"), dg4.dg4_mx4_pack(cfg(hidden, "f32"), V.float()), S.float())
    assert all(torch.equal(p, q) for p, q in zip(a, z))
