"""The projection with low-rank adapters against 64 bits, and the serving path as a whole."""
import numpy as np
import pytest
import torch

import kv8_ref as ref
import paper_2502_01681_amd as dg4
from gpu_utils import tdtype, to_np

pytestmark = pytest.mark.gpu

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def weights(seed, hidden, n, rank, dtype):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *shape: torch.randn(shape, generator=gen, dtype=torch.float64)
    W = (rnd(hidden, 3 * hidden) * hidden ** -0.5).to(tdtype(dtype)).cuda()
    down = (rnd(n, hidden, rank) * hidden ** -0.5).to(tdtype(dtype)).cuda()
    up = (rnd(n, rank, 3 * hidden) * rank ** -0.5).to(tdtype(dtype)).cuda()
    gain = (torch.rand(n, generator=gen) + 0.5).cuda()
    return W, down, up, gain


def rows_of(seed, rows, hidden, dtype):
    return torch.randn((rows, hidden), generator=torch.Generator().manual_seed(seed), dtype=torch.float64).to(tdtype(dtype)).cuda()


def reference(S, adapter, W, down, up, gain, dtype):
    """(Q|K|V in 64 bits, how far a computation in 32 bits may be). Sums of d and of rank products, each step within 2^-23 of the
    magnitudes summed; in bfloat16 S Down is carried as two bfloat16 numbers, each half a step off what it rounds: 2^-16; the
    result is rounded once."""
    s, w = S.double(), W.double()
    d = s.shape[1]
    y = s @ w
    size = (d + 8) * (s.abs() @ w.abs())
    for a in range(down.shape[0]):
        r = torch.nonzero(adapter == a).flatten()
        if not len(r):
            continue
        t, u, g = s[r] @ down[a].double(), up[a].double(), gain[a].double()
        y[r] += g * (t @ u)
        size[r] += g * (d + down.shape[2] + 12) * ((s[r].abs() @ down[a].double().abs()) @ u.abs())
        if dtype == "bf16":
            size[r] += g * 2.0 ** 7 * (t.abs() @ u.abs())
    return y, size * 2.0 ** -23 + HALF_STEP[dtype] * y.abs() + 1e-37


def project(cfg, packed, S, adapter, **kw):
    out = [torch.full_like(S, 7.0) for _ in range(3)]
    dg4.dg4_qkv_proj_lora(cfg, packed, S, adapter, *out, **kw)
    return out


def arrangement(kind, rows, n, rng):
    if kind == "one":
        a = np.full(rows, n - 1)
    elif kind == "runs":
        a = np.sort(rng.integers(-1, n, rows))[::-1].copy()
    elif kind == "own":
        a = np.arange(rows) % n
    else:                                          # any order, with rows that have none
        a = rng.integers(-1, n + 1, rows)
        a[rng.integers(0, rows, max(1, rows // 20))] = 2 ** 31 - 1
        a[rng.integers(0, rows, max(1, rows // 20))] = -2 ** 31
    return torch.from_numpy(a.astype(np.int32)).cuda()


@pytest.mark.parametrize("hidden", [128, 256])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rank", [1, 4, 8, 16, 27, 33, 64])
@pytest.mark.parametrize("kind,rows", [("one", 1), ("own", 64), ("any", 3), ("runs", 131), ("any", 700), ("runs", 4500), ("any", 4500), ("one", 5003), ("runs", 17_003),
                                       ("any", 16_500), ("runs", 33_100)])
def test_projection(hidden, dtype, rank, kind, rows):
    n = 9 if kind != "own" else 64
    print(f"lora {dtype} {hidden} rank={rank} {kind} rows={rows}", flush=True)
    cfg = dg4.LayerConfig(hidden, hidden // 32, 2, 1, dtype)
    W, down, up, gain = weights(rank, hidden, n, rank, dtype)
    S = rows_of(rows, rows, hidden, dtype)
    adapter = arrangement(kind, rows, n, np.random.default_rng(rows + rank))
    packed = dg4.dg4_lora_pack(cfg, W, down, up, gain)
    got = project(cfg, packed, S, adapter)
    want, bound = reference(S, adapter, W, down, up, gain, dtype)
    worst = ((torch.cat(got, 1).double() - want).abs() / bound).max()
    assert worst <= 1, float(worst)


@pytest.mark.parametrize("hidden,dtype,rank", [(128, "f32", 8), (256, "f32", 27), (128, "bf16", 64), (256, "bf16", 16)])
@pytest.mark.parametrize("rows", [6011, 33_011])
def test_a_row_depends_on_itself_alone(hidden, dtype, rank, rows):
    """The same bits in any range of rows, in any order, beside any other adapters; other rows stay."""
    n = 7
    cfg = dg4.LayerConfig(hidden, hidden // 32, 2, 1, dtype)
    W, down, up, gain = weights(3, hidden, n, rank, dtype)
    S, adapter = rows_of(4, rows, hidden, dtype), arrangement("runs", rows, n, np.random.default_rng(2))
    packed = dg4.dg4_lora_pack(cfg, W, down, up, gain)
    whole = project(cfg, packed, S, adapter)
    for lo, hi in ((0, 1), (1, 3), (5, 38), (100, 612), (63, 4200), (6010, 6011), (17, 17), (1, 6011), (rows - 17_000, rows - 1), (1, rows)):
        lo = max(lo, 0)
        part = project(cfg, packed, S, adapter, row_begin=lo, row_end=hi)
        for x, y in zip(part, whole):
            assert torch.equal(x[lo:hi], y[lo:hi]) and (x[:lo] == 7.0).all() and (x[hi:] == 7.0).all(), (lo, hi)
    order = torch.randperm(rows, generator=torch.Generator().manual_seed(1)).cuda()
    for some in (order, order[:200], order[:5]):
        for x, y in zip(project(cfg, packed, S[some].contiguous(), adapter[some].contiguous()), whole):
            assert torch.equal(x, y[some])
    # an adapter full of NaN and infinities reaches its own rows alone
    down[2], up[4] = float("nan"), float("inf")
    bad = dg4.dg4_lora_pack(cfg, W, down, up, gain)
    fine = (adapter != 2) & (adapter != 4)
    for mix, pick in ((torch.arange(rows, device="cuda"), slice(None)), (order, order)):
        for x, y in zip(project(cfg, bad, S[mix].contiguous(), adapter[mix].contiguous()), whole):
            keep = fine[mix]
            assert torch.equal(x[keep], y[pick][keep]) and not torch.isfinite(x[~keep].float()).any()
    # so does a row that is not finite
    T = S.clone()
    T[10], T[4000, 3] = float("nan"), float("inf")
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[10] = keep[4000] = False
    for x, y in zip(project(cfg, packed, T, adapter), whole):
        assert torch.equal(x[keep], y[keep]) and x[10].isnan().all() and not torch.isfinite(x[4000].float()).any()


@pytest.mark.parametrize("hidden,dtype", [(128, "f32"), (256, "f32"), (128, "bf16"), (256, "bf16")])
@pytest.mark.parametrize("rows", [50, 5000, 33_000])
def test_without_adapters(hidden, dtype, rows):
    cfg = dg4.LayerConfig(hidden, hidden // 32, 2, 1, dtype)
    W, down, up, gain = weights(3, hidden, 2, 8, dtype)
    S = rows_of(4, rows, hidden, dtype)
    plain = project(cfg, dg4.dg4_lora_pack(cfg, W), S, None)
    none = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    some = dg4.dg4_lora_pack(cfg, W, down, up)
    for other in (project(cfg, some, S, None), project(cfg, some, S, none), project(cfg, dg4.dg4_lora_pack(cfg, W), S, none * 0)):
        assert all(torch.equal(x, y) for x, y in zip(plain, other))
    want, bound = reference(S, none, W, down, up, gain, dtype)
    assert ((torch.cat(plain, 1).double() - want).abs() <= bound).all()
    # a gain that is not given is one
    one = project(cfg, dg4.dg4_lora_pack(cfg, W, down, up, torch.ones(2, device="cuda")), S, none * 0)
    assert all(torch.equal(x, y) for x, y in zip(project(cfg, some, S, none * 0), one))


@pytest.mark.parametrize("hidden,dtype,fmt", [(128, "f32", "int8"), (256, "bf16", "e4m3"), (256, "f32", "e4m3"), (128, "bf16", "int8")])
def test_serving_path(hidden, dtype, fmt):
    """Circuits of a batch through all of it: projection with each circuit's adapter, K and V into the store, attention over
    the store, rows read back. Checked step by step in 64 bits, then captured in a graph and replayed with other inputs."""
    sizes, n_adapters, rank = [61, 1, 140, 33, 90], 3, 8
    of = [0, -1, 2, 1, 0]
    n = sum(sizes)
    rng = np.random.default_rng(9)
    src, dst, inv, first = [], [], [], 0
    for size in sizes:                             # no edge from a circuit to another
        for v in range(3, size):
            for u in rng.choice(np.arange(max(0, v - 20), v), 2, replace=False):
                src.append(first + u); dst.append(first + v); inv.append(int(rng.integers(0, 2)))
        first += size
    g = dg4.dg4_build_levels(n, src, dst, inv, 2)
    g.upload()
    heads = hidden // 32
    cfg = dg4.LayerConfig(hidden, heads, 2, 1, dtype)
    W, down, up, gain = weights(5, hidden, n_adapters, rank, dtype)
    packed = dg4.dg4_lora_pack(cfg, W, down, up, gain)
    adapter = torch.from_numpy(np.repeat(of, sizes).astype(np.int32)).cuda()
    bias = torch.randn((heads, 4), generator=torch.Generator().manual_seed(3)).cuda()
    S = rows_of(6, n, hidden, dtype)
    Q, K, V, A, K2, V2 = (torch.zeros_like(S) for _ in range(6))
    codes = torch.zeros((n, 2 * hidden), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((n, heads, 2), dtype=torch.uint8, device="cuda")
    every = [Q, K, V, codes, scales, A, K2, V2]

    def calls():
        dg4.dg4_qkv_proj_lora(cfg, packed, S, adapter, Q, K, V)
        dg4.dg4_kv8_write(cfg, fmt, K, V, codes, scales)
        dg4.dg4_sparse_attn_kv8_fwd(cfg, fmt, g, Q, codes, scales, bias, A)
        dg4.dg4_kv8_read(cfg, fmt, codes, scales, K2, V2)
    calls()
    want, bound = reference(S, adapter, W, down, up, gain, dtype)
    assert ((torch.cat([Q, K, V], 1).double() - want).abs() <= bound).all()
    for part, x in enumerate((K, V)):
        code, byte = ref.quantise(to_np(x), fmt)
        assert np.array_equal(ref.VALUES[fmt][codes[:, part * hidden:(part + 1) * hidden].cpu().numpy()], code)
        assert np.array_equal(scales[:, :, part].cpu().numpy(), byte)
    kv = ref.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
    for got, x in zip((K2, V2), kv):
        assert torch.equal(got.cpu(), torch.from_numpy(x).to(tdtype(dtype)))
    a, a_bound = ref.attention(g.array("nbr_ptr"), g.array("nbr_idx"), g.array("nbr_rel"), range(n), to_np(Q), *kv, bias.cpu().numpy(), HALF_STEP[dtype])
    assert (np.abs(to_np(A) - a) <= a_bound).all()
    # the gates of a level as they come, by their numbers: the same store, the same rows
    for lo, hi in ((0, 40), (40, n)):
        ids = torch.from_numpy(rng.permutation(np.arange(lo, hi)).astype(np.int32)).cuda()
        at = ids.long()
        q, k, v = (torch.zeros((hi - lo, hidden), dtype=S.dtype, device="cuda") for _ in range(3))
        dg4.dg4_qkv_proj_lora(cfg, packed, S[at].contiguous(), adapter[at].contiguous(), q, k, v)
        before = codes.clone()
        dg4.dg4_kv8_write(cfg, fmt, k, v, codes, scales, ids=ids)
        assert torch.equal(before, codes) and torch.equal(q, Q[at])
        b = torch.zeros_like(q)
        dg4.dg4_sparse_attn_kv8_fwd(cfg, fmt, g, q, codes, scales, bias, b, ids=ids)
        assert torch.equal(b, A[at])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for step in range(4):
        S.copy_(rows_of(20 + step, n, hidden, dtype))
        adapter.copy_(adapter.roll(17))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in every]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, every)), step


def test_two_graphs_and_a_stream_share_the_packed_weights():
    cfg = dg4.LayerConfig(256, 8, 2, 1, "bf16")
    packed = dg4.dg4_lora_pack(cfg, *weights(1, 256, 4, 16, "bf16"))
    cases = [(rows_of(s, rows, 256, "bf16"), arrangement("any", rows, 4, np.random.default_rng(s))) for s, rows in ((1, 300), (2, 9000))]
    want = [project(cfg, packed, *c) for c in cases]
    outs = [[torch.zeros_like(c[0]) for _ in range(3)] for c in cases]
    graphs = []
    for c, out in zip(cases, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            dg4.dg4_qkv_proj_lora(cfg, packed, *c, *out)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for out in outs:
            for t in out:
                t.zero_()
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = project(cfg, packed, *cases[0])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for got, w in zip(outs, want) for x, y in zip(got, w))
        assert all(torch.equal(x, y) for x, y in zip(eager, want[0]))


def test_binding_checks():
    d, n, rank, rows = 128, 3, 8, 10
    cfg = dg4.LayerConfig(d, 4, 2, 1, "bf16")
    W, down, up, gain = weights(1, d, n, rank, "bf16")
    for args in ((W[:, :300], down, up, gain), (W.float(), down, up, gain), (W, down, None, gain), (W, down, up[:2], gain), (W, down.float(), up, gain),
                 (W, down, up, gain[:2]), (W, down, up, gain.double()), (W, down.cpu(), up, gain), (W, down.transpose(1, 2), up, gain),
                 (W.t(), down, up, gain), (W.t().contiguous(), down, up, gain), (W.flatten(), down, up, gain),
                 (W, torch.zeros((n, d, 65), dtype=W.dtype, device="cuda"), torch.zeros((n, 65, 3 * d), dtype=W.dtype, device="cuda"), gain)):
        with pytest.raises(dg4.DG4Error):
            dg4.dg4_lora_pack(cfg, *args)
    packed = dg4.dg4_lora_pack(cfg, W, down, up, gain)
    S, ad = rows_of(1, rows, d, "bf16"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    out = [torch.full_like(S, 7.0) for _ in range(3)]
    for args, kw in (((S.float(), ad, *out), {}), ((S, ad.long(), *out), {}), ((S, ad[:9], *out), {}), ((S, ad, out[0][:9], *out[1:]), {}),
                     ((S, ad, *out), dict(row_end=11)), ((S, ad, *out), dict(row_begin=-1)), ((S, ad, *out), dict(row_begin=5, row_end=4)),
                     ((S.cpu(), ad, *out), {}), ((S, ad.cpu(), *out), {})):
        with pytest.raises(dg4.DG4Error):
            dg4.dg4_qkv_proj_lora(cfg, packed, *args, **kw)
    with pytest.raises(dg4.DG4Error):
        dg4.dg4_qkv_proj_lora(dg4.LayerConfig(d, 4, 2, 1, "f32"), packed, S.float(), ad, *(t.float() for t in out))
    dg4.dg4_qkv_proj_lora(cfg, packed, S[:0], ad[:0], *(t[:0] for t in out))
    dg4.dg4_qkv_proj_lora(cfg, packed, S, ad, *out, row_begin=6, row_end=6)
    torch.cuda.synchronize()
    assert all((t == 7.0).all() for t in out)
