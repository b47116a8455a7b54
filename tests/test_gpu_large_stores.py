"""Sweeps over circuits whose K|V store of a layer is larger than 4 GiB: against level-by-level launches, whose kernels address
sources by 64-bit pointers, and sampled gates against the oracle."""
import numpy as np
import pytest
import torch

import oracle
import paper_2502_01681_amd as dg4
from gpu_utils import TOL, row_rel_err, tdtype, to_np

pytestmark = pytest.mark.gpu


def layered(n, width, hops, seed):
    """n gates, `width` to a level: every gate reads two neighbours of a random place in the level below."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.arange(width, n, device="cuda")
    at = torch.randint(0, width - 1, v.shape, generator=gen, device="cuda")
    a = (v // width - 1) * width + at
    src = torch.stack([a, a + 1], 1).flatten().to(torch.int32)
    dst = torch.stack([v, v], 1).flatten().to(torch.int32)
    inv = torch.randint(0, 2, src.shape, generator=gen, device="cuda").to(torch.uint8)
    return dg4.dg4_build_levels_device(n, src, dst, inv, hops)


def sweeps(g, hidden, dtype, hops, layers):
    gen = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    X = rnd(g.n, hidden).to(tdtype(dtype))
    W = [((rnd(hidden, 3 * hidden) * hidden ** -0.5).to(X.dtype), (rnd(hidden, hidden) * hidden ** -0.5).to(X.dtype), rnd(hidden // 32, 4)) for _ in range(layers)]
    yield X, W
    for per_level in (False, True):
        cfg = dg4.LayerConfig(hidden, hidden // 32, hops, layers, dtype, per_level=per_level)
        H = torch.full((g.n, hidden), float("nan"), dtype=X.dtype, device="cuda")
        ws = torch.empty(dg4.dg4_layer_workspace_bytes(cfg, g), dtype=torch.uint8, device="cuda")
        ws.fill_(0xFF)
        dg4.dg4_layer_fwd(cfg, g, X, W, H, workspace=ws)
        torch.cuda.synchronize()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        dg4.dg4_layer_fwd(cfg, g, X, W, H, workspace=ws)
        end.record()
        torch.cuda.synchronize()
        dg4.dg4_layer_status(cfg, g, ws)
        print(f"  {'level by level' if per_level else 'as it goes'}: {begin.elapsed_time(end):.2f} ms", flush=True)
        del ws
        yield H


def sampled(g, X, W, H, hidden, dtype):
    """The largest relative error of some gates, the last ones among them, given the embeddings of what they read."""
    rng = np.random.default_rng(3)
    gates = np.unique(np.concatenate([np.arange(g.n - 300, g.n), rng.integers(0, g.n, 300)]))
    ptr, idx, rel = g.array("nbr_ptr"), g.array("nbr_idx"), g.array("nbr_rel")
    rows = [slice(ptr[v], ptr[v + 1]) for v in gates]
    named = np.unique(np.concatenate([idx[r] for r in rows]))                  # (every row holds its gate)
    count = np.zeros(len(named), dtype=np.int64)
    at = np.searchsorted(named, gates)
    count[at] = [r.stop - r.start for r in rows]
    none = np.zeros(0, dtype=np.int32)
    cut = oracle.Graph(len(named), none, none, np.zeros(1, dtype=np.int64), np.concatenate([[0], np.cumsum(count)]).astype(np.int64),
                       np.searchsorted(named, np.concatenate([idx[r] for r in rows])).astype(np.int32), np.concatenate([rel[r] for r in rows]), g.hops)
    pick = torch.from_numpy(named).long().cuda()
    h = to_np(H[pick])
    ref = oracle.layer_nodes(cut, to_np(X[pick]), [to_np(w[0]) for w in W], [to_np(w[1]) for w in W], [to_np(w[2]) for w in W], hidden // 32, h, at, store=dtype)
    return row_rel_err(h[at], ref).max()


def check(n, width, hidden, dtype, hops, layers):
    print(f"layered circuit {dtype} {hidden}: {n} gates, {width} to a level, hops={hops} layers={layers}", flush=True)
    g = layered(n, width, hops, 1)
    (X, W), got, want = sweeps(g, hidden, dtype, hops, layers)
    assert not got.isnan().any()
    worst = 0.0
    for lo in range(0, n, 1 << 20):                # (a part at a time: the differences of all rows would be another store)
        x, y = got[lo:lo + (1 << 20)].float(), want[lo:lo + (1 << 20)].float()
        worst = max(worst, float(((x - y).norm(dim=1) / y.norm(dim=1).clamp_min(1e-30)).max()))
    err = sampled(g, X, W, got, hidden, dtype)
    print(f"  max rel err {worst:.3e}, of sampled gates against the oracle {err:.3e}", flush=True)
    assert worst <= 2 * TOL[dtype] and err <= TOL[dtype]


@pytest.mark.parametrize("hidden,dtype,hops,layers", [(256, "bf16", 3, 2), (128, "f32", 3, 1), (256, "bf16", 4, 1)])
def test_wide_circuits(hidden, dtype, hops, layers):
    n = 4_500_000
    assert n * 2 * hidden * (4 if dtype == "f32" else 2) > 2 ** 32
    check(n, 45_000, hidden, dtype, hops, layers)


def test_a_deep_circuit():
    """Few gates to a level: heads spread over compute units, a store of 256 bytes a gate for each."""
    n = 17_000_000
    assert n * 2 * 32 * 4 > 2 ** 32
    check(n, 900, 128, "f32", 2, 1)
