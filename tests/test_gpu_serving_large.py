"""Serving calls over arrays past 2 and 4 GiB: every form of the attention's addressing, rows of the store and of the projection."""
import numpy as np
import pytest
import torch

import kv8_ref as ref
import paper_2502_01681_amd as dg4
from gpu_utils import tdtype, to_np
from test_gpu_kv8 import HALF_STEP, cfg
from test_gpu_lora import weights

pytestmark = pytest.mark.gpu


def small_circuit(m, seed):
    """Edges of m gates, most with two fanins among those before."""
    rng = np.random.default_rng(seed)
    src, dst, inv = [], [], []
    for v in range(4, m):
        for u in rng.choice(np.arange(max(0, v - 12), v), 2, replace=False):
            src.append(u); dst.append(v); inv.append(int(rng.integers(0, 2)))
    return np.array(src), np.array(dst), np.array(inv, dtype=np.uint8)


# n rows of the store: offsets above 2^31 in the form that buffer addressing reaches (up to 3 GiB of codes), and past that form
@pytest.mark.parametrize("hidden,n,hops,dtype,fmt", [
    (256, 5_600_000, 2, "bf16", "e4m3"), (256, 5_600_000, 3, "f32", "int8"), (128, 11_200_000, 4, "bf16", "e4m3"),
    (256, 8_700_000, 3, "bf16", "e4m3"), (256, 8_700_000, 4, "f32", "int8"), (128, 17_400_000, 2, "f32", "e4m3"), (128, 17_400_000, 3, "bf16", "int8"),
    (128, 17_400_000, 4, "bf16", "e4m3")])
def test_attention_over_a_large_store(hidden, n, hops, dtype, fmt):
    """A circuit whose gates lie on both sides of every power of two of bytes; all other rows of the store are NaN."""
    row = 2 * hidden
    marks = [b // row for b in (2 ** 31, 0xC0000000, 2 ** 32) if b // row + 8 < n]
    places = np.unique(np.concatenate([[0, 1, 7, 100], [x + d for x in marks for d in (-3, -2, -1, 0, 1, 2)], np.linspace(1000, n - 40, 48), n - 1 - np.arange(6)]).astype(np.int64))
    m = len(places)
    print(f"kv8 attention over {n} rows of {row} bytes, {fmt} {dtype} hops={hops}, {m} gates in use", flush=True)
    src, dst, inv = small_circuit(m, hops)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(t).cuda()
    g = dg4.dg4_build_levels_device(n, dev(places[src], torch.int32), dev(places[dst], torch.int32), dev(inv, torch.uint8), hops)
    local = dg4.dg4_build_levels(m, src, dst, inv, hops)
    assert np.diff(local.array("nbr_ptr")).max() > {2: 4, 3: 8, 4: 16}[hops]
    codes = torch.full((n, row), 0x7F if fmt == "e4m3" else 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((n, hidden // 32, 2), 255, dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda: torch.randn((m, hidden), generator=gen, device="cuda").to(tdtype(dtype))
    K, V, Q = rnd(), rnd(), rnd()
    ids = dev(places, torch.int32)
    dg4.dg4_kv8_write(cfg(hidden, dtype), fmt, K, V, codes, scales, ids=ids)
    bias = torch.randn((hidden // 32, 4), generator=gen, device="cuda")
    bias[0, 2] = bias[1, 3] = bias[2, 0] = -np.inf
    bias[3] = -np.inf
    A = torch.full_like(Q, 7.0)
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q, codes, scales, bias, A, ids=ids)
    kv = ref.values(codes[ids.long()].cpu().numpy(), scales[ids.long()].cpu().numpy(), fmt)
    want, bound = ref.attention(local.array("nbr_ptr"), local.array("nbr_idx"), local.array("nbr_rel"), range(m), to_np(Q), *kv, bias.cpu().numpy(), HALF_STEP[dtype])
    err = np.abs(to_np(A) - want)
    assert (err <= bound).all(), (err / bound).max()
    # one of the other rows is what the store holds for it: NaN, and a gate by itself
    lone = torch.tensor([int(places[10]) + 5], dtype=torch.int32, device="cuda")
    B = torch.zeros((1, hidden), dtype=Q.dtype, device="cuda")
    dg4.dg4_sparse_attn_kv8_fwd(cfg(hidden, dtype, hops), fmt, g, Q[:1].contiguous(), codes, scales, torch.zeros_like(bias), B, ids=lone)
    assert B.isnan().all()


@pytest.mark.parametrize("hidden,dtype", [(256, "bf16"), (128, "f32")])
def test_rows_past_four_gigabytes(hidden, dtype):
    """S, K and V of 4.4 GB each, through the projection, into a store and back: rows on both sides of every mark against calls of
    those rows alone (a row's result depends on nothing else), and every row against its own values in the store."""
    rows = 8_600_000
    print(f"{rows} rows of {hidden} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    S = torch.empty((rows, hidden), dtype=tdtype(dtype), device="cuda").normal_(generator=gen)
    adapter = (torch.arange(rows, device="cuda") // 70_000 % 5 - 1).to(torch.int32)
    c = cfg(hidden, dtype)
    packed = dg4.dg4_lora_pack(c, *weights(1, hidden, 4, 16, dtype))
    out = [torch.zeros_like(S) for _ in range(3)]
    dg4.dg4_qkv_proj_lora(c, packed, S, adapter, *out)
    mark = [2 ** 31 // (hidden * S.element_size()), 2 ** 32 // (hidden * S.element_size())]
    some = torch.cat([torch.arange(300), *(torch.arange(x - 150, x + 150) for x in mark), torch.arange(rows - 300, rows),
                      torch.randint(0, rows, (3000,), generator=torch.Generator().manual_seed(2))]).cuda()
    few = [torch.zeros((len(some), hidden), dtype=S.dtype, device="cuda") for _ in range(3)]
    dg4.dg4_qkv_proj_lora(c, packed, S[some].contiguous(), adapter[some].contiguous(), *few)
    assert all(torch.equal(x[some], y) for x, y in zip(out, few))
    assert all(bool(x[lo:lo + 1_000_000].ne(0).any(1).all()) for x in out for lo in range(0, rows, 1_000_000))
    _, K, V = out
    codes = torch.zeros((rows, 2 * hidden), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((rows, hidden // 32, 2), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(c, "int8", K, V, codes, scales)
    code, byte = torch.zeros((len(some), 2 * hidden), dtype=torch.uint8, device="cuda"), torch.zeros((len(some), hidden // 32, 2), dtype=torch.uint8, device="cuda")
    dg4.dg4_kv8_write(c, "int8", few[1], few[2], code, byte)
    assert torch.equal(codes[some], code) and torch.equal(scales[some], byte)
    del S, out[0]
    back = [torch.zeros_like(K) for _ in range(2)]
    dg4.dg4_kv8_read(c, "int8", codes, scales, *back)
    for x, part in zip(back, (0, 1)):
        for lo in range(0, rows, 500_000):
            at = slice(lo, min(rows, lo + 500_000))
            value = codes[at, part * hidden:(part + 1) * hidden].view(torch.int8).float().unflatten(1, (-1, 32)) * torch.exp2(scales[at, :, part].float() - 127)[..., None]
            assert torch.equal(x[at], value.flatten(1).to(x.dtype))
