"""The projection with low-rank adapters where weights or what they make of a row are not finite, or at the end of the range."""
import numpy as np
import pytest
import torch

import paper_2502_01681_amd as dg4
from gpu_utils import tdtype
from test_gpu_lora import project, rows_of, weights

pytestmark = pytest.mark.gpu

# (hidden, dtype, rows): few rows, and many (a kernel of its own in bfloat16)
SIZES = [(128, "f32", 70), (128, "f32", 16_500), (256, "f32", 300), (128, "bf16", 70), (128, "bf16", 16_500), (256, "bf16", 70), (256, "bf16", 8_300)]


def exact(S, adapter, W, down, up, gain):
    """Q|K|V in 64 bits on the host. (A product there is what the definition says: T = 0 times an infinity is NaN.)"""
    S, W, down, up, gain = (t.double().cpu() for t in (S, W, down, up, gain))
    y, adapter = S @ W, adapter.cpu()
    for a in range(down.shape[0]):
        r = torch.nonzero(adapter == a).flatten()
        if len(r):
            t = gain[a] * (S[r] @ down[a])
            y[r] += torch.stack([t[:, q:q + 1] * up[a][q] for q in range(t.shape[1])]).sum(0)
    return y


@pytest.mark.parametrize("hidden,dtype,rows", SIZES)
@pytest.mark.parametrize("rank,at", [(3, 1), (8, 7), (16, 11), (27, 25), (64, 40)])
@pytest.mark.parametrize("mixed", [False, True])
def test_weights_that_are_not_finite(hidden, dtype, rows, rank, at, mixed):
    """Row `at` of Up_0 and Up_2 has infinities of either sign and a NaN; S Down times the gain is a number there that bfloat16
    holds (1, -2), or that it rounds up or down (0.3, 0.7), or zero."""
    n = 4
    print(f"lora infinite Up {dtype} {hidden} rank={rank} rows={rows} mixed={mixed}", flush=True)
    cfg = dg4.LayerConfig(hidden, hidden // 32, 2, 1, dtype)
    W, down, up, gain = weights(3, hidden, n, rank, dtype)
    gain[0], gain[2] = 0.3, 0.7
    S = rows_of(4, rows, hidden, dtype)
    down[:, :, at] = 0
    down[:, 0, at] = 1
    # (no other product is NaN or infinite: T at `at` is gain * S[:, 0])
    S[:, 0] = torch.tensor([1.0, -2.0, 1.25, 0.0, -1.0], dtype=S.dtype, device="cuda")[torch.arange(rows, device="cuda") % 5]
    for a in (0, 2):
        up[a, at, 3::7] = float("inf")
        up[a, at, 5::11] = float("-inf")
        up[a, at, 9] = float("nan")
    adapter = torch.arange(rows, device="cuda") % n if mixed else torch.arange(rows, device="cuda") * n // rows
    adapter = torch.where(torch.arange(rows, device="cuda") % 13 == 5, -1, adapter) if mixed else adapter
    adapter = adapter.to(torch.int32)
    got = torch.cat(project(cfg, dg4.dg4_lora_pack(cfg, W, down, up, gain), S, adapter), 1).double().cpu()
    want = exact(S, adapter, W, down, up, gain)
    assert int(want.isnan().sum()) and int((want == np.inf).sum()) and int((want == -np.inf).sum())
    assert torch.equal(got.isnan(), want.isnan())
    for x in (np.inf, -np.inf):
        assert torch.equal(got == x, want == x)
    # everything else is as good as with weights that are finite: a column's infinity reaches no other column and no other adapter
    ok = want.isfinite()
    s, w = S.double().cpu(), W.double().cpu()
    size = (hidden + 8) * (s.abs() @ w.abs())
    for a in range(n):
        r = torch.nonzero(adapter.cpu() == a).flatten()
        t = s[r] @ down[a].double().cpu()
        u = torch.nan_to_num(up[a].double().cpu(), 0, 0, 0).abs()
        g = float(gain[a])
        size[r] += g * (hidden + rank + 12) * ((s[r].abs() @ down[a].double().cpu().abs()) @ u)
        if dtype == "bf16":
            size[r] += g * 2.0 ** 7 * (t.abs() @ u)
    bound = size * 2.0 ** -23 + (2.0 ** -24 if dtype == "f32" else 2.0 ** -8) * want.abs() + 1e-37
    assert ((got - want).abs() <= bound)[ok].all()


@pytest.mark.parametrize("hidden,dtype,rows", SIZES)
def test_products_at_the_end_of_the_range(hidden, dtype, rows):
    """S Down times the gain is a float that rounds to an infinity of bfloat16 (3.3962e38 and more), the results are ordinary."""
    print(f"lora products of 3.4e38 {dtype} {hidden} rows={rows}", flush=True)
    cfg = dg4.LayerConfig(hidden, hidden // 32, 2, 1, dtype)
    W, down, up, gain = weights(3, hidden, 1, 8, dtype)
    S, down, up = torch.zeros((rows, hidden), dtype=W.dtype, device="cuda"), torch.zeros_like(down), up * 2.0 ** -120
    S[:, 0] = torch.where(torch.arange(rows, device="cuda") % 2 == 0, 1.0, -1.0).to(S.dtype)
    down[0, 0] = 1.0
    gain[0] = 3.4e38
    got = torch.cat(project(cfg, dg4.dg4_lora_pack(cfg, W, down, up, gain), S, torch.zeros(rows, dtype=torch.int32, device="cuda")), 1).double().cpu()
    want = exact(S, torch.zeros(rows, dtype=torch.int32), W, down, up, gain)
    # the sum over the ranks: eight products, each of a number off by 2^-16 (2^-23 in fp32), and the output's rounding
    size = W[0].double().abs() + float(gain[0]) * up[0].double().abs().sum(0)
    bound = (2.0 ** -16 if dtype == "bf16" else 0) * size + 2.0 ** -18 * size
    bound = bound.cpu() + (2.0 ** -24 if dtype == "f32" else 2.0 ** -8) * want.abs()
    assert ((got - want).abs() <= bound).all()


def test_threads_with_adapters_of_different_ranks():
    """Calls of the same kernel with little and with much shared memory, from two threads at once, on streams of their own."""
    import threading
    cfg = dg4.LayerConfig(256, 8, 2, 1, "bf16")
    jobs = []
    for rank in (1, 64):
        packed = dg4.dg4_lora_pack(cfg, *weights(rank, 256, 2, rank, "bf16"))
        S = rows_of(rank, 9_000, 256, "bf16")
        adapter = (torch.arange(9_000, device="cuda") // 4_500).to(torch.int32)
        jobs.append((packed, S, adapter, project(cfg, packed, S, adapter), [torch.zeros_like(S) for _ in range(3)]))
    torch.cuda.synchronize()
    failed = []

    def work(packed, S, adapter, want, out):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(200):
                    dg4.dg4_qkv_proj_lora(cfg, packed, S, adapter, *out)
                torch.cuda.current_stream().synchronize()
        except Exception as e:                     # (an assertion in a thread would be lost)
            failed.append(e)
    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    assert all(torch.equal(x, y) for job in jobs for x, y in zip(job[3], job[4]))
