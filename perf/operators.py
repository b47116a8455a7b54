"""Operators of the serving path: the K|V store in 8 bits (written, read back, attended over) and the Q|K|V projection with
low-rank adapters. `op` of a case says which:
  write  dg4_kv8_write: K and V rows quantised into the store, by row or by a list of gates
  read   dg4_kv8_read: rows of the store back in the working type
  attn   dg4_sparse_attn_kv8_fwd: attention over cone rows that reads the store
  proj   dg4_qkv_proj_lora: shared projection plus the adapter of each row's circuit
`run` computes them with elementary torch operations in 32 bits or, where `own` is true, through the framework's entry points.
`exact` computes them in 64 bits from the definitions. Circuits, features and weights are drawn from the seed, on the GPU.
"""
from __future__ import annotations

import math

import torch

own = False

HEAD = 32
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# largest code of a format: a block's scale is the smallest power of two with which its largest magnitude stays within this
LARGEST = {"e4m3": 448.0, "int8": 127.0}
# neighbour entries of a gate on the circuits drawn here (mean), by cone depth
ENTRIES = {1: 2.9, 2: 6.3, 3: 12.6, 4: 23.0, 5: 41.0, 6: 70.0, 7: 115.0, 8: 190.0}


def _case(name, **c):
    if name:
        c["name"] = name
    return c


def _store(name, op, n, rows, listed_rows, fmt, dtype, hidden):
    """rows of K|V go to (come from) a store of n gates: gates 0 .. rows-1, or `rows` listed gates in any order."""
    return _case(name, op=op, n=n, rows=rows, listed=listed_rows, fmt=fmt, dtype=dtype, hidden=hidden)


def _attn(name, n, rows, listed_rows, fmt, dtype, hidden, hops, window):
    """a circuit of n gates whose fanins lie mostly within `window` ids; all its gates attend, or `rows` of them."""
    return _case(name, op="attn", n=n, rows=rows, listed=listed_rows, fmt=fmt, dtype=dtype, hidden=hidden, hops=hops, window=window)


def _proj(name, rows, circuits, adapters, rank, dtype, hidden):
    """rows of `circuits` circuits of uneven size, one after the other, each with one of the adapters or none."""
    return _case(name, op="proj", rows=rows, circuits=circuits, adapters=adapters, rank=rank, dtype=dtype, hidden=hidden)


def listed():
    return [
        # the gates of one level of a deep circuit (201,024 gates, 760 levels) as the sweep finishes them: latency
        _store("write_level_bf16", "write", 201_024, 264, True, "e4m3", "bf16", 256),
        # an ordinary circuit whole, full precision, an odd number of rows
        _store("write_circuit_f32", "write", 20_257, 20_257, False, "int8", "f32", 128),
        # a million gates: bandwidth
        _store("write_large_bf16", "write", 1_004_096, 1_004_096, False, "e4m3", "bf16", 256),
        # the distinct sources of a level, back into rows for the projections that want them
        _store("read_frontier_bf16", "read", 201_024, 4_133, True, "int8", "bf16", 256),
        # a whole store back in full precision (a checkpoint of the embeddings, a check)
        _store("read_large_f32", "read", 402_193, 402_193, False, "e4m3", "f32", 256),
        # one gate asked for by itself
        _attn("attn_gate_f32", 1_032, 1, True, "int8", "f32", 128, 2, 64),
        # an ordinary circuit (ITC99 / EPFL size) in full precision
        _attn("attn_circuit_f32", 20_256, 20_256, False, "int8", "f32", 128, 2, 512),
        # a million gates, two-hop cones: the gather's throughput
        _attn("attn_large_bf16", 1_004_096, 1_004_096, False, "e4m3", "bf16", 256, 2, 1_024),
        # the paper's cone depth on its average ITC99 circuit (15,135 gates): rows of up to 511 sources
        _attn("attn_deep_bf16", 15_135, 15_135, False, "e4m3", "bf16", 128, 8, 1_300),
        # one row each of 64 requests, every one with its own adapter: latency, nothing shared but the projection
        _proj("proj_requests_bf16", 64, 64, 64, 16, "bf16", 256),
        # a batch of small circuits in full precision, odd sizes, some without an adapter
        _proj("proj_circuits_f32", 20_257, 23, 8, 8, "f32", 128),
        # a million gates of forty circuits: the projection of a large batch
        _proj("proj_large_bf16", 1_004_096, 40, 16, 16, "bf16", 256),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["write", "read", "attn", "attn", "proj", "proj"])
    dtype, hidden, fmt = rng.choice(["f32", "bf16"]), rng.choice([128, 256]), rng.choice(["e4m3", "int8"])
    if op in ("write", "read"):
        listed_rows = rng.random() < 0.5
        n = size(1, 900_000 if dtype == "bf16" else 400_000)
        return _store("", op, n, size(1, n) if listed_rows else n, listed_rows, fmt, dtype, hidden)
    if op == "attn":
        hops = rng.choice([1, 2, 2, 3, 3, 4, 5, 6, 7, 8])
        most = 600_000 if hops <= 2 else 200_000 if hops == 3 else 12_000 * 2 ** (8 - hops) // 2
        listed_rows = rng.random() < 0.4
        n = size(100, most)
        return _attn("", n, size(1, n) if listed_rows else n, listed_rows, fmt, dtype, hidden, hops, size(32, 4_096))
    rows = size(1, 700_000 if dtype == "bf16" else 150_000)
    rank = rng.choice([1, 4, 8, 8, 12, 16, 16, 27, 32, 64])
    adapters = min(size(1, 128), max(1, 1024 // rank))
    return _proj("", rows, min(rows, size(1, 200)), adapters, rank, dtype, hidden)


# ---------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(DTYPES[dtype])


def _kv(gen, rows, hidden, dtype):
    """K and V rows whose heads differ in size from gate to gate, as projections of LayerNorm outputs do."""
    heads = hidden // HEAD
    def one():
        size = torch.exp(0.5 * torch.randn((rows, heads, 1), generator=gen, device="cuda"))
        return (torch.randn((rows, heads, HEAD), generator=gen, device="cuda") * size).reshape(rows, hidden).to(DTYPES[dtype])
    return one(), one()


def _listed(gen, n, rows):
    return torch.randperm(n, generator=gen, device="cuda")[:rows].to(torch.int32)


def _circuit(gen, n, window):
    """Fanins of every gate (-1: none) and their inverter marks: primary inputs first, then AND gates with two distinct
    earlier fanins, four in five within the window, every tenth gate an inverter or buffer with one."""
    pi = max(2, min(n, n // 64 + 2))
    v = torch.arange(pi, n, device="cuda")
    rand = lambda: torch.rand(n - pi, generator=gen, device="cuda", dtype=torch.float64)
    near = torch.clamp(v - window, min=0)

    def fanin():
        first = torch.where(rand() < 0.8, near, torch.zeros_like(near))
        return first + (rand() * (v - first)).long()
    a, b = fanin(), fanin()
    b = torch.where(a == b, torch.where(a > 0, a - 1, a + 1), b)
    b = torch.where(rand() < 0.1, torch.full_like(b, -1), b)
    fan = torch.full((n, 2), -1, dtype=torch.int64, device="cuda")
    fan[pi:, 0], fan[pi:, 1] = a, b
    inv = torch.randint(0, 2, (n, 2), generator=gen, device="cuda")
    return fan, inv


def _cones(fan, inv, hops, gates):
    """Neighbour rows of `gates`: distinct sources within `hops` steps (-1: padding), each with the relation of its shortest
    path (0 itself, 1 fanin, 2 inverted fanin, 3 further up)."""
    none = 1 << 40
    ids, rel = [gates[:, None]], [torch.zeros_like(gates)[:, None]]
    for hop in range(1, hops + 1):
        at = ids[-1]
        nxt = torch.where((at >= 0)[..., None], fan[at.clamp(min=0)], -1)
        r = 1 + inv[at.clamp(min=0)] if hop == 1 else torch.full_like(nxt, 3)
        ids.append(nxt.flatten(1))
        rel.append(r.flatten(1))
    ids, rel = torch.cat(ids, 1), torch.cat(rel, 1)
    key = torch.where(ids >= 0, ids * 4 + rel, none).sort(dim=1).values
    again = torch.zeros_like(key, dtype=torch.bool)
    again[:, 1:] = key[:, 1:] >> 2 == key[:, :-1] >> 2
    key = torch.where(again, none, key)
    return torch.where(key < none, key >> 2, -1), torch.where(key < none, key & 3, 0)


def prepare(case, seed):
    gen = _gen(seed)
    s = dict(case)
    hidden, dtype = case["hidden"], case["dtype"]
    heads = hidden // HEAD
    if case["op"] == "proj":
        rows, circuits = case["rows"], case["circuits"]
        cuts = torch.rand(circuits, generator=gen, device="cuda") + 0.05
        start = torch.cat([torch.zeros(1, device="cuda"), (cuts.cumsum(0) / cuts.sum())[:-1]])
        # (a first row for every circuit, the other rows by the cuts)
        first = torch.maximum((start.double() * rows).long(), torch.arange(circuits, device="cuda"))
        of = torch.searchsorted(first.cummax(0).values, torch.arange(rows, device="cuda"), right=True) - 1
        # every adapter in turn; every sixteenth circuit has none
        which = torch.randperm(circuits, generator=gen, device="cuda")
        which = torch.where(which % 16 == 15, -1, which % case["adapters"])
        s["adapter"] = which[of].to(torch.int32)
        s["S"] = _normal(gen, (rows, hidden), dtype)
        s["W"] = _normal(gen, (hidden, 3 * hidden), dtype, hidden ** -0.5)
        s["down"] = _normal(gen, (case["adapters"], hidden, case["rank"]), dtype, hidden ** -0.5)
        s["up"] = _normal(gen, (case["adapters"], case["rank"], 3 * hidden), dtype, case["rank"] ** -0.5)
        s["gain"] = 0.25 + torch.rand(case["adapters"], generator=gen, device="cuda")
        s["out"] = [torch.zeros((rows, hidden), dtype=DTYPES[dtype], device="cuda") for _ in range(3)]
    else:
        n, rows = case["n"], case["rows"]
        s["ids"] = _listed(gen, n, rows) if case["listed"] else None
        s["codes"] = torch.zeros((n, 2 * hidden), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.zeros((n, heads, 2), dtype=torch.uint8, device="cuda")
        if case["op"] == "write":
            s["K"], s["V"] = _kv(gen, rows, hidden, dtype)
        else:
            K, V = _kv(gen, n, hidden, dtype)
            s["codes"], s["scales"] = _quantise(torch.cat([K, V], 1), case["fmt"])
            s["out"] = [torch.zeros((rows, hidden), dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
        if case["op"] == "attn":
            fan, inv = _circuit(gen, n, case["window"])
            gates = torch.arange(n, device="cuda") if s["ids"] is None else s["ids"].long()
            s["nbr"], s["rel"] = _cones(fan, inv, case["hops"], gates)
            s["fan"], s["inv"] = fan, inv
            s["Q"] = _normal(gen, (rows, hidden), dtype)
            s["bias"] = torch.randn((heads, 4), generator=gen, device="cuda")
    if own:
        import paper_2502_01681_amd as dg4
        s["cfg"] = dg4.LayerConfig(hidden, heads, case.get("hops", 2), 1, dtype)
        if case["op"] == "proj":     # weights laid out once, as a server keeps them
            s["packed"] = dg4.dg4_lora_pack(s["cfg"], s["W"], s["down"], s["up"], s["gain"])
        if case["op"] == "attn":     # the circuit's analysis, kept for all its layers
            have = s["fan"] >= 0
            dst = torch.arange(case["n"], device="cuda")[:, None].expand(-1, 2)
            s["graph"] = dg4.dg4_build_levels_device(case["n"], s["fan"][have].to(torch.int32), dst[have].to(torch.int32),
                                                     s["inv"][have].to(torch.uint8), case["hops"])
            s["graph"].upload()
    return s


# ----------------------------------------------------------------------------------------- plain forms

def _quantise(x, fmt):
    """Codes and scale bytes ([rows, heads, 2]) of K | V rows: blocks of 32 values, code = round(x / 2^e) (to nearest, ties to even) with the smallest
    e that keeps the block within the format, byte = e + 127. Everything but that rounding is exact."""
    x = x.float().unflatten(1, (-1, HEAD))
    top = x.abs().amax(2)
    m, e = torch.frexp(top.double())                   # top = m 2^e, m in [0.5, 1)
    mm, me = math.frexp(LARGEST[fmt])
    e = torch.where(m > mm, e - me + 1, e - me)
    byte = torch.where(top > 0, (e + 127).clamp(0, 254), 0)
    y = x * torch.exp2((127 - byte).double()).float()[..., None]
    codes = y.to(torch.float8_e4m3fn) if fmt == "e4m3" else y.round().to(torch.int8)
    return codes.view(torch.uint8).flatten(1), byte.to(torch.uint8).unflatten(1, (2, -1)).transpose(1, 2).contiguous()


def _values(codes, scales, fmt):
    """What the K or V parts of rows stand for, in 32 bits."""
    c = (codes.view(torch.float8_e4m3fn) if fmt == "e4m3" else codes.view(torch.int8)).float()
    return (c.unflatten(-1, (-1, HEAD)) * scales.view(torch.float8_e8m0fnu).float()[..., None]).flatten(-2)


def _plain(s):
    if s["op"] == "write":
        codes, scales = _quantise(torch.cat([s["K"], s["V"]], 1), s["fmt"])
        at = slice(0, s["rows"]) if s["ids"] is None else s["ids"].long()
        s["codes"][at] = codes
        s["scales"][at] = scales
        return _stored(s)
    dtype, hidden = DTYPES[s["dtype"]], s["hidden"]
    if s["op"] == "read":
        at = slice(0, s["rows"]) if s["ids"] is None else s["ids"].long()
        return {"K": _values(s["codes"][at, :hidden], s["scales"][at, :, 0], s["fmt"]).to(dtype),
                "V": _values(s["codes"][at, hidden:], s["scales"][at, :, 1], s["fmt"]).to(dtype)}
    if s["op"] == "attn":
        heads = hidden // HEAD
        nbr = s["nbr"].clamp(min=0)
        k = _values(s["codes"][:, :hidden][nbr], s["scales"][..., 0][nbr], s["fmt"]).unflatten(2, (heads, HEAD))
        score = (k * s["Q"].float().view(-1, 1, heads, HEAD)).sum(3) * HEAD ** -0.5 + s["bias"].t()[s["rel"]]
        del k
        score = torch.where((s["nbr"] >= 0)[..., None], score, -math.inf)
        p = torch.exp(score - score.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        v = _values(s["codes"][:, hidden:][nbr], s["scales"][..., 1][nbr], s["fmt"]).unflatten(2, (heads, HEAD))
        return {"A": (p[..., None] * v).sum(1).flatten(1).to(dtype)}
    x = s["S"].float()
    mine = s["adapter"][:, None] == torch.arange(s["adapters"], device="cuda", dtype=torch.int32)
    low = (x @ s["down"].float().permute(1, 0, 2).flatten(1)).unflatten(1, (s["adapters"], s["rank"]))
    low = low * torch.where(mine, s["gain"], torch.zeros_like(s["gain"]))[..., None]
    y = x @ s["W"].float() + low.flatten(1) @ s["up"].float().flatten(0, 1)
    return {"Q": y[:, :hidden].to(dtype), "K": y[:, hidden:2 * hidden].to(dtype), "V": y[:, 2 * hidden:].to(dtype)}


def _stored(s):
    """The store as the values that its bytes stand for."""
    return {"codes": s["codes"].view(torch.float8_e4m3fn if s["fmt"] == "e4m3" else torch.int8),
            "scales": s["scales"].view(torch.float8_e8m0fnu)}


def run(s):
    if not own:
        return _plain(s)
    import paper_2502_01681_amd as dg4
    if s["op"] == "write":
        dg4.dg4_kv8_write(s["cfg"], s["fmt"], s["K"], s["V"], s["codes"], s["scales"], ids=s["ids"])
        return _stored(s)
    if s["op"] == "read":
        dg4.dg4_kv8_read(s["cfg"], s["fmt"], s["codes"], s["scales"], *s["out"], ids=s["ids"])
        return {"K": s["out"][0], "V": s["out"][1]}
    if s["op"] == "attn":
        dg4.dg4_sparse_attn_kv8_fwd(s["cfg"], s["fmt"], s["graph"], s["Q"], s["codes"], s["scales"], s["bias"], s["out"][0],
                                    ids=s["ids"])
        return {"A": s["out"][0]}
    dg4.dg4_qkv_proj_lora(s["cfg"], s["packed"], s["S"], s["adapter"], *s["out"])
    return dict(zip("QKV", s["out"]))


# ------------------------------------------------------------------------------------------------ work

def work(case):
    es, d = (4 if case["dtype"] == "f32" else 2), case["hidden"]
    if case["op"] == "proj":
        used = min(case["adapters"], case["circuits"])
        return {"bytes": case["rows"] * (4 * d * es + 4) + 3 * d * d * es + used * case["rank"] * 4 * d * es,
                "flops": 2 * case["rows"] * d * (3 * d + 4 * case["rank"])}
    stored = 2 * d + 2 * (d // HEAD)
    rows, index = case["rows"], 4 if case["listed"] else 0
    if case["op"] in ("write", "read"):
        return {"bytes": rows * (2 * d * es + stored + index), "flops": rows * 4 * d}
    entries = ENTRIES[case["hops"]]
    return {"bytes": rows * (2 * d * es + 4 * entries + index) + min(case["n"], rows * entries) * stored,
            "flops": rows * entries * 4 * d}


# --------------------------------------------------------------------------------------------- 64 bits

def _exact_write(s):
    """Nearest codes by the spacing of the format at each value, in 64 bits."""
    fmt, d = s["fmt"], s["hidden"]
    codes = torch.zeros(s["codes"].shape, dtype=torch.float64, device="cuda")
    scales = torch.full(s["scales"].shape, 2.0 ** -127, dtype=torch.float64, device="cuda")
    for part, x in enumerate((s["K"], s["V"])):
        x = x.double().view(x.shape[0], -1, HEAD)
        top = x.abs().max(dim=2).values
        least = torch.full_like(top, 2.0 ** -127)
        # at most one step of the estimate is missing or too many
        scale = torch.maximum(torch.exp2(torch.floor(torch.log2(torch.clamp(top, min=1e-300) / LARGEST[fmt]))), least)
        for _ in range(2):
            scale = torch.where(top > LARGEST[fmt] * scale, scale * 2, scale)
            scale = torch.where((top <= LARGEST[fmt] * scale / 2) & (scale > least), scale / 2, scale)
        y = x / scale[..., None]
        if fmt == "e4m3":
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
            y = torch.round(y / step) * step
        else:
            y = torch.round(y)
        at = torch.arange(s["rows"], device="cuda") if s["ids"] is None else s["ids"].long()
        codes[at, part * d:(part + 1) * d] = y.flatten(1)
        scales[at, :, part] = scale
    return {"codes": codes, "scales": scales}


def _exact_values(s, part, rows):
    d, heads = s["hidden"], s["hidden"] // HEAD
    c = s["codes"][rows, part * d:(part + 1) * d].long()
    if s["fmt"] == "int8":
        v = torch.where(c < 128, c, c - 256).double()
    else:
        e, m = (c >> 3) & 15, (c & 7).double()
        v = torch.where(e > 0, (8 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9) * torch.where(c < 128, 1.0, -1.0)
    size = torch.exp2(s["scales"][rows, :, part].double() - 127)
    return v.view(-1, heads, HEAD) * size[..., None]


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    if s["op"] == "write":
        return _exact_write(s)
    if s["op"] == "read":
        rows = torch.arange(s["rows"], device="cuda") if s["ids"] is None else s["ids"].long()
        return {"K": _exact_values(s, 0, rows).flatten(1), "V": _exact_values(s, 1, rows).flatten(1)}
    if s["op"] == "attn":
        # by edges, a run of destinations at a time: sums over the edges of a destination
        d, heads = s["hidden"], s["hidden"] // HEAD
        out = torch.empty((s["rows"], d), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 21) // s["nbr"].shape[1])
        for r0 in range(0, s["rows"], step):
            nbr, rel = s["nbr"][r0:r0 + step], s["rel"][r0:r0 + step]
            dst, col = torch.nonzero(nbr >= 0, as_tuple=True)
            src, code = nbr[dst, col], rel[dst, col]
            q = s["Q"][r0:r0 + step].double().view(-1, heads, HEAD)[dst]
            w = torch.exp((q * _exact_values(s, 0, src)).sum(2) / math.sqrt(HEAD) + s["bias"].double()[:, code].t())
            total = torch.zeros((nbr.shape[0], heads), dtype=torch.float64, device="cuda").index_add_(0, dst, w)
            acc = torch.zeros((nbr.shape[0], heads, HEAD), dtype=torch.float64, device="cuda")
            acc.index_add_(0, dst, w[..., None] * _exact_values(s, 1, src))
            out[r0:r0 + step] = (acc / total[..., None]).flatten(1)
        return {"A": out}
    d = s["hidden"]
    y = s["S"].double() @ s["W"].double()
    order = torch.argsort(s["adapter"].long(), stable=True)
    name, count = torch.unique_consecutive(s["adapter"][order], return_counts=True)
    for a, rows in zip(name.tolist(), order.split(count.tolist())):
        if a >= 0:
            y[rows] += s["gain"][a].double() * (s["S"][rows].double() @ (s["down"][a].double() @ s["up"][a].double()))
    return {"Q": y[:, :d], "K": y[:, d:2 * d], "V": y[:, 2 * d:]}
