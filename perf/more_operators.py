"""What stands between the layers of a serving step, as cases that can be timed and compared.

A case is one pass through an operator on inputs made from a seed:

  norm     the residual stream takes a layer's output (s = x + r, rounded to the stream's type), is normalised (RMS or LayerNorm),
           reassembled by a map where there is one, and quantized per token by Eq. (2) at 4, 6 or 8 bits for the next layer;
           besides the codes a caller may ask for the normalised rows (an adapter reads them) and for what the codes stand for
  adapter  low-rank adapters of many requests beside a shared projection: out = y + scale_a (x A_a^T) B_a^T, each request's rows with
           its own adapter a, of its own rank, or with none; fused projections (q | k | v) have an A for each part

`own` false: elementary torch operations in 32 bits (64 where row statistics and values next to a rounding border need them), one
rounding at the end.  `own` true: the framework's calls.  Widths are those of `paper_2310_08041_amd/workloads.py` (4096, 5120, 8192
channels; 28672 into a down projection, 27648 out of an up/gate projection, 12288 out of q | k | v) or generic.
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NORMS = {"none": 0, "layer": 1, "rms": 2}
EPS = 1e-5


# ---------------------------------------------------------------- cases

def _norm(name, n, c, bits, x="bf16", r="bf16", norm="rms", expand=0.0, y="none", pad=0):
    """expand: share of channels that the map splits off, as many are merged (0: no map); y: type of the normalised rows and of what
    the codes stand for ("none": only the latter, bf16); pad: elements between the rows of x and r."""
    return dict(name=name, kind="norm", n=n, c=c, bits=bits, x=x, r=r, norm=norm, expand=expand, y=y, pad=pad)


def _adapter(name, seqs, new_lo, new_hi, c, parts, pool, used, rank_lo, rank, x="bf16", w="bf16", y="bf16", without=0, tail=0):
    """parts: outputs of each part, joined by +; pool adapters of which `used` are named; every `without`-th sequence has none (0: all
    have one); tail: rows of no sequence at the end."""
    return dict(name=name, kind="adapter", seqs=seqs, new_lo=new_lo, new_hi=new_hi, c=c, parts=parts, pool=pool, used=used,
                rank_lo=rank_lo, rank=rank, x=x, w=w, y=y, without=without, tail=tail)


def listed():
    return [
        # one interactive request's token between two layers: the smallest call, latency
        _norm("norm_decode_1", 1, 4096, 8),
        # sixteen requests decoded together (the decode configuration), through a reassembly map, 6-bit codes, adapters behind it
        _norm("norm_decode_16_map", 16, 8192, 6, expand=0.01, y="bf16"),
        # prefill of one 2048-token segment, 8-bit codes, no reassembly
        _norm("norm_prefill_2048", 2048, 8192, 8),
        # prefill of two segments in front of an up/gate projection (the 13B configuration): map, 4-bit codes, a float32 stream
        _norm("norm_prefill_4096_map", 4096, 5120, 4, r="f32", expand=0.01),
        # a ragged prompt of a ragged width: LayerNorm, float32, padded rows, a map with many computed channels
        _norm("norm_ragged_777_layer", 777, 5000, 8, x="f32", r="f32", norm="layer", expand=0.05, y="f32", pad=3),
        # eight segments at once: the largest, bandwidth
        _norm("norm_prefill_16384", 16384, 8192, 8),
        # one interactive request with an adapter: the smallest call
        _adapter("adapter_decode_1", 1, 1, 1, 4096, "4096", 8, 1, 16, 16),
        # sixteen requests, each with an adapter of its own, ranks 8 to 64 (the decode configuration's projection)
        _adapter("adapter_decode_16", 16, 1, 1, 8192, "8192", 32, 16, 8, 64),
        # a large decode batch on a dozen adapters, q | k | v in one projection, some requests without an adapter
        _adapter("adapter_decode_256_qkv", 256, 1, 1, 4096, "4096+4096+4096", 16, 12, 16, 16, without=8),
        # prefill of one segment through the widest layer (70B down), float32 result of the layer
        _adapter("adapter_prefill_2048_down", 1, 2048, 2048, 28672, "8192", 4, 1, 64, 64, y="f32"),
        # prompts and single tokens in one step, float32 throughout, ragged widths, requests without an adapter, padding rows
        _adapter("adapter_mixed_f32", 12, 1, 300, 5000, "4999", 9, 5, 3, 24, x="f32", w="f32", y="f32", without=4, tail=5),
        # prefill of several prompts through an up/gate projection (the 13B configuration)
        _adapter("adapter_prefill_upgate", 5, 300, 1200, 5120, "13824+13824", 8, 4, 16, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        while True:
            n, c = _log(rng, 1, 16384), _log(rng, 128, 16384)
            if rng.random() < 0.75:
                c = max(128, c // 128 * 128)
            if n * c <= 4096 * 8192:
                break
        x, r = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
        case = _norm("", n, c, rng.choice([4, 6, 8, 8]), x, r, rng.choice(["rms", "rms", "rms", "layer", "none"]),
                     rng.choice([0.0, 0.0, 0.01, 0.01, 0.05]), rng.choice(["none", "none", "bf16", "f32"]), rng.choice([0, 0, 0, 8, 3]))
    else:
        decode = rng.random() < 0.5
        while True:
            seqs = _log(rng, 1, 256) if decode else _log(rng, 1, 8)
            new_hi = 1 if decode else _log(rng, 2, 2048 // seqs)
            c, outs = _log(rng, 256, 28672), [_log(rng, 256, 13824) for _ in range(rng.choice([1, 1, 2, 3]))]
            if rng.random() < 0.75:
                c, outs = max(256, c // 128 * 128), [max(256, o // 128 * 128) for o in outs]
            rank, pool = rng.choice([8, 16, 16, 32, 64, 64, 128]), _log(rng, 1, 64)
            if rank * (len(outs) * c + sum(outs)) * max(pool, seqs) <= 400e6 and seqs * new_hi * (c + sum(outs)) <= 60e6:
                break
        x, w, y = rng.choice([("bf16", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "bf16", "f32"), ("f32", "bf16", "f32"), ("f32", "f32", "f32")])
        case = _adapter("", seqs, rng.choice([1, new_hi]), new_hi, c, "+".join(map(str, outs)), pool, rng.randint(1, min(pool, seqs)),
                        rng.choice([rank, max(1, rank // 4)]), rank, x, w, y, rng.choice([0, 0, 3, 8]), rng.choice([0, 0, 0, 4]))
    del case["name"]
    return case


def _spread(lo, hi, n):
    """n sizes from lo to hi, unevenly spread: the last is hi."""
    return [lo + int((hi - lo) * (((i + 1) * 0.6180339887498949) % 1.0)) for i in range(n - 1)] + [hi]


def _sequences(case):
    """Rows of each sequence, which of the `used` adapters it names (-1: none), and the ranks of these adapters."""
    new = _spread(case["new_lo"], case["new_hi"], case["seqs"])
    names = [-1 if case["without"] and i % case["without"] == case["without"] - 1 else i % case["used"] for i in range(case["seqs"])]
    return new, names, _spread(case["rank_lo"], case["rank"], case["used"])


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _activations(n, c, g, pad=0):
    """Rows as a model's hidden states: roughly normal, a few channels much larger for every token."""
    factor = torch.ones(c, device=DEV)
    few = torch.randperm(c, generator=g, device=DEV)[:max(1, c // 200)]
    factor[few] = torch.empty(few.numel(), device=DEV).uniform_(30.0, 100.0, generator=g)
    full = torch.randn((n, c + pad), generator=g, device=DEV)
    full[:, :c] *= factor
    return full[:, :c], few


def _map(c, expand, split, r):
    """A reassembly map in CSR form: the channels `split` become 2 to 8 sub-channels each, as many pairs and triples of neighbours on
    the disassembled axis as were split off are merged.  Returns row_ptr, src, scale."""
    parts = np.ones(c, np.int64)
    extra, k = max(1, int(c * expand)), 0
    while parts.sum() - c < extra:
        parts[split[k % split.size]] += 1 + int(r.randint(0, 3))
        k += 1
    parts[split] = np.minimum(parts[split], 8)
    rows = [[(ch, 1.0 / parts[ch])] for ch in range(c) for _ in range(parts[ch])]
    whole = [i for i in range(len(rows)) if parts[rows[i][0][0]] == 1]
    pick = r.permutation(len(whole))[:2 * (int(parts.sum()) - c)]
    drop = set()
    for a, b in zip(pick[0::2], pick[1::2]):                      # member a goes into b
        a, b = whole[a], whole[b]
        rows[b] = rows[b] + rows[a]
        drop.add(a)
    more = [i for i in range(len(rows)) if len(rows[i]) == 2]
    for i, a in zip(more[::4], [w for w in whole if w not in drop and len(rows[w]) == 1][7::31]):
        rows[i] = rows[i] + rows[a]
        drop.add(a)
    rows = [[(s, 1.0 / len(row)) if len(row) > 1 else (s, v) for s, v in row] for i, row in enumerate(rows) if i not in drop]
    return (np.cumsum([0] + [len(row) for row in rows]).astype(np.int32), np.array([s for row in rows for s, _ in row], np.int32),
            np.array([v for row in rows for _, v in row], np.float32))


def _row_bytes(k, bits):
    return -(-k // 256) * 256 * bits // 8


def _prepare_norm(case, seed):
    g = _gen(seed)
    n, c, pad = case["n"], case["c"], case["pad"]
    x, few = _activations(n, c, g, pad)
    r, _ = _activations(n, c, g, pad)
    x, r = (torch.empty_strided((n, c), (c + pad, 1), dtype=TYPES[t], device=DEV).copy_(v) for t, v in ((case["x"], x), (case["r"], r)))
    s = dict(case=case, x=x, r=r, sum=torch.empty((n, c), dtype=TYPES[case["r"]], device=DEV))
    s["gamma"] = torch.empty(c, device=DEV).uniform_(0.5, 1.5, generator=g)
    s["beta"] = torch.randn(c, generator=g, device=DEV) * 0.1 if case["norm"] == "layer" else None
    s["k"] = c
    if case["expand"]:
        csr = _map(c, case["expand"], few.cpu().numpy(), np.random.RandomState(seed % (1 << 31)))
        s["k"] = k = csr[0].size - 1
        # the plain form's tables: the l-th source of every channel and its scale, 0 where a channel has fewer
        count = np.diff(csr[0])
        src, scale = np.zeros((count.max(), k), np.int64), np.zeros((count.max(), k), np.float32)
        for l in range(count.max()):
            has = count > l
            src[l, has], scale[l, has] = csr[1][csr[0][:-1][has] + l], csr[2][csr[0][:-1][has] + l]
        s["csr"], s["src"], s["scale"] = csr, torch.from_numpy(src).to(DEV), torch.from_numpy(scale).to(DEV)
    out = TYPES["bf16" if case["y"] == "none" else case["y"]]
    s["values"] = torch.empty((n, s["k"]), dtype=out, device=DEV)
    s["y"] = None if case["y"] == "none" else torch.empty((n, c), dtype=out, device=DEV)
    if own:
        from paper_2310_08041_amd import binding as b
        s["b"] = b
        s["gather"] = b.DeviceGather(*s["csr"], c) if case["expand"] else None
        s["out"] = b.DeviceQAct(n, s["k"], case["bits"])
    return s


def _prepare_adapter(case, seed):
    g = _gen(seed)
    new, names, ranks = _sequences(case)
    outs = [int(o) for o in case["parts"].split("+")]
    rows, c, o, rank = sum(new) + case["tail"], case["c"], sum(outs), case["rank"]
    slot = torch.randperm(case["pool"], generator=g, device=DEV)[:case["used"]].cpu().tolist()
    of_slot = torch.full((case["pool"],), rank, dtype=torch.int32)
    for at, n in zip(slot, ranks):
        of_slot[at] = n
    adapter = torch.tensor([-1 if k < 0 else slot[k] for k in names], dtype=torch.int32)
    s = dict(case=case, new=new, outs=outs, rows=rows, names=adapter.tolist(), ranks=of_slot.tolist(), adapter=adapter.to(DEV), rank=of_slot.to(DEV))
    s["x"] = _activations(rows, c, g)[0].div_(8.0).to(TYPES[case["x"]])
    s["y"] = torch.randn((rows, o), generator=g, device=DEV).to(TYPES[case["y"]])
    s["out"] = torch.full_like(s["y"], 3.0)
    # what lies past an adapter's own rank is whatever was there
    w = TYPES[case["w"]]
    s["A"] = torch.empty((case["pool"], len(outs) * rank, c), dtype=w, device=DEV)
    s["B"] = torch.empty((case["pool"], o, rank), dtype=w, device=DEV)
    for at in range(case["pool"]):
        s["A"][at] = torch.randn((len(outs) * rank, c), generator=g, device=DEV) * (1.0 / math.sqrt(c))
        s["B"][at] = torch.randn((o, rank), generator=g, device=DEV) * (1.0 / math.sqrt(rank))
    s["factor"] = torch.empty(case["pool"], device=DEV).uniform_(0.5, 2.0, generator=g)
    s["row_start"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEV)
    s["row_seq"] = torch.tensor([i for i, n in enumerate(new) for _ in range(n)], dtype=torch.int64, device=DEV)
    s["row_new"] = torch.tensor([j for n in new for j in range(n)], dtype=torch.int64, device=DEV)
    if own:
        from paper_2310_08041_amd import binding as b
        s["b"] = b
        s["adapters"] = b.DeviceAdapters(s["A"], s["B"], s["factor"], s["rank"], outs)
        single = all(n == 1 for n in new) and not case["tail"]
        # which rows are whose: once for a step, whatever the number of layers and projections
        s["plan"] = b.DeviceAdapterPlan(rows, case["pool"])
        b.qllm_adapter_plan(s["plan"], s["adapter"], None if single else s["row_start"])
        s["workspace"] = torch.empty(b.qllm_adapter_workspace_bytes(s["adapters"], rows), dtype=torch.uint8, device=DEV)
    return s


def prepare(case, seed):
    case = dict(case)
    return _prepare_norm(case, seed) if case["kind"] == "norm" else _prepare_adapter(case, seed)


# ---------------------------------------------------------------- passes, in their plain form

def _packed(codes, bits):
    """uint8 codes [n, k], k a multiple of 256, packed as the layers read them."""
    if bits == 8:
        return codes
    if bits == 4:
        return codes[:, 0::2] | (codes[:, 1::2] << 4)
    four = codes.view(codes.shape[0], -1, 4).to(torch.int32)
    word = four[..., 0] | (four[..., 1] << 6) | (four[..., 2] << 12) | (four[..., 3] << 18)
    return torch.stack((word & 255, (word >> 8) & 255, word >> 16), -1).to(torch.uint8).flatten(1)


def _plain_norm(s):
    case = s["case"]
    s["sum"].copy_(s["x"].float() + s["r"].float())
    v = s["sum"].float()
    if case["norm"] == "rms":
        rstd = 1.0 / torch.sqrt(v.double().square().mean(-1, keepdim=True) + EPS)
        v = v * rstd.float() * s["gamma"]
    elif case["norm"] == "layer":
        mu = v.double().mean(-1, keepdim=True)
        rstd = 1.0 / torch.sqrt((v.double() - mu).square().mean(-1, keepdim=True) + EPS)
        v = (v - mu.float()) * rstd.float() * s["gamma"] + s["beta"]
    if s["y"] is not None:
        s["y"].copy_(v)
    if case["expand"]:
        z = v[:, s["src"][0]] * s["scale"][0]
        for l in range(1, s["src"].shape[0]):
            z = z + v[:, s["src"][l]] * s["scale"][l]
        v = z
    # Eq. (2): quotients rounded once to float32, products exact in 64 bits
    lo, hi = v.amin(-1, keepdim=True), v.amax(-1, keepdim=True)
    alpha = ((hi - lo).double() / (2 ** case["bits"] - 1)).float()
    alpha = torch.where(hi > lo, alpha, torch.ones_like(alpha))
    inv = (1.0 / alpha.double()).float().double()
    beta = -torch.round(lo.double() * inv)
    codes = (torch.round(v.double() * inv) + beta).clamp_(0, 2 ** case["bits"] - 1)
    s["values"].copy_(alpha * (codes - beta).float())
    k = s["k"]
    codes = torch.nn.functional.pad(codes.to(torch.uint8), (0, -(-k // 256) * 256 - k))
    return [s["sum"], s["values"], alpha[:, 0], beta[:, 0].to(torch.int32), codes.sum(-1, dtype=torch.int32), _packed(codes, case["bits"])] + \
        ([] if s["y"] is None else [s["y"]])


def _plain_adapter(s):
    case = s["case"]
    seqs, rank, n = case["seqs"], case["rank"], s["row_seq"].numel()
    parts = len(s["outs"])
    # the rows of every sequence in a padded block, its adapter's weights beside it, those past its rank (and of none) zero
    x = torch.zeros((seqs, max(s["new"]), case["c"]), device=DEV)
    x[s["row_seq"], s["row_new"]] = s["x"][:n].float()
    a = s["adapter"].long().clamp(min=0)
    live = (torch.arange(rank, device=DEV) < s["rank"][a][:, None]) & (s["adapter"] >= 0)[:, None]
    down = s["A"][a].float() * live.repeat(1, parts)[:, :, None]
    up = s["B"][a].float() * live[:, None]
    h = torch.matmul(x, down.transpose(-1, -2)).unflatten(-1, (parts, rank))
    at, delta = 0, []
    for p, o in enumerate(s["outs"]):
        delta.append(torch.matmul(h[:, :, p], up[:, at:at + o].transpose(-1, -2)))
        at += o
    delta = torch.cat(delta, -1) * s["factor"][a][:, None, None]
    s["out"][:n] = s["y"][:n].float() + delta[s["row_seq"], s["row_new"]]
    return s["out"]


# ---------------------------------------------------------------- passes, through the framework

def _own_norm(s):
    b, case, q = s["b"], s["case"], s["out"]
    b.qllm_add_norm_quant(s["x"], s["r"], s["sum"], NORMS[case["norm"]], s["gamma"], s["beta"], EPS, q, case["bits"], gather=s["gather"],
                          y_out=s["y"], values_out=s["values"])
    return [s["sum"], s["values"], q.scale, q.zero, q.rowsum, q.codes] + ([] if s["y"] is None else [s["y"]])


def _own_adapter(s):
    s["b"].qllm_adapter_apply(s["x"], s["adapters"], s["plan"], s["y"], s["out"], s["workspace"])
    return s["out"]


def run(state):
    if own:
        return _own_norm(state) if state["case"]["kind"] == "norm" else _own_adapter(state)
    return _plain_norm(state) if state["case"]["kind"] == "norm" else _plain_adapter(state)


# ---------------------------------------------------------------- the same from the definition, in 64 bits

def _exact_norm(s):
    case, bits = s["case"], s["case"]["bits"]
    # the sum is rounded to the stream's type by definition, and so are, to float32, the elementwise steps behind it
    f = lambda t: t.float().double()  # noqa: E731
    total = (s["x"].double() + s["r"].double()).float().to(s["sum"].dtype).double()
    y = total
    if case["norm"] != "none":
        mean = total.sum(1) / case["c"] if case["norm"] == "layer" else torch.zeros(case["n"], dtype=torch.float64, device=DEV)
        off = total - mean[:, None]
        root = f((torch.einsum("ij,ij->i", off, off) / case["c"] + EPS) ** -0.5)
        del off
        y = f(f(f(total - f(mean)[:, None]) * root[:, None]) * s["gamma"].double())
        y = y if s["beta"] is None else f(y + s["beta"].double())
    z = y
    if case["expand"]:
        row_ptr, src, scale = (torch.from_numpy(t).to(DEV) for t in s["csr"])
        count = torch.diff(row_ptr)
        z = torch.zeros((case["n"], s["k"]), dtype=torch.float64, device=DEV)
        for l in range(int(count.max())):
            ch = torch.nonzero(count > l)[:, 0]
            e = row_ptr[ch].long() + l
            z[:, ch] = f(z[:, ch] + f(y[:, src[e].long()] * scale[e].double()))
    low, high = z.min(1).values, z.max(1).values
    alpha = f(f(high - low) / (2 ** bits - 1))
    alpha[high == low] = 1.0
    inv = f(alpha.reciprocal())
    zero = -(low * inv).round()
    q = ((z * inv[:, None]).round() + zero[:, None]).clamp(0, 2 ** bits - 1)
    values = alpha[:, None] * (q - zero[:, None])
    whole = q.sum(1).to(torch.int32)
    return [total, values, alpha, zero.to(torch.int32), whole, None] + ([] if s["y"] is None else [y])


def _exact_adapter(s):
    case, rank = s["case"], s["case"]["rank"]
    out = torch.full((s["rows"], sum(s["outs"])), 3.0, dtype=torch.float64, device=DEV)
    at = 0
    for n, a in zip(s["new"], s["names"]):
        out[at:at + n] = s["y"][at:at + n].double()
        if a >= 0:
            col, r = 0, s["ranks"][a]
            for p, o in enumerate(s["outs"]):
                h = s["x"][at:at + n].double() @ s["A"][a, p * rank:p * rank + r].double().T
                out[at:at + n, col:col + o] += float(s["factor"][a]) * (h @ s["B"][a, col:col + o, :r].double().T)
                col += o
        at += n
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _exact_norm(s) if case["kind"] == "norm" else _exact_adapter(s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = lambda t: 2 if t in ("bf16", "none") else 4  # noqa: E731
    if case["kind"] == "norm":
        n, c = case["n"], case["c"]
        each = size(case["x"]) + 2 * size(case["r"]) + size(case["y"]) * (1 if case["y"] == "none" else 2)
        return {"bytes": float(n * c * each + n * _row_bytes(c, case["bits"]) + 12 * n + 4 * c), "flops": 12.0 * n * c}
    new, names, ranks = _sequences(case)
    outs = [int(o) for o in case["parts"].split("+")]
    width = len(outs) * case["c"] + sum(outs)
    has = [(n, ranks[a]) for n, a in zip(new, names) if a >= 0]
    weights = sum(ranks[a] for a in set(names) if a >= 0) * width
    return {"bytes": float(sum(n for n, _ in has) * case["c"] * size(case["x"]) + 2 * sum(new) * sum(outs) * size(case["y"]) + weights * size(case["w"])),
            "flops": 2.0 * width * sum(n * r for n, r in has)}
