"""The operators of a key/value cache held in 4 bits, as cases that can be timed and compared.

A case is one pass through an operator on inputs made from a seed:

  append   the q/k/v projection's rows of a step: rotary positions on q and k, Eq. (2) per token and head on k and v, codes into
           the pages of the sequences; read back, so that what the cache holds for the rows is among the outputs
  attend   softmax attention of a step's queries over the pages, grouped heads, causal, optionally a sliding window
  fork     continuations of prompts share the prompts' pages; a page that is only partly filled is copied, in every layer
  compact  pages in use move into free pages below them, in every layer, and the tables follow

`own` false: elementary torch operations in 32 bits (64 where angles and values next to a rounding border need them), one
rounding at the end.  `own` true: the framework's calls.  Shapes are those of `paper_2310_08041_amd/workloads.py` (heads of 128
channels: 4096 = 32 heads, 5120 = 40, 8192 = 64 of which 8 carry keys and values) or generic.

A page of one layer holds, head after head: codes of the keys [page, dim / 2] and of the values, then alpha (float32) and beta
(int32) of the keys and of the values, [page] each; code 2j in the low half of byte j.  A value is alpha * (code - beta).
"""
import math

import numpy as np
import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ROPES = {"none": 0, "halves": 1, "pairs": 2}
QMAX = 15


# ---------------------------------------------------------------- cases

def _append(name, seqs, len_lo, len_hi, new_lo, new_hi, heads, group, dim=128, page=64, dtype="bf16", rope="halves", tail=0):
    return dict(name=name, kind="append", seqs=seqs, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi, heads=heads,
                group=group, dim=dim, page=page, dtype=dtype, rope=rope, tail=tail)


def _attend(name, seqs, len_lo, len_hi, new_lo, new_hi, heads, group, dim=128, page=64, dtype="bf16", window=0, tail=0):
    return dict(name=name, kind="attend", seqs=seqs, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi, heads=heads,
                group=group, dim=dim, page=page, dtype=dtype, window=window, tail=tail)


def _pages(name, kind, layers, heads, pages, seqs, children=0, dim=128, page=64):
    return dict(name=name, kind=kind, layers=layers, heads=heads, pages=pages, seqs=seqs, children=children, dim=dim, page=page)


def listed():
    return [
        # sixteen requests decoded together (the decode configuration: 64 query heads, 8 of keys and values), one token each
        _append("append_decode_16", 16, 700, 4100, 1, 1, 8, 8),
        # prefill of one 2048-token segment (the 7B configuration)
        _append("append_prefill_2048", 1, 2048, 2048, 2048, 2048, 32, 1),
        # a ragged step in float32, neighbouring channels rotated together, at far positions, rows of padding at the end
        _append("append_ragged_f32", 5, 90000, 130000, 1, 301, 4, 3, dim=64, page=32, dtype="f32", rope="pairs", tail=11),
        # one interactive request, a short cache: the smallest call, latency
        _attend("attend_1_short", 1, 333, 333, 1, 1, 32, 1),
        # sixteen requests decoded together (the decode configuration)
        _attend("attend_decode_16", 16, 1000, 8000, 1, 1, 8, 8),
        # one request over a long document
        _attend("attend_1_long", 1, 131000, 131000, 1, 1, 8, 8),
        # a large decode batch of a model without shared heads (7B)
        _attend("attend_decode_64_mha", 64, 500, 3500, 1, 1, 32, 1),
        # prefill of one segment (7B)
        _attend("attend_prefill_2048", 1, 2048, 2048, 2048, 2048, 32, 1),
        # the next chunk of a long prompt (70B)
        _attend("attend_chunk_long", 1, 16000, 16000, 2000, 2000, 8, 8),
        # prompts and single tokens in one step, float32, a sliding window, heads of 64, padding rows
        _attend("attend_mixed_window_f32", 9, 40, 3000, 0, 260, 4, 3, dim=64, page=32, dtype="f32", window=1000, tail=5),
        # sixteen continuations of four prompts through 32 layers
        _pages("fork_16", "fork", 32, 8, 200, 4, children=16),
        # after many requests have ended: the pages in use move together, 32 layers
        _pages("compact_400", "compact", 32, 8, 400, 24),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "fork", "compact"])
    heads, group, dim = rng.choice([(8, 8, 128), (32, 1, 128), (40, 1, 128), (8, 4, 128), (4, 7, 128), (2, 6, 64), (8, 1, 64), (1, 16, 128), (5, 3, 64)])
    page, dtype = rng.choice([32, 64, 64, 128]), rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind in ("fork", "compact"):
        seqs = _log(rng, 2, 24)
        return {k: v for k, v in _pages("", kind, _log(rng, 2, 32), rng.choice([1, 2, 4, 8]), rng.randint(90, 400), seqs,
                                        children=rng.randint(seqs, 2 * seqs) if kind == "fork" else 0, dim=dim, page=page).items() if k != "name"}
    if kind == "append":
        seqs = _log(rng, 1, 64)
        new_hi = _log(rng, 1, max(1, 2000 // seqs))
        hi = _log(rng, new_hi + 1, 100000)
        c = _append("", seqs, min(hi, new_hi + (hi - new_hi) // 5), hi, rng.choice([1, new_hi]), new_hi, heads, group, dim, page, dtype,
                    rng.choice(["halves", "halves", "pairs", "none"]), rng.choice([0, 0, 3]))
    elif rng.random() < 0.6:                                     # decode
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 20, 130000 // seqs)
        c = _attend("", seqs, max(1, hi // 5), hi, 1, 1, heads, group, dim, page, dtype, rng.choice([0, 0, 0, max(1, hi // 3)]), rng.choice([0, 0, 2]))
    else:                                                        # chunks of prompts, mixed with single tokens
        seqs = _log(rng, 1, 6)
        new_hi = _log(rng, 2, 1500 // seqs)
        hi = new_hi + _log(rng, 1, 4000)
        c = _attend("", seqs, max(1, hi // 4), hi, rng.choice([0, 1, new_hi]), new_hi, heads, group, dim, page, dtype,
                    rng.choice([0, 0, 0, max(1, hi // 2)]), rng.choice([0, 0, 7]))
    return {k: v for k, v in c.items() if k != "name"}


def _spread(lo, hi, n):
    """n sizes from lo to hi, unevenly spread: the last is hi."""
    return [lo + int((hi - lo) * (((i + 1) * 0.6180339887498949) % 1.0)) for i in range(n - 1)] + [hi]


def _shape(case):
    """New rows and lengths (these among them) of the sequences of a step."""
    new = _spread(case["new_lo"], case["new_hi"], case["seqs"])
    length = _spread(case["len_lo"], case["len_hi"], case["seqs"])
    return new, [max(l, n) for l, n in zip(length, new)]


# ---------------------------------------------------------------- the plain form of the cache

def _page_bytes(case):
    return case["heads"] * case["page"] * (case["dim"] + 16)


def _parts(layer, heads, dim, page):
    """Views of a layer's pages: codes of the keys, of the values [pages, heads, page, dim / 2], alpha and beta of both [pages, heads, page]."""
    b = layer.view(layer.shape[0], heads, page * (dim + 16))
    c = page * dim // 2
    at = lambda k, t: b[:, :, 2 * c + 4 * page * k:2 * c + 4 * page * (k + 1)].view(t)
    return (b[:, :, :c].unflatten(-1, (page, dim // 2)), b[:, :, c:2 * c].unflatten(-1, (page, dim // 2)),
            at(0, torch.float32), at(1, torch.int32), at(2, torch.float32), at(3, torch.int32))


def _quantize(x):
    """Eq. (2) along the last axis of float32 values: alpha, beta, codes."""
    lo, hi = x.amin(-1), x.amax(-1)
    alpha = (hi - lo) / QMAX
    alpha = torch.where(alpha >= torch.finfo(torch.float32).tiny, alpha, torch.ones_like(alpha))
    inv = 1.0 / alpha
    beta = -torch.round(lo.double() * inv.double())
    codes = (torch.round(x.double() * inv.double()[..., None]) + beta[..., None]).clamp(0, QMAX)
    return alpha, beta.to(torch.int32), codes.to(torch.uint8)


def _pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(packed):
    return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)


def _values(packed, alpha, beta, dtype=torch.float32):
    return alpha.to(dtype)[..., None] * (_unpack(packed).to(dtype) - beta.to(dtype)[..., None])


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _kv_like(shape, g, heads, dim):
    """Keys or values as a model has them: roughly normal, a few channels of each head much larger."""
    size = torch.ones(heads, dim, device=DEV)
    size[:, torch.randperm(dim, generator=g, device=DEV)[:max(1, dim // 32)]] = 4.0
    return torch.randn(shape, generator=g, device=DEV) * size


def _filled(case, pages, g):
    """One layer's pages, full of quantized keys and values."""
    heads, dim, page = case["heads"], case["dim"], case["page"]
    layer = torch.zeros((pages, _page_bytes(case)), dtype=torch.uint8, device=DEV)
    kc, vc, ka, kb, va, vb = _parts(layer, heads, dim, page)
    step = max(1, (1 << 27) // (heads * page * dim))
    for at in range(0, pages, step):
        n = min(step, pages - at)
        for c, a, b in ((kc, ka, kb), (vc, va, vb)):
            alpha, beta, codes = _quantize(_kv_like((n, page, heads, dim), g, heads, dim).transpose(1, 2))
            c[at:at + n], a[at:at + n], b[at:at + n] = _pack(codes), alpha, beta
    return layer


def _prepare_step(case, seed):
    new, length = _shape(case)
    g = _gen(seed)
    page, heads, dim = case["page"], case["heads"], case["dim"]
    hq, rows, dtype = heads * case["group"], sum(new) + case["tail"], TYPES[case["dtype"]]
    need = [-(-l // page) for l in length]
    spare = 3 + sum(need) // 20
    pages = sum(need) + spare
    if case["kind"] == "append":                                 # only the pages that the new rows reach are looked at
        first = [(l - n) // page for l, n in zip(length, new)]
        pages = sum(n - f for n, f in zip(need, first)) + spare
    else:
        first = [0] * len(need)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(new), max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, (f, n) in enumerate(zip(first, need)):
        table[i, f:n] = order[at:at + n - f]
        at += n - f
    s = dict(case=case, new=new, length=length, table=table, rows=rows,
             row_start=torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEV),
             len_dev=torch.tensor(length, dtype=torch.int32, device=DEV),
             row_seq=torch.tensor([i for i, n in enumerate(new) for _ in range(n)], dtype=torch.int64, device=DEV),
             row_new=torch.tensor([j for n in new for j in range(n)], dtype=torch.int64, device=DEV),
             row_pos=torch.tensor([l - n + j for l, n in zip(length, new) for j in range(n)], dtype=torch.int64, device=DEV))
    if case["kind"] == "append":
        s["layer"] = torch.zeros((pages, _page_bytes(case)), dtype=torch.uint8, device=DEV)
        # the projection's output: q, k and v of a row lie one after the other
        qkv = torch.cat([_kv_like((rows, h, dim), g, h, dim).flatten(1) for h in (hq, heads, heads)], 1).to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :hq * dim], qkv[:, hq * dim:(hq + heads) * dim], qkv[:, (hq + heads) * dim:]
        s["inv_freq"] = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEV) / dim)
        s["q_out"] = torch.full((rows, hq * dim), 3.0, dtype=dtype, device=DEV)
        s["k_out"], s["v_out"] = (torch.full((rows, heads * dim), 3.0, dtype=dtype, device=DEV) for _ in range(2))
    else:
        s["layer"] = _filled(case, pages, g)
        s["q"] = torch.randn((rows, hq * dim), generator=g, device=DEV).mul_(0.6).to(dtype)
        s["out"] = torch.full((rows, hq * dim), 3.0, dtype=dtype, device=DEV)
        s["scale"] = 1.0 / math.sqrt(dim)
    if own:
        from paper_2310_08041_amd import binding as b
        s["b"] = b
        s["cache"] = b.DeviceKVCache(1, pages, heads, dim, page, pages=s["layer"][None])
        decode = all(n == 1 for n in new) and not case["tail"]
        s["batch"] = b.DeviceKVBatch(rows, s["table"], s["len_dev"], None if decode else s["row_start"])
        if case["kind"] == "attend":
            need = b.qllm_kv_attention_workspace_bytes(s["cache"], s["batch"], hq)
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return s


def _prepare_pages(case, seed):
    """A book of sequences of different lengths over scattered pages, and the pages of all layers."""
    g, r = _gen(seed), np.random.RandomState(seed % (1 << 31))
    page, pages, seqs = case["page"], case["pages"], case["seqs"]
    slots = seqs + case["children"]
    free = list(r.permutation(pages))
    if case["kind"] == "fork":                                   # room is left for a page of every child
        most = (pages - case["children"]) // seqs
    else:
        most = max(1, pages * 3 // (5 * seqs))
    table = np.full((slots, most), -1, np.int32)
    length, refs = np.zeros(slots, np.int32), np.zeros(pages, np.int32)
    for i, n in enumerate(_spread(max(1, most // 2), most, seqs)):
        table[i, :n] = [free.pop() for _ in range(n)]
        length[i] = n * page - r.randint(0, page)
        refs[table[i, :n]] = 1
    s = dict(case=case, table=table, length=length, refs=refs)
    if case["kind"] == "fork":
        s["parents"] = np.sort(r.randint(0, seqs, case["children"])).astype(np.int32)
        s["children"] = np.arange(seqs, slots, dtype=np.int32)
    words = case["layers"] * pages * _page_bytes(case) // 4
    pool = torch.randint(-(1 << 31), 1 << 31, (words,), generator=g, device=DEV, dtype=torch.int32)
    s["pool"] = pool.view(torch.uint8).view(case["layers"], pages, _page_bytes(case))
    if own:
        from paper_2310_08041_amd import binding as b
        s["b"] = b
        s["cache"] = b.DeviceKVCache(case["layers"], pages, case["heads"], case["dim"], page, pages=s["pool"])
    else:
        for k in ("table", "length", "refs") + (("parents", "children") if case["kind"] == "fork" else ()):
            s[k + "_dev"] = torch.from_numpy(s[k]).to(DEV)
    return s


def prepare(case, seed):
    case = dict(case)
    return _prepare_pages(case, seed) if case["kind"] in ("fork", "compact") else _prepare_step(case, seed)


# ---------------------------------------------------------------- passes, in their plain form

def _rotated(x, pos, inv_freq, rope):
    """x [rows, heads, dim] float32, rotated by its position; products and sums in 64 bits, rounded once."""
    if rope == "none":
        return x
    angle = pos.double()[:, None] * inv_freq
    c, s = angle.cos().float().double()[:, None], angle.sin().float().double()[:, None]
    half = x.shape[-1] // 2
    a, b = (x[..., :half], x[..., half:]) if rope == "halves" else (x[..., 0::2], x[..., 1::2])
    a, b = a.double(), b.double()
    a, b = (a * c - b * s).float(), (b * c + a * s).float()
    return torch.cat((a, b), -1) if rope == "halves" else torch.stack((a, b), -1).flatten(-2)


def _plain_append(s):
    case = s["case"]
    heads, dim, page, n = case["heads"], case["dim"], case["page"], s["row_pos"].numel()
    q, k, v = (s[t][:n].float().unflatten(-1, (-1, dim)) for t in ("q", "k", "v"))
    q, k = _rotated(q, s["row_pos"], s["inv_freq"], case["rope"]), _rotated(k, s["row_pos"], s["inv_freq"], case["rope"])
    s["q_out"][:n] = q.flatten(1).to(s["q_out"].dtype)
    kc, vc, ka, kb, va, vb = _parts(s["layer"], heads, dim, page)
    at, place = s["table"][s["row_seq"], s["row_pos"] // page].long(), s["row_pos"] % page
    for x, codes, alphas, betas, out in ((k, kc, ka, kb, s["k_out"]), (v, vc, va, vb, s["v_out"])):
        alpha, beta, c = _quantize(x)
        codes[at, :, place], alphas[at, :, place], betas[at, :, place] = _pack(c), alpha, beta
        out[:n] = _values(codes[at, :, place], alphas[at, :, place], betas[at, :, place]).flatten(1).to(out.dtype)
    return s["q_out"], s["k_out"], s["v_out"]


def _gathered(s, dtype=torch.float32):
    """Keys and values of all sequences [sequences, heads, padded length, dim]."""
    case = s["case"]
    tab = s["table"].long().clamp(min=0)
    kc, vc, ka, kb, va, vb = _parts(s["layer"], case["heads"], case["dim"], case["page"])
    flat = lambda x: x.transpose(1, 2).flatten(2, 3)             # [sequences, pages, heads, page, dim] -> heads first, pages joined
    return flat(_values(kc[tab], ka[tab], kb[tab], dtype)), flat(_values(vc[tab], va[tab], vb[tab], dtype))


def _plain_attend(s):
    case = s["case"]
    heads, group, dim = case["heads"], case["group"], case["dim"]
    seqs, most, n = case["seqs"], max(s["new"]), s["row_pos"].numel()
    k, v = _gathered(s)
    # queries of every sequence in a padded block [sequences, kv heads, new rows * group, dim]
    q = torch.zeros((seqs, most, heads, group, dim), device=DEV)
    q[s["row_seq"], s["row_new"]] = s["q"][:n].float().view(n, heads, group, dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(seqs, heads, most * group, dim)
    scores = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    t = torch.arange(k.shape[2], device=DEV)
    pos = (s["len_dev"] - torch.diff(s["row_start"]))[:, None] + torch.arange(most, device=DEV)
    seen = t <= pos[..., None]
    if case["window"]:
        seen = seen & (t > pos[..., None] - case["window"])
    seen = seen[:, None, :, None].expand(seqs, 1, most, group, t.numel()).flatten(2, 3)
    scores = scores.masked_fill_(~seen, -math.inf)
    p = (scores - scores.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = o.view(seqs, heads, most, group, dim).permute(0, 2, 1, 3, 4)
    s["out"][:n] = o[s["row_seq"], s["row_new"]].reshape(n, -1).to(s["out"].dtype)
    return s["out"]


def _plain_fork(s):
    page, pool = s["case"]["page"], s["pool"]
    table, length, refs = s["table_dev"].clone(), s["length_dev"].clone(), s["refs_dev"].clone()
    par, chi = s["parents_dev"].long(), s["children_dev"].long()
    rows, whole = table[par], length[par].long() // page
    col = torch.arange(table.shape[1], device=DEV)
    shared = rows[col < whole[:, None]].long()
    part = torch.nonzero(length[par] % page)[:, 0]
    fresh = torch.nonzero(refs == 0)[:part.numel(), 0]
    old = rows[part, whole[part]].long()
    rows[part, whole[part]] = fresh.to(torch.int32)
    table[chi], length[chi] = rows, length[par]
    refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    refs[fresh] = 1
    pool[:, fresh] = pool[:, old]
    return table, length, refs, pool


def _plain_compact(s):
    pool = s["pool"]
    table, refs = s["table_dev"].clone(), s["refs_dev"].clone()
    used = refs > 0
    number = torch.arange(refs.numel(), device=DEV)
    high = number >= used.sum()
    src, dst = torch.nonzero(used & high)[:, 0], torch.nonzero(~used & ~high)[:, 0]
    to = number.clone()
    to[src] = dst
    table = torch.where(table >= 0, to[table.long().clamp(min=0)].to(torch.int32), table)
    refs[dst], refs[src] = refs[src], torch.zeros_like(refs[src])
    pool[:, dst] = pool[:, src]
    return table, refs, pool


# ---------------------------------------------------------------- passes, through the framework

def _own_append(s):
    b, case = s["b"], s["case"]
    b.qllm_kv_append(s["cache"], 0, s["batch"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], rope=ROPES[case["rope"]], inv_freq=s["inv_freq"])
    b.qllm_kv_read(s["cache"], 0, s["batch"], s["k_out"], s["v_out"])
    return s["q_out"], s["k_out"], s["v_out"]


def _own_attend(s):
    s["b"].qllm_kv_attention(s["q"], s["cache"], 0, s["batch"], s["scale"], s["out"], s["workspace"], window=s["case"]["window"])
    return s["out"]


def _own_pages(s):
    b, case = s["b"], s["case"]
    book = b.KVBook(case["page"], s["table"].copy(), s["length"].copy(), s["refs"].copy())
    if case["kind"] == "fork":
        src, dst = b.qllm_kv_fork_host(book, s["parents"], s["children"])
    else:
        src, dst = b.qllm_kv_compact_host(book)
    b.qllm_kv_copy_pages(s["cache"], src, dst)
    table = torch.from_numpy(book.table).to(DEV)
    return (table, book.length, book.refs, s["pool"]) if case["kind"] == "fork" else (table, book.refs, s["pool"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "fork": _own_pages, "compact": _own_pages}[kind](state)
    return {"append": _plain_append, "attend": _plain_attend, "fork": _plain_fork, "compact": _plain_compact}[kind](state)


# ---------------------------------------------------------------- the same from the definition, in 64 bits

def _exact_append(s):
    case = s["case"]
    dim, half = case["dim"], case["dim"] // 2
    n = sum(s["new"])
    pos = torch.cat([torch.arange(l - m, l, dtype=torch.float64, device=DEV) for l, m in zip(s["length"], s["new"])])
    outs = []
    for name in ("q", "k", "v"):
        x = s[name][:n].double().view(n, -1, dim)
        if name != "v" and case["rope"] != "none":
            # channel d goes with its partner, which enters with a minus in the first of the two
            d = torch.arange(dim, device=DEV)
            pair, first, other = (d % half, d < half, (d + half) % dim) if case["rope"] == "halves" else (d // 2, d % 2 == 0, d ^ 1)
            a = torch.outer(pos, s["inv_freq"][pair])
            cos, sin = torch.cos(a).float().double(), torch.sin(a).float().double() * torch.where(first, -1.0, 1.0)
            x = x * cos[:, None] + x[..., other] * sin[:, None]
        if name == "q":
            y = x
        else:
            x = x.float()                                        # the quantizer's input and its alpha and 1 / alpha are float32 by definition
            low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            alpha = (high - low) / 15.0
            alpha[alpha < 2.0 ** -126] = 1.0
            inv, a64 = (1.0 / alpha).double(), alpha.double()
            beta = -(low.double() * inv).round()
            y = a64 * (((x.double() * inv).round() + beta).clamp(0.0, 15.0) - beta)
        out = torch.full((s["rows"], x.shape[1] * dim), 3.0, dtype=torch.float64, device=DEV)
        out[:n] = y.reshape(n, -1)
        outs.append(out)
    return tuple(outs)


def _exact_attend(s):
    case = s["case"]
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    kc, vc, ka, kb, va, vb = _parts(s["layer"], heads, dim, page)
    out = torch.full((s["rows"], heads * group * dim), 3.0, dtype=torch.float64, device=DEV)
    at = 0
    for i, (n, length) in enumerate(zip(s["new"], s["length"])):
        if n:
            tab = s["table"][i, :-(-length // page)].long()
            pos = torch.arange(length - n, length, device=DEV)[:, None]
            t = torch.arange(length, device=DEV)
            hidden = (t > pos) | ((t <= pos - case["window"]) if case["window"] else torch.zeros_like(t > pos))
            for h in range(heads):
                key, val = (_values(c[tab, h], a[tab, h], z[tab, h], torch.float64).reshape(-1, dim)[:length] for c, a, z in ((kc, ka, kb), (vc, va, vb)))
                for j in range(group):
                    col = (h * group + j) * dim
                    x = (s["q"][at:at + n, col:col + dim].double() @ key.T) * s["scale"]
                    x[hidden] = -math.inf
                    out[at:at + n, col:col + dim] = torch.softmax(x, -1) @ val
        at += n
    return out


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return _exact_append(s) if case["kind"] == "append" else _exact_attend(s)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    page_bytes = _page_bytes(case)
    if case["kind"] == "compact":
        used = sum(_spread(max(1, case["pages"] * 3 // (5 * case["seqs"]) // 2), max(1, case["pages"] * 3 // (5 * case["seqs"])), case["seqs"]))
        moved = used * (1 - used / case["pages"])                # on average
        return {"bytes": 2.0 * moved * case["layers"] * page_bytes, "flops": 0}
    if case["kind"] == "fork":
        return {"bytes": 2.0 * case["children"] * case["layers"] * page_bytes, "flops": 0}
    new, length = _shape(case)
    heads, hq, dim = case["heads"], case["heads"] * case["group"], case["dim"]
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "append":
        rows = sum(new)
        # q in and out, k and v in, their codes out, and what was written read back and given out
        return {"bytes": float(rows * dim * size * (2 * hq + 4 * heads) + 4 * rows * heads * (dim // 2 + 8)), "flops": 6.0 * rows * dim * (hq + 2 * heads)}
    tokens = pairs = 0
    for n, l in zip(new, length):
        w = case["window"] or l
        first, last = l - n, l - 1
        if n:
            tokens += l - max(0, first - w + 1)
            pairs += sum(min(p + 1, w) for p in range(first, last + 1))
    return {"bytes": float(tokens * heads * (dim + 16) + 2 * sum(new) * hq * dim * size), "flops": 4.0 * dim * hq * pairs}
