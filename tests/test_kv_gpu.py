"""The 4-bit key/value cache on the device against its numpy statement: pages bit for bit, attention within bounds that come from
the roundings it makes (see `tolerance`)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2310_08041_amd import binding
    return binding


def _t(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _bf16(x):
    """The float32 values that bfloat16 tensors of x hold."""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def _heads_like(rng, rows, heads, dim):
    """Roughly normal, with channels that are large for every token, zero vectors, constant and one-sided ones among them."""
    x = rng.standard_normal((rows, heads, dim)).astype(np.float32)
    x[..., rng.integers(0, dim, 2)] *= 20.0
    if rows > 3:
        x[0] = 0.0
        x[1, :, :] = 0.75
        x[2] = np.abs(x[2]) + 30.0
    return x


class Made:
    pass


def make(rng, heads, group, dim, page, lengths, new, slots=None, n_lines=None, rows=None, spare=3, extra_cols=1, garbage=0xFF, filled=True):
    """A cache of one layer with every token of every line quantized into scattered pages; what no token owns holds `garbage`
    bytes (NaN as alpha)."""
    from oracle import kv_cache as okv
    c = Made()
    c.heads, c.group, c.dim, c.page = heads, group, dim, page
    n = len(lengths)
    n_lines = n if n_lines is None else n_lines
    c.slot = None if slots is None else np.asarray(slots, np.int32)
    line_of = list(range(n)) if slots is None else list(slots)
    c.length = np.zeros(n_lines, np.int32)
    for i, l in zip(line_of, lengths):
        if 0 <= i < n_lines:
            c.length[i] = l
    need = -(-c.length // page)
    c.n_pages = int(need.sum()) + spare
    order = rng.permutation(c.n_pages).astype(np.int32)
    c.table = np.full((n_lines, max(1, int(need.max()) + extra_cols)), -1, np.int32)
    at = 0
    for i in range(n_lines):
        c.table[i, :need[i]] = order[at:at + need[i]]
        at += need[i]
    c.row_start = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    c.rows = rows if rows is not None else (n if new is None else int(sum(new)))
    raw = np.full((c.n_pages, heads * page * (dim + 16)), garbage, np.uint8)
    c.pages = okv.Pages(raw, heads, dim, page)
    if filled:
        for i in range(n_lines):
            l = int(c.length[i])
            if l:
                tok = [(r, i, r) for r in range(l)]
                okv.append(c.pages, c.table, tok, _heads_like(rng, l, heads, dim), _heads_like(rng, l, heads, dim))
    c.tokens = okv.rows_of(c.rows, c.row_start, c.slot, c.length)
    return c


def on_device(b, c):
    cache = b.DeviceKVCache(1, c.n_pages, c.heads, c.dim, c.page, pages=_t(c.pages.raw)[None])
    batch = b.DeviceKVBatch(c.rows, _t(c.table), _t(c.length), None if c.row_start is None else _t(c.row_start),
                            None if c.slot is None else _t(c.slot))
    return cache, batch


APPEND = [  # dtype, rope, heads, group, dim, page, lengths, new rows, far
    ("bf16", 1, 2, 4, 128, 64, [1, 64, 65, 200], [1, 64, 3, 130], 0),
    ("bf16", 2, 3, 1, 64, 32, [33, 32, 31], [33, 1, 0], 0),
    ("bf16", 0, 1, 7, 128, 256, [300], [300], 0),
    ("f32", 1, 1, 3, 64, 128, [129, 5], [129, 5], 0),
    ("f32", 2, 5, 2, 128, 32, [40, 1, 1, 96], None, 0),
    ("bf16", 1, 40, 1, 128, 64, [17, 100], None, 0),
    ("f32", 1, 1, 1, 128, 32, [1000000], [40], 1000000),                 # far positions: the angle needs its 64 bits
]


@pytest.mark.parametrize("dtype,rope,heads,group,dim,page,lengths,new,far", APPEND)
def test_append_writes_the_pages_of_the_definition(oracle, b, dtype, rope, heads, group, dim, page, lengths, new, far):
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(hash((rope, heads, dim, page)) % 1000)
    if far:
        c = make(rng, heads, group, dim, page, [64], new, filled=False)
        # the line holds a million tokens, of which only the last pages are there
        cols = -(-far // page)
        c.table = np.full((1, cols), -1, np.int32)
        c.table[0, cols - 3:] = [2, 0, 1]
        c.length[0] = far
        c.tokens = okv.rows_of(c.rows, c.row_start, c.slot, c.length)
    else:
        c = make(rng, heads, group, dim, page, lengths, new, filled=False, rows=None if new is None else sum(new) + 2)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    hq = heads * group
    qkv = _heads_like(rng, c.rows, hq + 2 * heads, dim)
    if dtype == "bf16":
        qkv = _bf16(qkv)
    inv_freq = 10000.0 ** (-np.arange(0, dim, 2) / dim)
    cache, batch = on_device(b, c)
    x = _t(qkv.reshape(c.rows, -1), td)
    q, k, v = x[:, :hq * dim], x[:, hq * dim:(hq + heads) * dim], x[:, (hq + heads) * dim:]
    q_out = torch.full((c.rows, hq * dim), 3.0, dtype=td, device="cuda")
    b.qllm_kv_append(cache, 0, batch, k, v, q=q, q_out=q_out, rope=rope, inv_freq=_t(inv_freq) if rope else None)
    k_out, v_out = (torch.full((c.rows, heads * dim), 3.0, dtype=td, device="cuda") for _ in range(2))
    b.qllm_kv_read(cache, 0, batch, k_out, v_out)
    torch.cuda.synchronize()

    positions = np.zeros(c.rows)
    owned = np.zeros(c.rows, bool)
    for r, _, p in c.tokens:
        positions[r], owned[r] = p, True
    turned = okv.rotate(qkv[:, :hq + heads], positions, inv_freq, rope)
    okv.append(c.pages, c.table, c.tokens, turned[:, hq:], qkv[:, hq + heads:])
    assert np.array_equal(cache.pages[0].cpu().numpy(), c.pages.raw)               # every byte, those of no token too
    want_q = np.where(owned[:, None, None], _bf16(turned[:, :hq]) if dtype == "bf16" else turned[:, :hq], 3.0)
    assert np.array_equal(q_out.float().cpu().numpy().reshape(want_q.shape), want_q.astype(np.float32))
    for value, out in ((0, k_out), (1, v_out)):
        want = np.full((c.rows, heads, dim), 3.0)
        for r, line, p in c.tokens:
            pg = okv.page_at(c.table, c.n_pages, page, line, p)
            if pg >= 0:
                for h in range(heads):
                    want[r, h] = c.pages.get(pg, h, p % page, value)[0]
        want = want.astype(np.float32)
        assert np.array_equal(out.float().cpu().numpy().reshape(want.shape), _bf16(want) if dtype == "bf16" else want)


def test_append_takes_rows_of_any_stride_and_alignment_and_rotates_in_place(oracle, b):
    """Rows that miss 16-byte alignment, q rotated in place, no q at all: the same pages."""
    import torch
    rng = np.random.default_rng(5)
    heads, group, dim, page = 2, 2, 64, 32
    c = make(rng, heads, group, dim, page, [50, 7], [20, 7], filled=False)
    qkv = _bf16(_heads_like(rng, c.rows, heads * group + 2 * heads, dim)).reshape(c.rows, -1)
    f = _t(10000.0 ** (-np.arange(0, dim, 2) / dim))
    wq, wk = heads * group * dim, heads * dim
    got = []
    for pad, off in ((0, 0), (8, 8), (3, 1), (1, 5)):
        cache, batch = on_device(b, c)
        buf = torch.zeros((c.rows, wq + 2 * wk + pad + off), dtype=torch.bfloat16, device="cuda")
        x = buf[:, off:off + wq + 2 * wk]
        x.copy_(_t(qkv))
        q, k, v = x[:, :wq], x[:, wq:wq + wk], x[:, wq + wk:]
        b.qllm_kv_append(cache, 0, batch, k, v, q=q, q_out=q, rope=1, inv_freq=f)
        alone, _ = on_device(b, c)
        b.qllm_kv_append(alone, 0, batch, k, v, rope=1, inv_freq=f)
        assert torch.equal(alone.pages, cache.pages)
        out = torch.zeros((c.rows, wk + pad + off), dtype=torch.bfloat16, device="cuda")
        b.qllm_kv_read(cache, 0, batch, v_out=out[:, off:off + wk])
        got.append((cache.pages.clone(), q.clone(), out[:, off:off + wk].clone()))
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other))


def test_append_skips_what_is_not_there(oracle, b):
    """Lines outside the table, pages outside the cache, tokens before the first and behind the line's end: nothing is written for
    them, the others are as ever."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(6)
    heads, dim, page = 2, 128, 32
    c = make(rng, heads, 1, dim, page, [40, 33, 70, 10, 64], [5, 33, 4, 12, 40], slots=[4, -1, 7, 2, 1], n_lines=5, filled=False, rows=100, extra_cols=0)
    c.length[1] = 90                                        # longer than its line's pages
    c.table[4, 1] = c.n_pages                               # outside the cache
    c.table[1, 0] = -7
    c.tokens = okv.rows_of(c.rows, c.row_start, c.slot, c.length)
    kv = _heads_like(rng, c.rows, 2 * heads, dim)
    cache, batch = on_device(b, c)
    b.qllm_kv_append(cache, 0, batch, _t(kv[:, :heads].reshape(c.rows, -1)), _t(kv[:, heads:].reshape(c.rows, -1)))
    out = torch.full((c.rows, heads * dim), 9.0, device="cuda")
    b.qllm_kv_read(cache, 0, batch, out)
    okv.append(c.pages, c.table, c.tokens, kv[:, :heads], kv[:, heads:])
    assert np.array_equal(cache.pages[0].cpu().numpy(), c.pages.raw)
    there = {r for r, line, p in c.tokens if okv.page_at(c.table, c.n_pages, page, line, p) >= 0}
    assert 0 < len(there) < c.rows
    kept = (out == 9.0).all(1).cpu().numpy()
    assert [r for r in range(c.rows) if not kept[r]] == sorted(there)


# ---------------------------------------------------------------- attention

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}                 # half a step, relative


def tolerance(want, absv, err_s, err_o, q_type, out_type):
    """Roundings, element by element: the output's own; that of every weight p alpha before it meets the values (bf16 for bf16
    queries, 24 bits for fp32 ones), the same rounded number standing in all sums: where the weights' own sum is taken of the
    rounded ones, w (1 + d) gives sum w d (v - out) / (1 + ..), at most half a step of sum w |v| and of |out|; the scores' fp32
    error, which moves weights and their sum by at most e^E - 1 each; the fp32 sums."""
    p = HALF[q_type]
    return HALF[out_type] * (np.abs(want) + p * absv) * (1 + 2.0 ** -7) + p * (1 + 2.0 ** -7) * (absv + np.abs(want)) + 2.0 * np.expm1(err_s) * absv + 2.0 * err_o + 1e-30


ATTEND = [  # q, out, heads, group, dim, page, lengths, new rows, window, slots, lines, rows behind the last
    ("bf16", "bf16", 2, 1, 128, 64, [1], None, 0, None, None, 0),
    ("bf16", "bf16", 1, 8, 128, 64, [1, 31, 32, 33, 64, 500], None, 0, None, None, 0),
    ("bf16", "f32", 2, 3, 64, 32, [40, 129, 7], None, 0, [2, 0, 3], 4, 0),
    ("bf16", "bf16", 1, 17, 128, 128, [130, 257], None, 0, None, None, 0),         # more query heads than a tile has rows
    ("bf16", "bf16", 2, 2, 128, 32, [70, 5, 64], [70, 5, 64], 0, None, None, 3),   # whole prompts, rows of padding
    ("bf16", "bf16", 1, 4, 128, 64, [300, 90, 0, 12], [33, 1, 0, 12], 0, None, None, 0),
    ("bf16", "bf16", 1, 5, 64, 32, [200, 77], [100, 3], 50, None, None, 1),        # a window
    ("bf16", "bf16", 1, 1, 128, 32, [400], None, 1, None, None, 0),                # a window of the token itself
    ("f32", "f32", 2, 3, 64, 32, [150, 40], [60, 40], 0, None, None, 0),
    ("f32", "f32", 1, 2, 128, 64, [333, 1, 65], None, 100, None, None, 0),
    ("f32", "bf16", 1, 1, 128, 256, [270], [270], 0, None, None, 0),
    ("bf16", "f32", 1, 3, 128, 64, [3, 5], [5, 2], 0, None, None, 0),              # more new rows than tokens: rows that see nothing
    ("bf16", "bf16", 1, 8, 128, 64, [1500, 2100], None, 0, None, None, 0),         # long enough to be split
    ("bf16", "bf16", 1, 2, 128, 64, [700], [300], 0, None, None, 0),               # a chunk of a prompt, several tiles
    ("bf16", "bf16", 2, 1, 64, 32, [330, 140], [140, 140], 90, None, None, 0),
]


@pytest.mark.parametrize("q_type,out_type,heads,group,dim,page,lengths,new,window,slots,lines,tail", ATTEND)
def test_attention_within_the_bounds_of_its_roundings(oracle, b, q_type, out_type, heads, group, dim, page, lengths, new, window, slots, lines, tail):
    import torch
    from oracle import kv_cache as okv
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    rng = np.random.default_rng(sum(lengths) + 7 * dim + window)
    n_rows = (len(lengths) if new is None else sum(new)) + tail
    c = make(rng, heads, group, dim, page, lengths, new, slots=slots, n_lines=lines, rows=n_rows)
    q = rng.standard_normal((c.rows, heads * group, dim)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    scale = 1.0 / np.sqrt(dim)
    cache, batch = on_device(b, c)
    out = torch.full((c.rows, heads * group * dim), 5.0, dtype=types[out_type], device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), types[q_type]), cache, 0, batch, scale, out, ws, window=window)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(scale), window, out=np.full(q.shape, 5.0))
    got = out.double().cpu().numpy().reshape(want.shape)
    assert np.isfinite(got).all()
    tol = tolerance(want, *bounds, q_type, out_type)
    for r in set(range(c.rows)) - {t[0] for t in c.tokens}:
        assert (got[r] == 5.0).all()                          # rows of no sequence
    worst = np.abs(got - want) / tol
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


PROMPTS = [  # out, heads, group, dim, page, lengths, new rows, window, rows behind the last: enough rows for the prompts kernel
    ("bf16", 16, 8, 128, 64, [200], [140], 0, 0),
    ("bf16", 32, 1, 128, 128, [530], [530], 0, 3),
    ("f32", 20, 3, 64, 32, [150, 40, 0, 300, 7], [150, 1, 0, 180, 7], 70, 2),    # with single tokens and short ones beside them
    ("bf16", 24, 5, 128, 32, [333, 128, 65], [60, 128, 1], 0, 0),
    ("f32", 16, 16, 128, 256, [90], [90], 5, 0),
    ("bf16", 32, 4, 64, 64, [100, 129], [129, 129], 0, 0),                        # rows before the first token: they see nothing
]


@pytest.mark.parametrize("out_type,heads,group,dim,page,lengths,new,window,tail", PROMPTS)
def test_attention_of_prompts_within_the_bounds_of_its_roundings(oracle, b, out_type, heads, group, dim, page, lengths, new, window, tail):
    import torch
    from oracle import kv_cache as okv
    td = torch.bfloat16 if out_type == "bf16" else torch.float32
    rng = np.random.default_rng(sum(lengths) + dim)
    c = make(rng, heads, group, dim, page, lengths, new, rows=sum(new) + tail)
    assert c.rows * group // 128 * heads >= 128
    hq = heads * group
    q = _bf16(rng.standard_normal((c.rows, hq, dim)).astype(np.float32))
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(dim ** -0.5), window, out=np.full(q.shape, 5.0))
    tol = tolerance(want, *bounds, "bf16", out_type)
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    for pad, off in ((0, 0), (5, 3)):                          # 16-byte aligned rows and others
        qd = torch.zeros((c.rows, hq * dim + pad + off), dtype=torch.bfloat16, device="cuda")[:, off:off + hq * dim]
        qd.copy_(_t(q.reshape(c.rows, -1)))
        out = torch.full((c.rows, hq * dim + pad + off), 5.0, dtype=td, device="cuda")
        b.qllm_kv_attention(qd, cache, 0, batch, dim ** -0.5, out[:, off:off + hq * dim], ws, window=window)
        got = out[:, off:off + hq * dim].double().cpu().numpy().reshape(want.shape)
        assert (out[:, :off] == 5.0).all() and (out[:, off + hq * dim:] == 5.0).all()
        for r in set(range(c.rows)) - {t[0] for t in c.tokens}:
            assert (got[r] == 5.0).all()
        worst = np.abs(got - want) / tol
        assert np.isfinite(got).all() and worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("q_type,heads,group,lengths,new", [("bf16", 1, 4, [700, 40], None), ("f32", 1, 2, [150], None), ("bf16", 16, 8, [190], [140])])
def test_attention_over_keys_and_values_far_from_zero(oracle, b, q_type, heads, group, lengths, new):
    """Vectors whose offset is hundreds to millions of times their range: beta needs more bits than one bf16 has, in places only."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(21)
    c = make(rng, heads, group, 128, 64, lengths, new)
    for i, l in enumerate(lengths):
        far = np.zeros(l)
        far[rng.integers(0, l, l // 8)] = 1.0
        far[10:12] = 3e4
        sign = rng.choice([-1.0, 1.0], (l, heads, 1))
        k = rng.standard_normal((l, heads, 128)) * 0.02 + far[:, None, None] * sign * 3.0
        v = rng.standard_normal((l, heads, 128)) * 0.05 + far[:, None, None] * sign * 40.0
        k[10:12] *= 1e-4
        okv.append(c.pages, c.table, [(r, i, r) for r in range(l)], k.astype(np.float32), v.astype(np.float32))
    q = rng.standard_normal((c.rows, heads * group, 128)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    cache, batch = on_device(b, c)
    out = torch.empty((c.rows, heads * group * 128), device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16 if q_type == "bf16" else torch.float32), cache, 0, batch, 0.05, out, ws)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.05))
    got = out.double().cpu().numpy().reshape(want.shape)
    worst = np.abs(got - want) / tolerance(want, *bounds, q_type, "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


def test_attention_does_not_see_tokens_that_are_not_there(oracle, b):
    """Pages outside the cache, lines outside the table, a length beyond the line: as if those tokens did not exist."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(8)
    c = make(rng, 1, 4, 128, 32, [200, 64, 50, 100, 96], [3, 2, 4, 5, 1], slots=[3, 5, 0, -1, 2], n_lines=4, extra_cols=0)
    c.table[3, 2], c.table[3, 4], c.table[0, 0], c.table[0, 1] = -1, c.n_pages + 3, 1 << 30, -(1 << 31)
    c.length[2] = 200                                         # its line has room for fewer
    c.tokens = okv.rows_of(c.rows, c.row_start, c.slot, c.length)
    q = _bf16(rng.standard_normal((c.rows, 4, 128)).astype(np.float32))
    cache, batch = on_device(b, c)
    out = torch.full((c.rows, 512), 5.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, 4), dtype=torch.uint8, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, 0.1, out, ws)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.1))
    got = out.double().cpu().numpy().reshape(want.shape)
    assert (np.abs(got - want) <= tolerance(want, *bounds, "bf16", "bf16")).all()
    assert (want[3:5] == 0).all() and (want[5:9] == 0).all()  # a line outside the table, a line without pages: zeros


def test_attention_reaches_pages_beyond_32_bits(oracle, b):
    """Pages that lie more than 2^32 bytes into the cache: append, read and attention give what they give at its start."""
    import torch
    rng = np.random.default_rng(9)
    heads, dim, page = 8, 128, 256
    page_bytes = b.qllm_kv_page_bytes(heads, dim, page)
    n_pages = (1 << 32) // page_bytes + 8
    pages = torch.empty((1, n_pages, page_bytes), dtype=torch.uint8, device="cuda")
    cache = b.DeviceKVCache(1, n_pages, heads, dim, page, pages=pages)
    kv = _t(_heads_like(rng, 300, 2 * heads, dim).reshape(300, -1), torch.bfloat16)
    q = torch.randn((300, 16 * dim), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    got = []
    for table in ([[0, 1]], [[n_pages - 1, (1 << 32) // page_bytes + 1]]):
        batch = b.DeviceKVBatch(300, _t(np.array(table, np.int32)), _t(np.array([300], np.int32)), _t(np.array([0, 300], np.int32)))
        b.qllm_kv_append(cache, 0, batch, kv[:, :heads * dim], kv[:, heads * dim:])
        out, back = torch.empty_like(q), torch.empty((300, heads * dim), device="cuda")
        ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, 16), dtype=torch.uint8, device="cuda")
        b.qllm_kv_attention(q, cache, 0, batch, 0.1, out, ws)
        b.qllm_kv_read(cache, 0, batch, back)
        got.append((out, back))
        pages[:, :2].fill_(0xFF)                                 # not to be found by the second round
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and torch.isfinite(got[0][0]).all()


@pytest.mark.parametrize("layers,n_pages,heads,dim,page,n", [(1, 5, 1, 64, 32, 1), (3, 40, 2, 128, 64, 17), (2, 900, 1, 64, 32, 600)])
def test_copying_pages_in_every_layer(b, layers, n_pages, heads, dim, page, n):
    import torch
    rng = np.random.default_rng(n)
    raw = rng.integers(0, 256, (layers, n_pages, heads * page * (dim + 16)), dtype=np.uint8)
    cache = b.DeviceKVCache(layers, n_pages, heads, dim, page, pages=_t(raw))
    places = rng.permutation(n_pages)
    dst, src = places[:n], rng.choice(places[n:], n)              # a source may be copied more than once
    dst, src = np.append(dst, places[n]), np.append(src, places[n])
    b.qllm_kv_copy_pages(cache, src, dst)
    raw[:, dst] = raw[:, src]
    assert np.array_equal(cache.pages.cpu().numpy(), raw)
    b.qllm_kv_copy_pages(cache, [], [])


def _step(b, c, rng, book, cache, slots, n, hq, layers):
    """One step of a serving loop through every layer: room, append, attention.  Returns the layers' outputs."""
    import torch
    if n:
        b.qllm_kv_reserve_host(book, slots, [n] * len(slots))
    rows = max(n, 1) * len(slots)
    start = np.arange(len(slots) + 1, dtype=np.int32) * max(n, 1)
    batch = b.DeviceKVBatch(rows, _t(book.table), _t(book.length), _t(start), _t(np.asarray(slots, np.int32)))
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda")
    outs = []
    for layer in range(layers):
        x = _t(rng.standard_normal((rows, (hq + 2 * cache.heads) * cache.dim)).astype(np.float32), torch.bfloat16)
        q, k, v = x.split([hq * cache.dim, cache.heads * cache.dim, cache.heads * cache.dim], 1)
        if n:
            b.qllm_kv_append(cache, layer, batch, k, v, q=q, q_out=q, rope=1, inv_freq=c)
        out = torch.empty((rows, hq * cache.dim), dtype=torch.bfloat16, device="cuda")
        outs.append(b.qllm_kv_attention(q, cache, layer, batch, cache.dim ** -0.5, out, ws))
    return outs


def test_a_serving_loop_with_forks_and_compaction(b):
    """Prompts, tokens, continuations that share pages, requests that end, pages that move together: what attention gives depends on
    none of it.  A second cache plays the same loop without sharing and without moving."""
    import torch
    heads, hq, dim, page, layers = 2, 6, 128, 32, 2
    f = _t(10000.0 ** (-np.arange(0, dim, 2) / dim))
    r1, r2 = np.random.default_rng(11), np.random.default_rng(11)
    book, cache = b.KVBook.empty(6, 12, 40, page), b.DeviceKVCache(layers, 40, heads, dim, page)
    plain, other = b.KVBook.empty(6, 12, 80, page), b.DeviceKVCache(layers, 80, heads, dim, page)
    step = lambda bk, ca, rng, slots, n: _step(b, f, rng, bk, ca, slots, n, hq, layers)
    both = lambda slots, n: [torch.equal(x, y) for x, y in zip(step(book, cache, r1, slots, n), step(plain, other, r2, slots, n))]
    assert all(both([0, 1, 2], 70))                                     # prompts
    assert all(both([2, 0, 1], 1))
    # line 3 and 4 continue line 1, line 5 line 2; the other cache gets whole copies
    src, dst = b.qllm_kv_fork_host(book, [1, 1, 2], [3, 4, 5])
    b.qllm_kv_copy_pages(cache, src, dst)
    assert src.size == 3 and (book.refs > 1).any()
    for child, parent in ((3, 1), (4, 1), (5, 2)):
        n = int(plain.length[parent])
        b.qllm_kv_reserve_host(plain, [child], [n])
        k = -(-n // page)
        b.qllm_kv_copy_pages(other, plain.table[parent, :k], plain.table[child, :k])
    for _ in range(3):
        assert all(both([5, 1, 3, 4, 0, 2], 1))
    assert all(both([3, 4], 33))
    for bk in (book, plain):
        b.qllm_kv_free_host(bk, [0, 1])
    src, dst = b.qllm_kv_compact_host(book)
    assert src.size and (book.table < (book.refs > 0).sum()).all()
    b.qllm_kv_copy_pages(cache, src, dst)
    assert all(both([2, 3, 4, 5], 0))                                   # queries only, nothing appended
    assert all(both([2, 3, 4, 5], 1))
    b.qllm_kv_free_host(book, [2, 3, 4, 5])
    assert not book.refs.any() and (book.table == -1).all() and not book.length.any()


def test_calls_on_other_streams_and_two_at_once(oracle, b):
    """Two steps in flight on two streams, each with its own workspace, give what they give one after the other."""
    import torch
    rng = np.random.default_rng(12)
    made = [make(rng, 2, 4, 128, 64, [900, 300, 650], None), make(rng, 2, 4, 128, 64, [800, 70], [60, 70])]
    work = []
    for c in made:
        cache, batch = on_device(b, c)
        q = _t(rng.standard_normal((c.rows, 8 * 128)).astype(np.float32), torch.bfloat16)
        ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, 8), dtype=torch.uint8, device="cuda")
        work.append((cache, batch, q, ws))
    alone = [b.qllm_kv_attention(q, ca, 0, ba, 0.1, torch.empty_like(q), ws) for ca, ba, q, ws in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(5):
        outs = [torch.full_like(q, 9.0) for _, _, q, _ in work]
        torch.cuda.synchronize()
        for (ca, ba, q, ws), s, o in zip(work, streams, outs):
            b.qllm_kv_attention(q, ca, 0, ba, 0.1, o, ws, stream=s)
            with torch.cuda.stream(s):
                b.qllm_kv_attention(q, ca, 0, ba, 0.1, o, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(alone, outs))


def test_a_decode_step_replayed_as_a_graph(oracle, b):
    """Append and attention captured once; lengths and rows change between the replays, other work runs in between, a second graph
    shares the workspace."""
    import torch
    rng = np.random.default_rng(13)
    heads, hq, dim, page = 2, 8, 128, 64
    c = make(rng, heads, 4, dim, page, [500, 63, 64, 1200], None, extra_cols=2, spare=20)
    c.table[:, -2:] = np.arange(c.n_pages - 8, c.n_pages, dtype=np.int32).reshape(4, 2)
    for i in range(4):                                                        # the next pages right behind the present ones
        k = -(-int(c.length[i]) // page)
        c.table[i, k:k + 2] = c.table[i, -2:].copy()
    cache, batch = on_device(b, c)
    eager, ebatch = on_device(b, c)
    f = _t(10000.0 ** (-np.arange(0, dim, 2) / dim))
    x = torch.zeros((4, (hq + 2 * heads) * dim), dtype=torch.bfloat16, device="cuda")
    q, k, v = x.split([hq * dim, heads * dim, heads * dim], 1)
    q_out, out = torch.zeros((4, hq * dim), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, hq * dim), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda")

    def step(ca, ba, qo, o):
        b.qllm_kv_append(ca, 0, ba, k, v, q=q, q_out=qo, rope=1, inv_freq=f)
        b.qllm_kv_attention(qo, ca, 0, ba, 0.09, o, ws)

    fresh = lambda: x.copy_(_t(rng.standard_normal(x.shape).astype(np.float32)))
    fresh()
    q2, o2 = torch.empty_like(q_out), torch.empty_like(out)
    step(cache, batch, q_out, out)                                            # loads the kernels before the capture
    step(eager, ebatch, q2, o2)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(cache, batch, q_out, out)
        graphs.append(g)
    for i in range(6):
        fresh()
        batch.length.add_(1), ebatch.length.add_(1)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        step(eager, ebatch, q2, o2)
        (torch.randn(1000, device="cuda") * 2).sum().item()
        assert torch.equal(q2, q_out) and torch.equal(o2, out) and torch.equal(cache.pages, eager.pages)


def test_empty_steps_are_no_ops(b):
    import torch
    cache = b.DeviceKVCache(1, 4, 2, 64, 32)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    for batch in (b.DeviceKVBatch(0, i32(0, 1)[None], i32(5), i32(0)), b.DeviceKVBatch(0, i32(0, 1)[None], i32(5), i32(0, 0)),
                  b.DeviceKVBatch(3, i32(0, 1)[None], i32(5), i32(0))):
        x = torch.full((batch.rows, 128), 2.0, device="cuda")
        ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, 2), dtype=torch.uint8, device="cuda")
        b.qllm_kv_append(cache, 0, batch, x, x)
        b.qllm_kv_read(cache, 0, batch, x)
        b.qllm_kv_attention(x, cache, 0, batch, 1.0, x, ws)
        assert (x == 2.0).all() and not cache.pages.any()


@pytest.mark.parametrize("q_type,group,new,slots", [("bf16", 3, True, True), ("f32", 1, True, False), ("bf16", 8, False, True), ("bf16", 1, False, False)])
def test_attention_of_more_sequences_than_a_wave_has_lanes(oracle, b, q_type, group, new, slots):
    """Two hundred sequences, some without rows, some without tokens, their lines in any order."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(31 + group)
    n = 200
    lengths = rng.integers(0, 60, n)
    lengths[77] = 700
    n_new = np.minimum(rng.integers(0, 4, n), lengths).tolist() if new else None
    c = make(rng, 1, group, 64, 32, lengths.tolist(), n_new, slots=rng.permutation(n).tolist() if slots else None, n_lines=n if slots else None)
    q = rng.standard_normal((c.rows, group, 64)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    cache, batch = on_device(b, c)
    out = torch.full((c.rows, group * 64), 5.0, device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16 if q_type == "bf16" else torch.float32), cache, 0, batch, 0.125, out, ws)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.125))
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, q_type, "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


def test_attention_of_many_sequences_over_one_shared_line(oracle, b):
    """Hundreds of sequences continue one long line: a wave has more steps of a sequence than it has lanes, twice over."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(32)
    n, tokens, group = 1500, 9000, 2
    c = make(rng, 1, group, 64, 64, [tokens], None)
    table = np.repeat(c.table, n, 0)
    length = np.full(n, tokens, np.int32)
    length[::3] -= rng.integers(0, 3000, 500).astype(np.int32)
    cache = b.DeviceKVCache(1, c.n_pages, 1, 64, 64, pages=_t(c.pages.raw)[None])
    batch = b.DeviceKVBatch(n, _t(table), _t(length))
    q = _bf16(rng.standard_normal((n, group, 64)).astype(np.float32))
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((n, group * 64), device="cuda")
    b.qllm_kv_attention(_t(q.reshape(n, -1), torch.bfloat16), cache, 0, batch, 0.125, out, ws)
    some = [(r, 0, int(length[r]) - 1) for r in range(0, n, 31)]
    want, *bounds = okv.attention(q, c.pages, c.table, some, c.length, np.float32(0.125))
    rows = [r for r, _, _ in some]
    worst = (np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", "f32"))[rows]
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("lengths,new,window", [([2500], [130], 0), ([2300, 40], [140, 3], 0), ([2200], [2200], 2100)])
def test_attention_of_prompts_behind_many_tokens(oracle, b, lengths, new, window):
    """More tokens than a wave keeps page numbers of at a time."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(33)
    heads, group = 2, 256 if window == 0 else 16
    c = make(rng, heads, group, 64, 32, lengths, new)
    hq = heads * group
    if window:                                                # the prompt's last rows are enough to look at
        c.tokens = c.tokens[-40:]
    q = _bf16(rng.standard_normal((c.rows, hq, 64)).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((c.rows, hq * 64), dtype=torch.bfloat16, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, 0.125, out, ws, window=window)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.125), window)
    rows = sorted({r for r, _, _ in c.tokens})
    worst = (np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", "bf16"))[rows]
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("scale", [-0.2, 0.0, 1e-30, 3.0])
@pytest.mark.parametrize("heads,lengths,new", [(1, [300, 20], [3, 20]), (24, [200], [180])])
def test_attention_with_scales_of_any_sign_and_size(oracle, b, heads, lengths, new, scale):
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(34)
    c = make(rng, heads, 4, 128, 64, lengths, new)
    q = _bf16(0.3 * rng.standard_normal((c.rows, heads * 4, 128)).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * 4), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((c.rows, heads * 512), device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, scale, out, ws)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(scale))
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("heads,group,lengths,new", [(2, 4, [900, 40], None), (16, 8, [300], [200]), (16, 2, [300, 70], [260, 1])])
def test_attention_writes_over_its_queries_and_keeps_rows_apart(oracle, b, heads, group, lengths, new):
    """out may be q; a query that is not finite spoils its own output alone."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(35)
    c = make(rng, heads, group, 128, 64, lengths, new)
    cache, batch = on_device(b, c)
    x = _bf16(rng.standard_normal((c.rows, heads * group, 128)).astype(np.float32))
    q = _t(x.reshape(c.rows, -1), torch.bfloat16)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda")
    out = b.qllm_kv_attention(q, cache, 0, batch, 0.1, torch.empty_like(q), ws)
    over = q.clone()
    b.qllm_kv_attention(over, cache, 0, batch, 0.1, over, ws)
    assert torch.equal(over, out)
    at = c.rows // 2
    q[at, 128] = float("nan")                                # query head 1
    q[at, 5 * 128] = float("inf")                            # and 5
    got = b.qllm_kv_attention(q, cache, 0, batch, 0.1, torch.empty_like(q), ws).double().cpu().numpy().reshape(x.shape)
    want, *bounds = okv.attention(x, c.pages, c.table, c.tokens, c.length, np.float32(0.1))
    off = np.abs(got - want) / tolerance(want, *bounds, "bf16", "bf16")
    assert np.isnan(got[at, 1]).all()
    off[at, [1, 5]] = 0.0
    assert off.max() <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))


def test_chunks_of_a_prompt_replayed_as_a_graph_on_another_stream(oracle, b):
    """A prompt in chunks of 200 rows beside single tokens, captured on a stream of its own: lengths and rows change between the
    replays, other work runs in between, a second graph shares the workspace."""
    import torch
    rng = np.random.default_rng(36)
    heads, group, dim, page = 16, 8, 64, 32
    hq = heads * group
    c = make(rng, heads, group, dim, page, [200, 50, 33], [200, 1, 1], extra_cols=22, spare=80)
    free = np.setdiff1d(np.arange(c.n_pages), c.table[c.table >= 0])
    c.table[c.table < 0] = free[:(c.table < 0).sum()]
    cache, batch = on_device(b, c)
    eager, ebatch = on_device(b, c)
    f = _t(10000.0 ** (-np.arange(0, dim, 2) / dim))
    x = torch.zeros((c.rows, (hq + 2 * heads) * dim), dtype=torch.bfloat16, device="cuda")
    q, k, v = x.split([hq * dim, heads * dim, heads * dim], 1)
    q_out, out, q2, o2 = (torch.zeros((c.rows, hq * dim), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda")

    def step(ca, ba, qo, o):
        b.qllm_kv_append(ca, 0, ba, k, v, q=q, q_out=qo, rope=2, inv_freq=f)
        b.qllm_kv_attention(qo, ca, 0, ba, 0.125, o, ws)

    fresh = lambda: x.copy_(_t(rng.standard_normal(x.shape).astype(np.float32)))
    fresh()
    step(cache, batch, q_out, out)                                            # loads the kernels before the capture
    step(eager, ebatch, q2, o2)
    torch.cuda.synchronize()
    graphs, side = [], torch.cuda.Stream()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step(cache, batch, q_out, out)
        graphs.append(g)
    more = torch.tensor([200, 1, 1], dtype=torch.int32, device="cuda")
    for i in range(3):
        fresh()
        batch.length.add_(more), ebatch.length.add_(more)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[i % 2].replay()
        torch.cuda.synchronize()
        step(eager, ebatch, q2, o2)
        (torch.randn(1000, device="cuda") * 2).sum().item()
        assert torch.equal(q2, q_out) and torch.equal(o2, out) and torch.equal(cache.pages, eager.pages)


@pytest.mark.parametrize("out_type,heads,group,dim,lengths,new,window", [
    ("bf16", 40, 16, 64, [150], [140], 0),                                     # more tiles than the card holds workgroups
    ("f32", 32, 16, 128, [200, 90, 40], [130, 1, 3], 60),
    ("bf16", 16, 8, 64, [20 + i for i in range(90)], [5 + i % 9 for i in range(90)], 0),   # more sequences than a wave has lanes
    ("bf16", 2, 20, 128, [4 + i % 7 for i in range(130)], [i % 6 for i in range(130)], 0),
])
def test_attention_of_many_prompt_tiles_and_of_many_prompts(oracle, b, out_type, heads, group, dim, lengths, new, window):
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(37)
    new = [min(n, l) for n, l in zip(new, lengths)]
    c = make(rng, heads, group, dim, 32, lengths, new)
    hq = heads * group
    q = _bf16(rng.standard_normal((c.rows, hq, dim)).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.full((c.rows, hq * dim), 5.0, dtype=torch.bfloat16 if out_type == "bf16" else torch.float32, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, 0.125, out, ws, window=window)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.125), window)
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", out_type)
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("heads,group,lengths,new", [(1, 4, [300, 40], None), (16, 8, [190], [140])])
def test_attention_over_values_of_very_different_ranges(oracle, b, heads, group, lengths, new):
    """Values from 2^-45 to 2^45 in one line, keys of all ranges below one, some of them nothing but rounding noise."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(38)
    c = make(rng, heads, group, 128, 64, lengths, new)
    for i, l in enumerate(lengths):
        k = rng.standard_normal((l, heads, 128)) * np.exp2(rng.integers(-40, 1, (l, heads, 1)))
        v = rng.standard_normal((l, heads, 128)) * np.exp2(rng.integers(-45, 46, (l, heads, 1)))
        k[5], v[6], v[7] = 1e-38, 0.0, -3.0
        okv.append(c.pages, c.table, [(r, i, r) for r in range(l)], k.astype(np.float32), v.astype(np.float32))
    q = _bf16(rng.standard_normal((c.rows, heads * group, 128)).astype(np.float32))
    cache, batch = on_device(b, c)
    out = torch.empty((c.rows, heads * group * 128), device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, 0.09, out, ws)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.09))
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("out_type,heads,group,dim,page,lengths,new,window", [
    ("bf16", 2, 16, 128, 64, [3000], [130], 0),
    ("f32", 2, 32, 64, 32, [2100], [70], 0),
    ("bf16", 4, 16, 128, 128, [2600, 400, 1500], [70, 1, 40], 0),             # a line of one part, a single token beside them
    ("f32", 4, 16, 64, 32, [2600, 300, 1500], [70, 20, 40], 1100),            # parts that some rows see nothing of
    ("bf16", 1, 64, 128, 64, [5000], [60], 0),                                # as many parts as a tile can have
])
def test_attention_of_prompts_shared_by_workgroups(oracle, b, out_type, heads, group, dim, page, lengths, new, window):
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(39)
    c = make(rng, heads, group, dim, page, lengths, new)
    hq = heads * group
    tiles, tokens = c.rows * group // 128 * heads, c.table.shape[1] * page
    assert tiles >= (16 if len(new) == 1 else 48) and tiles * tokens >= 96000 * (len(new) > 1) and (c.rows * group // 128 + len(new)) * heads <= 128 and tokens >= 2000
    q = _bf16(rng.standard_normal((c.rows, hq, dim)).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda")
    qd, outs = _t(q.reshape(c.rows, -1), torch.bfloat16), []
    for garbage in (0xFF, 0x00):
        ws.fill_(garbage)
        out = torch.full((c.rows, hq * dim), 5.0, dtype=torch.bfloat16 if out_type == "bf16" else torch.float32, device="cuda")
        outs.append(b.qllm_kv_attention(qd, cache, 0, batch, 0.1, out, ws, window=window))
    assert torch.equal(*outs)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.1), window)
    worst = np.abs(outs[0].double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", out_type)
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("heads,group,dim,lengths,new", [(5, 3, 64, [373, 900, 1400], None), (40, 1, 128, [38, 56, 20], [38, 38, 20]), (8, 8, 128, [62, 15], [59, 2]), (2, 8, 128, [4000], None)])
def test_float32_attention_is_as_exact_as_float32_arithmetic(oracle, b, heads, group, dim, lengths, new):
    """The error against 64 bits (norms) is at most twice that of float32 softmax attention on the cache's values themselves, for
    keys and values without a large common part; the codes' offsets of 16 and the zero points cost no bits."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(40)
    c = make(rng, heads, group, dim, 64, lengths, new)
    for i, l in enumerate(lengths):
        okv.append(c.pages, c.table, [(r, i, r) for r in range(l)], *(rng.standard_normal((l, heads, dim)).astype(np.float32) for _ in range(2)))
    q = rng.standard_normal((c.rows, heads * group, dim)).astype(np.float32)
    cache, batch = on_device(b, c)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1)), cache, 0, batch, dim ** -0.5, out, ws)
    want = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(dim ** -0.5))[0]
    plain = np.zeros(want.shape)
    for i, l in enumerate(lengths):
        every = b.DeviceKVBatch(l, _t(c.table[i:i + 1]), _t(np.array([l], np.int32)), _t(np.array([0, l], np.int32)))
        k, v = (torch.empty((l, heads * dim), device="cuda") for _ in range(2))
        b.qllm_kv_read(cache, 0, every, k, v)
        k, v = (x.cpu().reshape(l, heads, dim) for x in (k, v))
        for r, line, p in (t for t in c.tokens if t[1] == i):
            for o in range(heads * group):
                s = (k[:p + 1, o // group] @ torch.from_numpy(q[r, o])) * np.float32(dim ** -0.5)
                plain[r, o] = (torch.softmax(s, 0) @ v[:p + 1, o // group]).numpy()
    got = out.double().cpu().numpy().reshape(want.shape)
    off, plain_off = np.linalg.norm(got - want), np.linalg.norm(plain - want)
    assert off <= 2.0 * plain_off + 2.0 ** -25 * np.linalg.norm(want), (off / plain_off, off / np.linalg.norm(want))


def test_append_read_and_copies_on_a_stream_and_in_a_graph(oracle, b):
    """A stream given by hand and the current one, then one graph of append, copy and read whose inputs change between the replays:
    the graph keeps the list of pages that it was captured with."""
    import torch
    rng = np.random.default_rng(41)
    heads, dim, page = 3, 64, 32
    c = make(rng, heads, 2, dim, page, [40, 70], [40, 70], filled=False, spare=8)
    used = c.table[c.table >= 0]
    free = np.setdiff1d(np.arange(c.n_pages), used)
    src, dst = used[:4].copy(), free[:4].astype(np.int32)
    f = _t(10000.0 ** (-np.arange(0, dim, 2) / dim))
    k, v, k_out = (torch.zeros((c.rows, heads * dim), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    fresh = lambda: [t.copy_(_t(rng.standard_normal(t.shape).astype(np.float32))) for t in (k, v)]

    def step(ca, ba, out, s=None):
        b.qllm_kv_append(ca, 0, ba, k, v, rope=1, inv_freq=f, stream=s)
        b.qllm_kv_copy_pages(ca, src, dst, stream=s)
        b.qllm_kv_read(ca, 0, ba, out, stream=s)

    def same(x, y):
        torch.cuda.synchronize()
        (torch.randn(1000, device="cuda") * 2).sum().item()
        assert torch.equal(x[0].pages, y[0].pages) and torch.equal(x[1], y[1])
        pages = x[0].pages[0].cpu().numpy()
        assert np.array_equal(pages[dst], pages[src])

    fresh()
    eager, ebatch = on_device(b, c)
    want = torch.zeros_like(k_out)
    step(eager, ebatch, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other, obatch = on_device(b, c)
    torch.cuda.synchronize()
    step(other, obatch, k_out, side)
    same((other, k_out), (eager, want))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(other, obatch, k_out)
    kept = src.copy()
    for _ in range(3):
        fresh()
        k_out.zero_()
        torch.cuda.synchronize()
        src[:] = -1                                            # the caller's list may change once the call is back
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        src[:] = kept
        step(eager, ebatch, want)
        same((other, k_out), (eager, want))


@pytest.mark.parametrize("heads,group,new,window", [(8, 16, 30, 700), (8, 160, 3, 2200), (1, 3, 5, 700)])
def test_attention_at_the_last_positions_that_a_line_can_have(oracle, b, heads, group, new, window):
    """A line of 2^31 tokens less a few, of which the last pages are there: what its newest queries see is what they see in a short line
    that ends in the same way."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(43)
    dim, page, tokens = 64, 256, 2500
    hq = heads * group
    c = make(rng, heads, group, dim, page, [tokens], [new], extra_cols=0)
    columns = (2 ** 31 - 1) // page
    far = torch.full((2, columns), -1, dtype=torch.int32, device="cuda")       # two lines: nothing of the first may be found
    far[0] = 0
    far[1, columns - c.table.shape[1]:] = _t(c.table[0])
    length = columns * page - (c.table.shape[1] * page - tokens)
    q = _bf16(rng.standard_normal((new, hq, dim)).astype(np.float32))
    cache, _ = on_device(b, c)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    batch = b.DeviceKVBatch(new, far, i32(7, length), i32(0, new), i32(1))
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.full((new, hq * dim), 5.0, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(new, -1), torch.bfloat16), cache, 0, batch, 0.125, out, ws, window=window)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.125), window)
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, "bf16", "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2 ** 24, 1 << 40])
@pytest.mark.parametrize("q_type,heads,group,lengths,new", [("bf16", 1, 2, [5, 40], [12, 3]), ("f32", 1, 3, [70], [90]), ("bf16", 16, 8, [100], [140]),
                                                            ("bf16", 32, 4, [100, 129], [129, 129])])
def test_a_window_larger_than_any_line_with_rows_before_the_first_token(oracle, b, q_type, heads, group, lengths, new, window):
    """The largest windows are no window, also where a sequence has more new rows than tokens."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(44)
    c = make(rng, heads, group, 64, 32, lengths, new)
    hq = heads * group
    q = rng.standard_normal((c.rows, hq, 64)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    qd = _t(q.reshape(c.rows, -1), torch.bfloat16 if q_type == "bf16" else torch.float32)
    outs = [b.qllm_kv_attention(qd, cache, 0, batch, 0.125, torch.full((c.rows, hq * 64), 5.0, device="cuda"), ws, window=w) for w in (window, 0)]
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.125), window)
    worst = np.abs(outs[0].double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, *bounds, q_type, "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
    assert torch.equal(*outs) and (outs[0] != 0).any()


KINDS = [(2, 3, 64, [70, 200], None), (16, 8, 128, [190], [140]), (24, 5, 64, [333, 128, 65], [60, 128, 1])]   # single tokens; prompts; both


@pytest.mark.parametrize("bits", [0x00000001, 0x00200000, 0x007fffff, 0x80000001, 0x00000000, 0x7f800000, 0xff800000, 0xbf800000])
@pytest.mark.parametrize("heads,group,dim,lengths,new", KINDS)
def test_what_lies_in_unseen_places_does_not_matter(oracle, b, heads, group, dim, lengths, new, bits):
    """Places of no token hold any numbers, as alpha too: subnormal ones (whose reciprocal is infinite), zero, infinities, negative ones."""
    import torch
    rng = np.random.default_rng(45)
    word = np.frombuffer(np.uint32(bits).tobytes(), np.uint8)
    outs = []
    for garbage in (0x3c, np.tile(word, heads * 32 * (dim + 16) // 4)):
        rng = np.random.default_rng(45)
        c = make(rng, heads, group, dim, 32, lengths, new, garbage=garbage)
        q = _t(rng.standard_normal((c.rows, heads * group * dim)).astype(np.float32), torch.bfloat16)
        cache, batch = on_device(b, c)
        ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
        outs.append(b.qllm_kv_attention(q, cache, 0, batch, 0.1, torch.empty((c.rows, heads * group * dim), device="cuda"), ws))
    assert torch.isfinite(outs[0]).all() and torch.equal(*outs)


@pytest.mark.parametrize("every", [1, 3, 17])
@pytest.mark.parametrize("heads,group,dim,lengths,new", KINDS)
def test_tokens_that_nobody_wrote_are_zero_keys_and_values(oracle, b, heads, group, dim, lengths, new, every):
    """A length may count tokens that were never appended, in pages of zeros; and an alpha of zero, or one below the normal floats,
    makes a zero value whatever the codes: it takes its share of the weights, in both kernels."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(46)
    c = make(rng, heads, group, dim, 32, lengths, new)
    for line in range(len(lengths)):
        for t in range(0, lengths[line], every):
            p = okv.page_at(c.table, c.n_pages, 32, line, t)
            for h in range(heads):
                kind = (t // every + h) % 3 if every > 1 else 0
                if kind == 0:                                            # as a new cache has it
                    for value in (0, 1):
                        c.pages.put(p, h, t % 32, value, np.zeros(dim, np.uint8), 0.0, 0)
                else:                                                    # codes and zero point of any value
                    c.pages.put(p, h, t % 32, 1, rng.integers(0, 16, dim).astype(np.uint8), 0.0 if kind == 1 else 1e-40, int(rng.integers(-300, 300)))
    q = _bf16(rng.standard_normal((c.rows, heads * group, dim)).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, 0.1, out, ws)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.1))
    got = out.double().cpu().numpy().reshape(want.shape)
    worst = np.abs(got - want) / tolerance(want, *bounds, "bf16", "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
    if every == 1:
        assert not got.any()


# Ordinary heads, few tokens, float32 out: the bounds are 1e-4 to 3e-4 of the values here and tell a weight of 8 bits, a window of one
# token more or less and a missing newest token from what is promised (test_kv_cpu.py plants each of them in the statement).
CLOSE = [  # q, heads, group, dim, page, lengths, new rows, window: all of them the kernel for few rows
    ("bf16", 2, 1, 128, 64, [1, 2, 3, 5, 9, 33], None, 0),
    ("bf16", 1, 8, 128, 64, [31, 40, 64, 130], None, 0),
    ("bf16", 2, 3, 64, 32, [40, 129, 7], None, 0),
    ("bf16", 1, 4, 64, 32, [150, 90], [5, 2], 50),
    ("bf16", 1, 2, 128, 64, [300, 120], None, 100),
    ("f32", 2, 3, 64, 32, [50, 40], [20, 40], 0),
    ("f32", 1, 2, 128, 64, [333, 1, 65], None, 100),
    ("f32", 1, 1, 64, 128, [40], [40], 7),
]
PARTS = {"bf16": 2.0 ** -16, "f32": 2.0 ** -24}               # of a weight, left out at most


def close_case(q_type, heads, group, dim, page, lengths, new, window):
    """A cache of ordinary heads, queries, and the statement's output with its close bounds."""
    from oracle import kv_cache as okv
    rng = np.random.default_rng(47 + sum(lengths) + dim)
    c = make(rng, heads, group, dim, page, lengths, new, filled=False)
    for i, l in enumerate(lengths):
        okv.append(c.pages, c.table, [(r, i, r) for r in range(l)], *(rng.standard_normal((l, heads, dim)).astype(np.float32) for _ in range(2)))
    q = rng.standard_normal((c.rows, heads * group, dim)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(dim ** -0.5), window, close=True)
    return c, q, want, okv.attention_bound(want, *bounds, PARTS[q_type], 2.0 ** -24)


@pytest.mark.parametrize("q_type,heads,group,dim,page,lengths,new,window", CLOSE)
def test_attention_of_few_rows_keeps_the_bits_it_promises(oracle, b, q_type, heads, group, dim, page, lengths, new, window):
    import torch
    c, q, want, bound = close_case(q_type, heads, group, dim, page, lengths, new, window)
    cache, batch = on_device(b, c)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16 if q_type == "bf16" else torch.float32), cache, 0, batch, dim ** -0.5, out, ws, window=window)
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / bound
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


CLOSE_PROMPTS = [  # the same for the kernel for prompts: weights of one bf16 part, above and below the line
    ("bf16", 2, 4, 128, 64, [60], [60], 7),
    ("bf16", 1, 16, 64, 32, [90], [33], 0),
    ("bf16", 3, 2, 128, 32, [40, 130], [40, 100], 20),
    ("bf16", 2, 8, 64, 128, [100, 20, 9], [50, 1, 9], 12),
]


def close_prompts_case(*case):
    """As close_case; twice the scores' bound (an operation per 16 channels there)."""
    from oracle import kv_cache as okv
    c, q, want, _ = close_case(*case)
    bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(c.dim ** -0.5), case[7], close=True)[1:]
    return c, q, want, okv.attention_bound(want, bounds[0], 2.0 * bounds[1], bounds[2], 2.0 ** -8, 2.0 ** -24)


@pytest.mark.parametrize("q_type,heads,group,dim,page,lengths,new,window", CLOSE_PROMPTS)
def test_attention_of_prompts_sees_the_tokens_it_should(oracle, b, q_type, heads, group, dim, page, lengths, new, window):
    import torch
    c, q, want, bound = close_prompts_case(q_type, heads, group, dim, page, lengths, new, window)
    cache, batch = on_device(b, c)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, dim ** -0.5, out, ws, window=window)
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / bound
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


WINDOWED = [("f32", 1, 2, 128, [333, 1, 65], None, 100), ("f32", 4, 3, 64, [700, 90], [60, 90], 50),
            ("f32", 2, 1, 64, [40, 20], [40, 20], 7)]


def float32_softmax(c, q, k, v, scale, window, r, o, p):
    """Attention of one row and head in float32 steps over the cache's values (k, v [tokens, heads, dim] float32)."""
    import torch
    lo = max(0, p + 1 - window) if window else 0
    s = (k[lo:p + 1, o // c.group] @ torch.from_numpy(q[r, o])) * np.float32(scale)
    return (torch.softmax(s, 0) @ v[lo:p + 1, o // c.group]).numpy()


def exactness(got, want, plain):
    """How many times float32 arithmetic's error (norms), with half a bit of the result beside it."""
    n = np.linalg.norm
    return n(got - want) / (2.0 * n(plain - want) + 2.0 ** -25 * n(want))


def windowed_case(q_type, heads, group, dim, lengths, new, window):
    import torch
    c, q, want, _ = close_case(q_type, heads, group, dim, 64, lengths, new, window)
    plain = np.zeros(want.shape)
    for i, l in enumerate(lengths):
        k, v = (torch.from_numpy(np.array([[c.pages.get(c.table[i, t // 64], h, t % 64, value)[0] for h in range(heads)] for t in range(l)], np.float32)) for value in (0, 1))
        for r, line, p in (t for t in c.tokens if t[1] == i):
            for o in range(heads * group):
                plain[r, o] = float32_softmax(c, q, k, v, dim ** -0.5, window, r, o, p)
    return c, q, want, plain


@pytest.mark.parametrize("q_type,heads,group,dim,lengths,new,window", WINDOWED)
def test_float32_attention_in_a_window_is_as_exact_as_float32_arithmetic(oracle, b, q_type, heads, group, dim, lengths, new, window):
    import torch
    c, q, want, plain = windowed_case(q_type, heads, group, dim, lengths, new, window)
    cache, batch = on_device(b, c)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1)), cache, 0, batch, dim ** -0.5, out, ws, window=window)
    off = exactness(out.double().cpu().numpy().reshape(want.shape), want, plain)
    assert off <= 1.0, off


@pytest.mark.parametrize("heads,dim,page,rope", [(2, 64, 32, 0), (3, 128, 64, 2), (1, 128, 32, 1)])
def test_append_and_read_of_vectors_far_from_zero(oracle, b, heads, dim, page, rope):
    """Offsets of 10^5 to 10^8 times the range, on both sides of the quotient (2^21) from which codes are made in 64 bits and of the
    zero point (2^23) from which they are read in 64 bits; tiny and huge ranges."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(48)
    n = 120
    c = make(rng, heads, 1, dim, page, [n], [n], filled=False)
    k, v = (rng.standard_normal((n, heads, dim)) for _ in range(2))
    for x in (k, v):
        beta = np.exp2(rng.uniform(15, 27, (n, heads, 1))) * rng.choice([-1.0, 1.0], (n, heads, 1))
        beta[::7] = rng.choice([2.0 ** 21, 2.0 ** 23, -2.0 ** 21, -2.0 ** 23], beta[::7].shape) + rng.integers(-9, 9, beta[::7].shape)
        low, high = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
        x -= np.where(rng.random((n, heads, 1)) < 0.9, beta * (high - low) / 15, 0.0)
        x *= np.exp2(rng.integers(-80, 81, (n, heads, 1)))
    k, v = k.astype(np.float32), v.astype(np.float32)
    inv_freq = 10000.0 ** (-np.arange(0, dim, 2) / dim)
    turned = okv.rotate(k, [p for _, _, p in c.tokens], inv_freq, rope)
    okv.append(c.pages, c.table, c.tokens, turned, v)
    betas = np.abs(okv.quantize(v)[2].astype(np.int64))
    assert (betas > 2 ** 23).any() and ((betas > 2 ** 21) & (betas < 2 ** 23)).any() and (betas < 2 ** 21).any()
    cache = b.DeviceKVCache(1, c.n_pages, heads, dim, page, pages=torch.full((1, c.n_pages, heads * page * (dim + 16)), 0xFF, dtype=torch.uint8, device="cuda"))
    batch = b.DeviceKVBatch(n, _t(c.table), _t(c.length), _t(c.row_start))
    b.qllm_kv_append(cache, 0, batch, _t(k.reshape(n, -1)), _t(v.reshape(n, -1)), rope=rope, inv_freq=_t(inv_freq) if rope else None)
    assert np.array_equal(cache.pages[0].cpu().numpy(), c.pages.raw)
    for td in (torch.float32, torch.bfloat16):
        outs = [torch.zeros((n, heads * dim), dtype=td, device="cuda") for _ in range(2)]
        b.qllm_kv_read(cache, 0, batch, *outs)
        for value, out in enumerate(outs):
            want = np.array([[c.pages.get(okv.page_at(c.table, c.n_pages, page, line, p), h, p % page, value)[0] for h in range(heads)] for _, line, p in c.tokens])
            want = want.astype(np.float32)
            assert np.array_equal(out.float().cpu().numpy().reshape(want.shape), _bf16(want) if td is torch.bfloat16 else want)


def test_a_row_that_cannot_be_quantized_leaves_the_others_alone(oracle, b):
    """NaN, infinities, and finite numbers whose range is none (its codes are unspecified too): every other byte of the pages, and
    what attention gives to rows that do not see the token."""
    import torch
    rng = np.random.default_rng(49)
    n, heads, dim, page = 70, 2, 128, 32
    c = make(rng, heads, 2, dim, page, [n], [n], filled=False)
    k, v = (rng.standard_normal((n, heads, dim)).astype(np.float32) for _ in range(2))
    q = _t(rng.standard_normal((n, 2 * heads * dim)).astype(np.float32), torch.bfloat16)
    got = []
    for bad in (None, np.nan, np.inf, -np.inf, "range"):
        k2, v2 = k.copy(), v.copy()
        if bad == "range":
            k2[40, 1, [3, 77]] = v2[40, 1, [3, 77]] = [3e38, -3e38]
        elif bad is not None:
            k2[40, 1, 5] = v2[40, 1, 6] = bad
        cache, batch = on_device(b, c)
        b.qllm_kv_append(cache, 0, batch, _t(k2.reshape(n, -1)), _t(v2.reshape(n, -1)))
        outs = []
        for rows in (n, 3):                                    # the kernel for prompts, that for few rows
            few = b.DeviceKVBatch(rows, _t(c.table), _t(np.array([n if rows == n else 40], np.int32)), _t(np.array([0, rows], np.int32)))
            ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, few, 2 * heads), dtype=torch.uint8, device="cuda")
            out = b.qllm_kv_attention(q[:rows], cache, 0, few, 0.1, torch.empty_like(q[:rows]), ws).view(rows, 2 * heads, dim)
            outs += [out[:40].clone(), out[:, :2].clone()]     # rows before the token; the other key/value head
        ours = cache.pages[0].cpu().numpy().copy()
        p, place = c.table[0, 40 // page], 40 % page
        for value in (0, 1):
            _, code, par = c.pages._at(p, 1, place, value)
            for at, size in ((code, dim // 2), (par, 4), (par + 4 * page, 4)):
                ours[p, at:at + size] = 0
        got.append((ours, outs))
    for ours, outs in got[1:]:
        assert np.array_equal(ours, got[0][0]) and all(torch.equal(x, y) and torch.isfinite(x).all() for x, y in zip(outs, got[0][1]))


@pytest.mark.parametrize("n,dtype", [(150, "bf16"), (700, "f32"), (5000, "bf16")])
def test_append_and_read_of_more_sequences_than_a_wave_has_lanes(oracle, b, n, dtype):
    """The search for a row's sequence takes two and three trips; some sequences have no rows, some no tokens, lines in any order."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(50)
    heads, dim, page = 1, 64, 32
    lengths = rng.integers(0, 50, n)
    new = np.minimum(rng.choice([0, 0, 1, 1, 2, 5], n), lengths)
    new[n - 1] = 0
    c = make(rng, heads, 1, dim, page, lengths.tolist(), new.tolist(), slots=rng.permutation(n).tolist(), n_lines=n, rows=int(new.sum()) + 70, filled=False)
    kv = rng.standard_normal((c.rows, 2, heads, dim)).astype(np.float32)
    kv = _bf16(kv) if dtype == "bf16" else kv
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache, batch = on_device(b, c)
    b.qllm_kv_append(cache, 0, batch, _t(kv[:, 0].reshape(c.rows, -1), td), _t(kv[:, 1].reshape(c.rows, -1), td))
    out = torch.full((c.rows, heads * dim), 9.0, device="cuda")
    b.qllm_kv_read(cache, 0, batch, v_out=out)
    okv.append(c.pages, c.table, c.tokens, kv[:, 0], kv[:, 1])
    assert np.array_equal(cache.pages[0].cpu().numpy(), c.pages.raw)
    want = np.full((c.rows, heads, dim), 9.0, np.float32)
    for r, line, p in c.tokens:
        want[r, 0] = c.pages.get(okv.page_at(c.table, c.n_pages, page, line, p), 0, p % page, 1)[0]
    assert np.array_equal(out.cpu().numpy().reshape(want.shape), want)


@pytest.mark.parametrize("q_type,group,most,window", [("bf16", 3, 2, 0), ("f32", 2, 3, 9), ("bf16", 20, 3, 0)])
def test_attention_of_more_sequences_than_are_listed_with_rows_of_their_own(oracle, b, q_type, group, most, window):
    """More than 512 sequences of 0 to `most` rows: with few rows each, in float32, and with sequences of the kernel for prompts among them."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(51)
    n, dim = 600, 64
    lengths = rng.integers(0, 25, n)
    new = np.minimum(rng.integers(0, most + 1, n) if group < 20 else rng.choice([1, 2, 3, 3], n), lengths)
    c = make(rng, 1, group, dim, 32, lengths.tolist(), new.tolist(), slots=rng.permutation(n).tolist(), n_lines=n, rows=int(new.sum()) + 5)
    assert (c.rows * group > 32 * n) == (group == 20)
    q = rng.standard_normal((c.rows, group, dim)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    cache, batch = on_device(b, c)
    out = torch.full((c.rows, group * dim), 5.0, device="cuda")
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16 if q_type == "bf16" else torch.float32), cache, 0, batch, 0.125, out, ws, window=window)
    want, *bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.125), window, out=np.full(q.shape, 5.0))
    got = out.double().cpu().numpy().reshape(want.shape)
    assert (got[c.rows - 5:] == 5.0).all()
    worst = np.abs(got - want) / tolerance(want, *bounds, q_type, "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


def test_what_is_read_is_rounded_to_float_and_then_to_its_type(oracle, b):
    """bf16 reads go through float32: where the exact product lies next to a border between two bf16 numbers the second rounding may
    go the other way than a single one would."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(52)
    dim, page = 64, 256
    alpha = rng.uniform(0.01, 1.0, 400000).astype(np.float32)
    codes = np.arange(16)
    exact = alpha[:, None].astype(np.float64) * (codes - 7.0)                       # 24 + 4 bits: exact in 64
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(exact), 1e-9))) - 7)          # bf16 numbers are this far apart
    once = np.rint(exact / step) * step
    twice = _bf16(exact.astype(np.float32))
    odd = np.flatnonzero((once != twice).any(1))
    assert odd.size > 3
    raw = np.zeros((1, page * (dim + 16)), np.uint8)
    pages = okv.Pages(raw, 1, dim, page)
    chosen = np.concatenate([odd, np.arange(page)])[:page]
    for t, i in enumerate(chosen):
        pages.put(0, 0, t, 1, np.tile(codes, dim // 16).astype(np.uint8), alpha[i], 7)
    cache = b.DeviceKVCache(1, 1, 1, dim, page, pages=_t(raw)[None])
    batch = b.DeviceKVBatch(page, _t(np.zeros((1, 1), np.int32)), _t(np.array([page], np.int32)), _t(np.array([0, page], np.int32)))
    out = torch.empty((page, dim), dtype=torch.bfloat16, device="cuda")
    b.qllm_kv_read(cache, 0, batch, v_out=out)
    got = out.double().cpu().numpy()[:, :16]
    assert np.array_equal(got, twice[chosen]) and (got != once[chosen]).any()


@pytest.mark.parametrize("far", [2.0 ** 27, 2.0 ** 30])
def test_prompts_over_keys_of_the_smallest_ranges(oracle, b, far):
    """Keys whose alpha is 2^-100, far from zero: their factor counts as 2^-90, which is nothing for queries below 2^30."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(53)
    heads, group, dim, page, n = 16, 4, 128, 32, 90
    c = make(rng, heads, group, dim, page, [n], [n])
    for t in range(n):
        for h in range(heads):
            c.pages.put(int(c.table[0, t // page]), h, t % page, 0, rng.integers(0, 16, dim).astype(np.uint8), 2.0 ** -100, int(far * rng.choice([-1, 1]) * rng.uniform(0.5, 1.0)))
    q = _bf16((np.exp2(rng.uniform(0, 29, (n, heads * group, 1))) * rng.uniform(-1.9, 1.9, (n, heads * group, dim))).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((n, heads * group * dim), device="cuda")
    b.qllm_kv_attention(_t(q.reshape(n, -1), torch.bfloat16), cache, 0, batch, 1.0, out, ws)
    want, absv, err_s, err_o = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(1.0))
    # the factor in place of 2^-100: a score of up to 2^-90 (15 + |beta|) sum |q|, both sides of it
    more = 2.0 * 2.0 ** -90 * (15 + far) * np.abs(q.astype(np.float64)).sum(-1, keepdims=True)
    assert more.max() < 2.0 ** -21
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / tolerance(want, absv, err_s + more, err_o, "bf16", "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("exponent", [-84, 76])
@pytest.mark.parametrize("heads,group,dim,lengths,new", KINDS)
def test_values_at_the_ends_of_their_range(oracle, b, heads, group, dim, lengths, new, exponent):
    """All values as small and as large as attention's sums are stated to hold: alphas of 2^-87 and of 2^78."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(54)
    c = make(rng, heads, group, dim, 32, lengths, new)
    for i, l in enumerate(lengths):
        k, v = (rng.standard_normal((l, heads, dim)) for _ in range(2))
        okv.append(c.pages, c.table, [(r, i, r) for r in range(l)], k.astype(np.float32), np.ldexp(v, exponent).astype(np.float32))
    q = _bf16(rng.standard_normal((c.rows, heads * group, dim)).astype(np.float32))
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, 0.1, out, ws)
    want, absv, err_s, err_o = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(0.1))
    back = 2.0 ** -exponent                                    # the bounds as they are for values around 1
    got = out.double().cpu().numpy().reshape(want.shape) * back
    worst = np.abs(got - want * back) / tolerance(want * back, absv * back, err_s, err_o * back, "bf16", "f32")
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


@pytest.mark.parametrize("q_type,heads,group,dim,page,lengths,new,window", CLOSE_PROMPTS)
def test_attention_of_prompts_with_float32_out_keeps_two_parts_of_a_weight(oracle, b, q_type, heads, group, dim, page, lengths, new, window):
    """What the kernel for few rows keeps: a caller who asks for float32 gets it whatever the number of rows."""
    import torch
    c, q, want, bound = two_part_prompts_case(q_type, heads, group, dim, page, lengths, new, window)
    cache, batch = on_device(b, c)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, heads * group), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.empty((c.rows, heads * group * dim), device="cuda")
    b.qllm_kv_attention(_t(q.reshape(c.rows, -1), torch.bfloat16), cache, 0, batch, dim ** -0.5, out, ws, window=window)
    worst = np.abs(out.double().cpu().numpy().reshape(want.shape) - want) / bound
    assert worst.max() <= 1.0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


def two_part_prompts_case(*case):
    """As close_prompts_case, 2^-16 of a weight left out."""
    from oracle import kv_cache as okv
    c, q, want, _ = close_case(*case)
    bounds = okv.attention(q, c.pages, c.table, c.tokens, c.length, np.float32(c.dim ** -0.5), case[7], close=True)[1:]
    return c, q, want, okv.attention_bound(want, bounds[0], 2.0 * bounds[1], bounds[2], 2.0 ** -16, 2.0 ** -24)


@pytest.mark.parametrize("q_type,heads,group,new", [("bf16", 1, 3, [2, 0, 5, 1]), ("f32", 2, 2, [30, 1, 0, 40]), ("bf16", 16, 8, [90, 0, 33, 1]), ("bf16", 1, 20, [3, 2, 1] * 40)])
def test_rows_before_the_first_sequence_and_a_line_named_more_than_once(oracle, b, q_type, heads, group, new):
    """row_start may begin behind row 0, attention and read may name a line twice: rows of no sequence stay as they were."""
    import torch
    from oracle import kv_cache as okv
    rng = np.random.default_rng(55)
    dim, page, lead, tail = 64, 32, 7, 4
    n, hq = len(new), heads * group
    slots = [i % 3 for i in range(n)]
    c = make(rng, heads, group, dim, page, [100, 47, 130], None)
    start = (lead + np.concatenate([[0], np.cumsum(new)])).astype(np.int32)
    rows = int(start[-1]) + tail
    tokens = okv.rows_of(rows, start, np.array(slots), c.length)
    q = rng.standard_normal((rows, hq, dim)).astype(np.float32)
    q = _bf16(q) if q_type == "bf16" else q
    cache, _ = on_device(b, c)
    batch = b.DeviceKVBatch(rows, _t(c.table), _t(c.length), _t(start), _t(np.array(slots, np.int32)))
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    out = torch.full((rows, hq * dim), 5.0, device="cuda")
    b.qllm_kv_attention(_t(q.reshape(rows, -1), torch.bfloat16 if q_type == "bf16" else torch.float32), cache, 0, batch, 0.125, out, ws)
    k_out, v_out = (torch.full((rows, heads * dim), 9.0, device="cuda") for _ in range(2))
    b.qllm_kv_read(cache, 0, batch, k_out, v_out)
    want, *bounds = okv.attention(q, c.pages, c.table, tokens, c.length, np.float32(0.125), out=np.full(q.shape, 5.0))
    got = out.double().cpu().numpy().reshape(want.shape)
    off = np.abs(got - want) / tolerance(want, *bounds, q_type, "f32")
    assert off.max() <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    k_got, v_got = (x.cpu().numpy().reshape(rows, heads, dim) for x in (k_out, v_out))
    for r in [*range(lead), *range(rows - tail, rows)]:
        assert (got[r] == 5.0).all() and (k_got[r] == 9.0).all() and (v_got[r] == 9.0).all()
    for r, line, p in tokens:
        at = okv.page_at(c.table, c.n_pages, page, line, p)
        for h in range(heads):
            assert np.array_equal(k_got[r, h], c.pages.get(at, h, p % page, 0)[0].astype(np.float32))
            assert np.array_equal(v_got[r, h], c.pages.get(at, h, p % page, 1)[0].astype(np.float32))


@pytest.mark.parametrize("heads,group,dim,lengths,new", [(2, 16, 128, [3000], [130]), (4, 16, 128, [2600, 400, 1500], [70, 1, 40])])
def test_prompts_shared_by_workgroups_write_over_their_queries(oracle, b, heads, group, dim, lengths, new):
    """A tile's parts read its queries in several workgroups, the output comes from a second kernel: the same bits in place and
    through a graph."""
    import torch
    rng = np.random.default_rng(56)
    c = make(rng, heads, group, dim, 64, lengths, new)
    hq = heads * group
    cache, batch = on_device(b, c)
    q = _t(rng.standard_normal((c.rows, hq * dim)).astype(np.float32), torch.bfloat16)
    ws = torch.empty(b.qllm_kv_attention_workspace_bytes(cache, batch, hq), dtype=torch.uint8, device="cuda").fill_(0xFF)
    want = b.qllm_kv_attention(q, cache, 0, batch, 0.1, torch.empty_like(q), ws)
    over = q.clone()
    b.qllm_kv_attention(over, cache, 0, batch, 0.1, over, ws)
    assert torch.equal(over, want)
    torch.cuda.synchronize()
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        b.qllm_kv_attention(over, cache, 0, batch, 0.1, over, ws)
    for _ in range(3):
        over.copy_(q)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(over, want)
        assert torch.equal(b.qllm_kv_attention(q, cache, 0, batch, 0.1, torch.empty_like(q), ws), want)
