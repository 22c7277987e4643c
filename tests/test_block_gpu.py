"""What stands between the layers, on the device: the residual's addition with norm, reassembly and codes bit for bit against the CPU
oracle, adapters against a plain statement in 64 bits within bounds made of the roundings they are allowed."""
import numpy as np
import pytest
import torch

from helpers import random_csr_map
from oracle import api as orc

F32, BF16 = torch.float32, torch.bfloat16
NORM = {"none": 0, "layer": 1, "rms": 2}

gpu = pytest.mark.gpu


def binding():
    from paper_2310_08041_amd import binding
    return binding


# ---------------------------------------------------------------- the residual's addition, norm, reassembly, codes

def strided(t, dtype, pad, lead):
    """The host array t on the device as dtype, rows `pad` elements apart, the first one `lead` elements into its memory."""
    n, c = t.shape
    store = torch.full((lead + n * (c + pad) + 8,), 7.0, dtype=dtype, device="cuda")
    view = store[lead:lead + n * (c + pad)].view(n, c + pad)[:, :c]
    view.copy_(torch.from_numpy(t))
    return view, store


def rounded(t, dtype):
    """float32 values rounded to dtype, as float32."""
    return orc.widen_bf16(orc.round_to_bf16(t)) if dtype == BF16 else t


def draw(rng, n, c, dtype):
    x = rng.standard_normal((n, c)).astype(np.float32)
    x[:, rng.integers(0, c, max(1, c // 100))] *= 60.0
    return rounded(x, dtype)


def expected(x, r, rd, norm, gamma, beta, eps, csr, bits):
    s = r if x is None else rounded(r + x, rd)
    y = s if norm == "none" else orc.norm(np.ascontiguousarray(s), NORM[norm], gamma, beta if norm == "layer" else None, eps)
    z = y if csr is None else orc.apply_map(y, *csr)
    codes, alpha, zero, rowsum = orc.quantize_rows(z, bits)
    values = (alpha[:, None].astype(np.float64) * (codes.astype(np.float64) - zero[:, None])).astype(np.float32)
    return dict(s=s, y=y, codes=codes, alpha=alpha, zero=zero, rowsum=rowsum, values=values)


def check_norm(n, c, norm="rms", xd=BF16, rd=BF16, od=BF16, bits=8, special=0, c_out=None, pad=0, lead=0, into=None, outs=True, shift=True, seed=0,
               big=1.0, eps=1e-5):
    """One call against the oracle; special: every special-th channel of a random map is computed (0: no map); into: what sum_out is."""
    b = binding()
    rng = np.random.default_rng([seed, n, c, bits])
    r = draw(rng, n, c, rd) * np.float32(big)
    x = None if xd is None else draw(rng, n, c, xd) * np.float32(big)
    gamma = rng.uniform(0.5, 1.5, c).astype(np.float32)
    beta = rng.standard_normal(c).astype(np.float32) if norm == "layer" and shift else None
    csr = random_csr_map(rng, c, c_out or c, special) if special else None
    e = expected(x, r, rd, norm, gamma, beta, eps, csr, bits)
    k = e["codes"].shape[1]
    rt, r_store = strided(r, rd, pad, lead)
    xt, x_store = (None, None) if x is None else strided(x, xd, pad, lead)
    st, s_store = strided(np.zeros((n, c), np.float32), rd, pad, lead) if into is None else ({"residual": rt, "x": xt, "none": None}[into], None)
    yt, y_store = strided(np.zeros((n, c), np.float32), od, pad, lead) if outs else (None, None)
    vt, v_store = strided(np.zeros((n, k), np.float32), od, pad, lead) if outs else (None, None)
    q = b.DeviceQAct(n, k, bits)
    for t in (q.codes, q.scale, q.zero, q.rowsum):
        t.fill_(99)
    before = (r_store.clone(), None if x is None else x_store.clone())
    gather = b.DeviceGather(*csr, c) if csr else None
    b.qllm_add_norm_quant(xt, rt, st, NORM[norm], torch.from_numpy(gamma).cuda(), None if beta is None else torch.from_numpy(beta).cuda(), eps, q, bits,
                          gather=gather, y_out=yt, values_out=vt)
    torch.cuda.synchronize()
    codes = q.codes.cpu().numpy()
    assert np.array_equal(codes, orc.pack_codes(e["codes"], bits, codes.shape[1]))
    assert np.array_equal(q.scale.cpu().numpy(), e["alpha"]) and np.array_equal(q.zero.cpu().numpy(), e["zero"])
    assert np.array_equal(q.rowsum.cpu().numpy(), e["rowsum"])
    if st is not None and x is not None:
        assert np.array_equal(st.float().cpu().numpy(), e["s"])
    if outs:
        assert np.array_equal(yt.float().cpu().numpy(), rounded(e["y"], od))
        assert np.array_equal(vt.float().cpu().numpy(), rounded(e["values"], od))
    # nothing beside the rows is written, inputs stay
    for store, was, width in ((s_store, None, c), (y_store, None, c), (v_store, None, k)):
        if store is not None:
            rest = store.clone()
            rest[lead:lead + n * (width + pad)].view(n, width + pad)[:, :width] = 7.0
            assert (rest == 7.0).all()
    if into != "residual":
        assert torch.equal(r_store, before[0])
    if x is not None and into != "x":
        assert torch.equal(x_store, before[1])


WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 127, 255, 256, 257, 500, 511, 512, 513, 1000, 1024, 2047, 2048, 2056, 2049, 4096, 4100, 5000, 5120, 8192, 8200, 12000,
          16384, 16392, 20000, 28672, 32760, 32768]


@gpu
@pytest.mark.parametrize("c", WIDTHS)
def test_norm_widths(c):
    check_norm(3, c, bits=8)
    check_norm(2, c, norm="layer", xd=F32, rd=F32, od=F32, bits=4, pad=1)
    check_norm(2, c, norm="none", xd=F32, rd=BF16, od=F32, bits=6, lead=1)


@gpu
@pytest.mark.parametrize("c", [c for c in WIDTHS if c >= 7])
def test_norm_widths_through_a_map(c):
    for bits, special, c_out in ((4, 9, None), (6, 3, c + 5), (8, 50, max(1, c - 3))):
        if (c_out or c) <= 32768 and (c + 7) // 8 * 8 + (c_out or c) // special + 1 <= 40448:
            check_norm(2, c, bits=bits, special=special, c_out=c_out, norm=("rms", "layer", "none")[bits // 2 % 3])


@gpu
@pytest.mark.parametrize("norm", list(NORM))
@pytest.mark.parametrize("xd,rd,od", [(BF16, BF16, BF16), (BF16, F32, BF16), (F32, F32, F32), (F32, BF16, F32), (None, BF16, F32), (None, F32, BF16)])
def test_norm_types(norm, xd, rd, od):
    for bits in (4, 6, 8):
        check_norm(17, 776, norm, xd, rd, od, bits, special=11, seed=1)
        check_norm(5, 333, norm, xd, rd, od, bits, seed=2, pad=3, lead=5)


@gpu
def test_norm_one_entry_maps_and_no_copies():
    """A map of computed channels alone; one channel out of many; many out of one."""
    check_norm(4, 200, special=1, bits=4)
    check_norm(4, 2000, special=1, c_out=1, bits=8)
    check_norm(4, 1, special=2, c_out=700, bits=6)


@gpu
@pytest.mark.parametrize("into", ["residual", "x", "none"])
def test_norm_sum_in_place(into):
    check_norm(33, 1032, into=into, special=7)
    check_norm(6, 4096, into=into, xd=F32, rd=F32, od=F32, outs=False)
    check_norm(6, 4099, into=into, pad=5, lead=3)


@gpu
def test_norm_options():
    check_norm(9, 640, norm="layer", shift=False)
    check_norm(9, 640, outs=False)
    check_norm(700, 136, bits=4, special=5, outs=False)
    check_norm(3, 512, eps=0.0)


@gpu
def test_norm_large_values():
    """Quotients beyond the fast rounding's range: a row far from zero with a small spread, without a norm."""
    b = binding()
    n, c = 3, 520
    rng = np.random.default_rng(5)
    r = (1.0e6 + rng.uniform(0, 0.5, (n, c))).astype(np.float32)
    r[1] = -r[1]
    e = expected(None, r, F32, "none", None, None, 0.0, None, 8)
    assert (np.abs(e["zero"]) > 1 << 22).any()
    q, v = b.DeviceQAct(n, c, 8), torch.empty((n, c), device="cuda")
    b.qllm_add_norm_quant(None, torch.from_numpy(r).cuda(), None, 0, None, None, 0.0, q, 8, values_out=v)
    assert np.array_equal(q.codes.cpu().numpy()[:, :c], e["codes"]) and np.array_equal(q.zero.cpu().numpy(), e["zero"])
    assert np.array_equal(v.cpu().numpy(), e["values"])


@gpu
def test_norm_constant_rows_and_rows_that_are_not_finite():
    b = binding()
    n, c = 6, 1000
    r = torch.randn(n, c, device="cuda")
    r[0] = 0.0
    r[2, 17] = float("nan")
    r[4, 999] = float("inf")
    q, y = b.DeviceQAct(n, c, 8), torch.empty_like(r)
    g = torch.ones(c, device="cuda")
    b.qllm_add_norm_quant(None, r, None, 2, g, None, 1e-5, q, 8, y_out=y)
    clean = torch.nan_to_num(r, nan=0.0, posinf=0.0)
    q2, y2 = b.DeviceQAct(n, c, 8), torch.empty_like(r)
    b.qllm_add_norm_quant(None, clean, None, 2, g, None, 1e-5, q2, 8, y_out=y2)
    for i in (0, 1, 3, 5):
        assert torch.equal(q.codes[i], q2.codes[i]) and torch.equal(y[i], y2[i]) and q.scale[i] == q2.scale[i] and q.rowsum[i] == q2.rowsum[i]
    assert q.scale[0] == 1.0 and q.zero[0] == 0 and q.rowsum[0] == 0


@gpu
def test_norm_only():
    """Without codes: the sum and the normalised rows."""
    b = binding()
    for c in (40, 4096, 9000):
        rng = np.random.default_rng(c)
        x, r = draw(rng, 4, c, BF16), draw(rng, 4, c, F32)
        e = expected(x, r, F32, "rms", np.ones(c, np.float32), None, 1e-6, None, 8)
        xt, rt = torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(r).cuda()
        y = torch.empty((4, c), dtype=BF16, device="cuda")
        b.qllm_add_norm_quant(xt, rt, rt, 2, torch.ones(c, device="cuda"), None, 1e-6, y_out=y)
        assert np.array_equal(rt.cpu().numpy(), e["s"]) and np.array_equal(y.float().cpu().numpy(), rounded(e["y"], BF16))


@gpu
def test_norm_feeds_the_layer():
    """What qllm_norm_reassemble_quant makes of the sum, bit for bit, so that qllm_int_gemm takes the codes."""
    b = binding()
    n, c = 70, 1024
    rng = np.random.default_rng(3)
    x, r = torch.from_numpy(draw(rng, n, c, BF16)).cuda().bfloat16(), torch.from_numpy(draw(rng, n, c, BF16)).cuda().bfloat16()
    csr = random_csr_map(rng, c, 1030, 13)
    gamma = torch.from_numpy(rng.uniform(0.5, 1.5, c).astype(np.float32)).cuda()
    for bits in (4, 6, 8):
        two, one = b.DeviceQAct(n, 1030, bits), b.DeviceQAct(n, 1030, bits)
        s = torch.empty_like(x)
        b.qllm_add_norm_quant(x, r, s, 2, gamma, None, 1e-5, one, bits, gather=b.DeviceGather(*csr, c))
        plan = b.qllm_plan_map_host(*csr, c)[0]
        b.qllm_norm_reassemble_quant(s, 2, gamma, None, 1e-5, b.DeviceMap(*csr, c, plan), bits, two)
        for name in ("codes", "scale", "zero", "rowsum"):
            assert torch.equal(getattr(one, name), getattr(two, name)), (bits, name)


@gpu
def test_norm_many_rows():
    """More rows than the card holds at once, each against the same row alone."""
    b = binding()
    n, c = 5000, 264
    x, r = torch.randn(n, c, device="cuda").bfloat16(), torch.randn(n, c, device="cuda").bfloat16()
    g = torch.ones(c, device="cuda")
    q, s = b.DeviceQAct(n, c, 8), torch.empty_like(r)
    b.qllm_add_norm_quant(x, r, s, 2, g, None, 1e-5, q, 8)
    for i in (0, 1, 1023, 2500, 4999):
        one, t = b.DeviceQAct(1, c, 8), torch.empty_like(r[:1])
        b.qllm_add_norm_quant(x[i:i + 1], r[i:i + 1], t, 2, g, None, 1e-5, one, 8)
        assert torch.equal(one.codes[0], q.codes[i]) and torch.equal(t[0], s[i]) and one.scale[0] == q.scale[i] and one.rowsum[0] == q.rowsum[i]


@gpu
def test_norm_as_many_computed_channels_as_fit():
    """The widest row with as many computed channels as there is room for on chip, some of many entries."""
    b = binding()
    c, computed = 32768, 7680
    rng = np.random.default_rng(9)
    count = np.ones(computed, np.int64)
    count[::7], count[5] = 3, 300
    row_ptr = np.concatenate([[0], np.cumsum(count)]).astype(np.int32)
    src, scale = rng.integers(0, c, row_ptr[-1]).astype(np.int32), rng.uniform(-1, 1, row_ptr[-1]).astype(np.float32)
    r = draw(rng, 3, c, BF16)
    e = expected(None, r, BF16, "rms", np.ones(c, np.float32), None, 1e-5, (row_ptr, src, scale), 8)
    q = b.DeviceQAct(3, computed, 8)
    b.qllm_add_norm_quant(None, torch.from_numpy(r).cuda().bfloat16(), None, 2, torch.ones(c, device="cuda"), None, 1e-5, q, 8,
                          gather=b.DeviceGather(row_ptr, src, scale, c))
    assert np.array_equal(q.codes.cpu().numpy()[:, :computed], e["codes"]) and np.array_equal(q.rowsum.cpu().numpy(), e["rowsum"])


@gpu
def test_norm_no_rows():
    b = binding()
    r = torch.empty((0, 64), device="cuda")
    b.qllm_add_norm_quant(r, r, r, 2, torch.ones(64, device="cuda"), None, 1e-5, b.DeviceQAct(0, 64, 8), 8, y_out=r)


FAR = (1 << 31) + 8                                # a row stride whose second row lies past 2^32 bytes of bf16


def far_rows(c, seed):
    """Two rows of c bf16 channels, FAR elements apart."""
    t = torch.empty(FAR + c + 8, dtype=BF16, device="cuda").as_strided((2, c), (FAR, 1))
    return t.copy_(torch.randn((2, c), generator=torch.Generator().manual_seed(seed)))


@gpu
def test_norm_rows_far_apart():
    b = binding()
    c = 1000
    x, r = far_rows(c, 1), far_rows(c, 2)
    g = torch.ones(c, device="cuda")
    q, q2, near = b.DeviceQAct(2, c, 4), b.DeviceQAct(2, c, 4), r.contiguous()
    y = far_rows(c, 3)
    b.qllm_add_norm_quant(x.contiguous(), near, near, 2, g, None, 1e-5, q2, 4)
    b.qllm_add_norm_quant(x, r, r, 2, g, None, 1e-5, q, 4, y_out=y)
    assert torch.equal(q.codes, q2.codes) and torch.equal(r, near) and torch.equal(q.scale, q2.scale)
    assert torch.isfinite(y.float()).all()


@gpu
def test_norm_more_rows_than_a_launch():
    """A launch counts its lanes in 32 bits; the same bits as from calls of a quarter of the rows."""
    b = binding()
    n, c = (1 << 25) + 5, 8
    r, g = torch.randn(n, c, device="cuda", dtype=BF16), torch.ones(c, device="cuda")
    q = b.DeviceQAct(n, c, 4)
    for t in (q.codes, q.scale, q.zero, q.rowsum):
        t.zero_()
    b.qllm_add_norm_quant(None, r, None, 2, g, None, 1e-5, q, 4)
    for i in range(0, n, 1 << 23):
        k = min(1 << 23, n - i)
        part = b.DeviceQAct(k, c, 4)
        b.qllm_add_norm_quant(None, r[i:i + k], None, 2, g, None, 1e-5, part, 4)
        for all_rows, rows in ((q.codes, part.codes), (q.scale, part.scale), (q.zero, part.zero), (q.rowsum, part.rowsum)):
            assert torch.equal(all_rows[i:i + k], rows), i


@gpu
def test_norm_on_two_streams_at_once():
    """Nothing is shared between calls: the same bits beside another call on another stream."""
    b = binding()
    n, c = 900, 2048
    rng = np.random.default_rng(4)
    csr = random_csr_map(rng, c, 2040, 9)
    gather, g = b.DeviceGather(*csr, c), torch.ones(c, device="cuda")
    sets = []
    for k in range(2):
        x, r = (torch.randn(n, c, device="cuda").bfloat16() for _ in range(2))
        sets.append((x, r, torch.empty_like(r), b.DeviceQAct(n, 2040, 6)))
    want = []
    for x, r, s, q in sets:
        b.qllm_add_norm_quant(x, r, s, 2, g, None, 1e-5, q, 6, gather=gather)
        torch.cuda.synchronize()
        want.append((s.clone(), q.codes.clone(), q.rowsum.clone()))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (x, r, s, q), st in zip(sets, streams):
            s.zero_(), q.codes.zero_(), q.rowsum.zero_()
        torch.cuda.synchronize()
        for (x, r, s, q), st in zip(sets, streams):
            b.qllm_add_norm_quant(x, r, s, 2, g, None, 1e-5, q, 6, gather=gather, stream=st)
        torch.cuda.synchronize()
        for (x, r, s, q), w in zip(sets, want):
            assert torch.equal(s, w[0]) and torch.equal(q.codes, w[1]) and torch.equal(q.rowsum, w[2])


# ---------------------------------------------------------------- adapters

U = 2.0 ** -24


def adapters_reference(s, rows):
    """out and its bound, in 64 bits on the host.

    Of h = sum_c A x: the terms are exact (bf16) or rounded once; a wave adds up at most 16 ceil(C / 256) of them or of the matrix
    operations' sums, 4 waves and at most ceil(C / 256) slices follow; each addition may be off by one unit of what has been added up in
    magnitude: (18 ceil(C / 256) + 6) 2 U sum |A x|.  h meets B with 2^-17 of itself left out (two bf16 parts, bf16 B and y) or 2^-24; the
    scale and each of rank / 4 + 4 operations round once; the result is rounded to fp32 and to y's type."""
    x, A, B, y = (s[k].double().cpu().numpy() for k in ("x", "A", "B", "y"))
    scale = np.ones(A.shape[0]) if s["scale"] is None else s["scale"].double().cpu().numpy()
    ranks = [s["rank"]] * A.shape[0] if s["ranks"] is None else np.clip(s["ranks"].cpu().numpy(), 0, s["rank"])
    out, bound = y.copy(), np.zeros_like(y)
    turns = -(-s["c"] // 256)
    left = 2.0 ** -17 if s["B"].dtype == BF16 and s["y"].dtype == BF16 else U
    half = torch.finfo(s["y"].dtype).eps / 2
    for rs, a in rows:
        if not 0 <= a < A.shape[0]:
            continue
        col, k = 0, int(ranks[a])
        for p, o in enumerate(s["parts"]):
            Ap, Bp = A[a, p * s["rank"]:p * s["rank"] + k], B[a, col:col + o, :k]
            h, h_abs = x[rs] @ Ap.T, np.abs(x[rs]) @ np.abs(Ap).T
            h_off = (18 * turns + 6) * 2 * U * h_abs
            d, d_abs = h @ Bp.T * scale[a], np.abs(h) @ np.abs(Bp).T * abs(scale[a])
            out[rs, col:col + o] += d
            off = abs(scale[a]) * (h_off @ np.abs(Bp).T) + (left + (s["rank"] / 4 + 8) * 2 * U) * d_abs
            bound[rs, col:col + o] += off + 2 * U * (np.abs(y[rs, col:col + o]) + d_abs) + half * (np.abs(out[rs, col:col + o]) + off)
            col += o
    return out, bound


def make_adapters(news, names, n_adapters, rank, c, parts, xd=BF16, wd=BF16, yd=BF16, ranks=None, scale=True, pad=0, lead=0, tail=0, seed=0, junk=True):
    """A step of sequences of news[i] rows with adapter names[i]; what lies past an adapter's ranks is NaN."""
    g = torch.Generator().manual_seed(seed)
    rows, o = sum(news) + tail, sum(parts)
    s = dict(c=c, rank=rank, parts=parts, n_adapters=n_adapters, rows=rows)
    s["x"], s["x_store"] = strided(torch.randn((rows, c), generator=g).numpy(), xd, pad, lead)
    s["y"], s["y_store"] = strided(torch.randn((rows, o), generator=g).numpy(), yd, pad, lead)
    A, B = torch.randn((n_adapters, len(parts), rank, c), generator=g) / max(1, c) ** 0.5, torch.randn((n_adapters, o, rank), generator=g)
    s["ranks"] = None if ranks is None else torch.tensor(ranks, dtype=torch.int32).cuda()
    if ranks is not None and junk:
        for a, k in enumerate(ranks):
            A[a, :, max(0, min(k, rank)):] = float("nan")
            B[a, :, max(0, min(k, rank)):] = float("nan")
    s["A"], s["B"] = A.flatten(1, 2).to(wd).cuda(), B.to(wd).cuda()
    s["scale"] = (torch.rand(n_adapters, generator=g) + 0.5).cuda() if scale else None
    starts = np.cumsum([0] + list(news))
    s["row_start"] = torch.tensor(starts, dtype=torch.int32).cuda()
    s["adapter"] = torch.tensor(names, dtype=torch.int32).cuda()
    s["of"] = [(slice(int(starts[i]), int(starts[i + 1])), a) for i, a in enumerate(names)]
    return s


def apply(s, out=None, single=False, stream=None):
    b = binding()
    ad = b.DeviceAdapters(s["A"], s["B"], s["scale"], s["ranks"], s["parts"])
    plan = b.DeviceAdapterPlan(s["rows"], s["n_adapters"])
    b.qllm_adapter_plan(plan, s["adapter"], None if single else s["row_start"])
    ws = torch.full((b.qllm_adapter_workspace_bytes(ad, s["rows"]),), 255, dtype=torch.uint8, device="cuda")   # NaN as float
    out = torch.full_like(s["y"], 3.0) if out is None else out
    b.qllm_adapter_apply(s["x"], ad, plan, s["y"], out, ws)
    torch.cuda.synchronize()
    return out, (ad, plan, ws)


def check_adapters(single=False, **kw):
    s = make_adapters(**kw)
    want, bound = adapters_reference(s, s["of"])
    y_store = s["y_store"].clone()
    out, _ = apply(s, single=single)
    served = sum(kw["news"])
    got = out.double().cpu().numpy()
    assert torch.equal(s["y_store"], y_store)
    assert (out[served:] == 3.0).all()                             # rows of no sequence
    for rs, a in s["of"]:
        if not 0 <= a < s["n_adapters"]:
            assert torch.equal(out[rs], s["y"][rs])                # no adapter: a copy, bit for bit
    off = np.abs(got - want)[:served]
    assert (off <= bound[:served]).all(), (np.nanmax(off / np.maximum(bound[:served], 1e-300)), np.isnan(got[:served]).sum())
    # in place the same bits, and nothing beside the rows and columns
    ys = s["y_store"].clone()
    view = ys.as_strided(s["y"].shape, s["y"].stride(), s["y"].storage_offset())
    t = dict(s, y=view, y_store=ys)
    apply(t, out=view, single=single)
    assert torch.equal(view[:served], out[:served]) and torch.equal(view[served:], s["y"][served:])
    view.copy_(s["y"])
    assert torch.equal(ys, y_store)


@gpu
@pytest.mark.parametrize("c", [1, 7, 8, 16, 17, 63, 64, 65, 100, 255, 256, 257, 500, 1024, 1030, 4096])
def test_adapter_inputs(c):
    check_adapters(news=[1, 3, 20, 0, 70], names=[2, 0, 1, 1, 0], n_adapters=3, rank=16, c=c, parts=[80])
    check_adapters(news=[2, 17], names=[0, 1], n_adapters=2, rank=8, c=c, parts=[33], xd=F32, wd=F32, yd=F32, pad=1, lead=1)


@gpu
@pytest.mark.parametrize("parts", [[1], [2], [15], [16], [64], [65], [255], [256], [257], [700], [64, 64], [5, 300, 1], [256, 17, 256, 40], [1, 1, 1, 1]])
def test_adapter_outputs(parts):
    check_adapters(news=[1, 18, 65], names=[1, 0, 1], n_adapters=2, rank=16, c=130, parts=parts)
    check_adapters(news=[4, 30], names=[1, 0], n_adapters=2, rank=24, c=70, parts=parts, xd=BF16, wd=BF16, yd=F32, pad=3, lead=1)
    check_adapters(news=[4, 30], names=[1, 0], n_adapters=2, rank=8, c=70, parts=parts, xd=F32, wd=F32, yd=F32)


@gpu
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 48, 64, 72, 96, 128, 136, 200, 256])
def test_adapter_ranks(rank):
    own = [0, 1, rank, rank - 1, rank // 2, rank + 9, -3]
    for xd, wd, yd in ((BF16, BF16, BF16), (BF16, BF16, F32), (F32, F32, F32)):
        check_adapters(news=[3, 1, 17, 2, 40, 1, 2], names=[0, 1, 2, 3, 4, 5, 6], n_adapters=7, rank=rank, c=200, parts=[90, 40], xd=xd, wd=wd, yd=yd, ranks=own)


@gpu
@pytest.mark.parametrize("xd", [BF16, F32])
@pytest.mark.parametrize("wd", [BF16, F32])
@pytest.mark.parametrize("yd", [BF16, F32])
def test_adapter_types(xd, wd, yd):
    check_adapters(news=[5, 1, 100, 9], names=[3, -1, 0, 3], n_adapters=4, rank=16, c=333, parts=[129], xd=xd, wd=wd, yd=yd, tail=4, ranks=[16, 5, 7, 12])
    check_adapters(news=[1] * 9, names=[0, 1, 2, 3, 0, 1, 2, 3, 0], n_adapters=4, rank=32, c=512, parts=[128, 128], xd=xd, wd=wd, yd=yd, scale=False, single=True)


@gpu
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 63, 64, 65, 128, 200, 300])
def test_adapter_rows(rows):
    check_adapters(news=[rows], names=[0], n_adapters=1, rank=16, c=300, parts=[70])
    check_adapters(news=[1] * rows, names=[(7 * i) % 5 - 1 for i in range(rows)], n_adapters=4, rank=8, c=520, parts=[70], single=True)
    check_adapters(news=[rows, 0, 3], names=[1, 0, -1], n_adapters=70, rank=8, c=64, parts=[24], yd=F32, tail=2)


@gpu
def test_adapter_none_at_all():
    check_adapters(news=[4, 5], names=[-1, 99], n_adapters=3, rank=8, c=64, parts=[24])
    check_adapters(news=[0, 0], names=[1, 0], n_adapters=3, rank=8, c=64, parts=[24], tail=6)
    check_adapters(news=[], names=[], n_adapters=3, rank=8, c=64, parts=[24], tail=6)


@gpu
def test_adapter_one_row_does_not_spoil_another():
    s = make_adapters(news=[3, 40, 2], names=[0, 0, 1], n_adapters=2, rank=16, c=100, parts=[50])
    clean, _ = apply(s)
    s["x"][1, 5] = float("nan")
    s["x"][20, 7] = float("inf")
    s["B"][1, 3, 2] = float("inf")
    out, _ = apply(s)
    rows = [i for i in range(43) if i not in (1, 20)]
    assert torch.equal(out[rows], clean[rows])
    assert torch.isnan(out[1]).all() and torch.equal(out[43:, 4:], clean[43:, 4:]) and not torch.isfinite(out[43:, 3]).any()


@gpu
def test_adapter_copies_keep_the_sign_of_zero():
    s = make_adapters(news=[2, 2], names=[-1, 0], n_adapters=1, rank=8, c=64, parts=[32], yd=F32, ranks=[0])
    s["y"].fill_(-0.0)
    out, _ = apply(s)
    assert torch.signbit(out).all()


@gpu
def test_adapter_rows_of_a_sequence_do_not_depend_on_the_others():
    """The same bits alone, beside others on the same adapter, and in another order."""
    kw = dict(n_adapters=3, rank=16, c=700, parts=[100])
    a = make_adapters(news=[5, 30, 1, 64], names=[2, 1, 2, 2], **kw)
    out, _ = apply(a)
    b = dict(a, row_start=torch.tensor([0, 5, 35, 36, 100], dtype=torch.int32).cuda(), adapter=torch.tensor([2, 1, -1, -1], dtype=torch.int32).cuda())
    alone, _ = apply(b)
    assert torch.equal(alone[:35], out[:35])
    for _ in range(3):
        again, _ = apply(a)
        assert torch.equal(again, out)


@gpu
def test_adapter_plan_of_contradictory_arrays_reaches_nothing_else():
    """Sequences that overlap, run backwards or past the end, places out of range: every index is checked on the device."""
    s = make_adapters(news=[10, 10, 10], names=[0, 1, 2], n_adapters=3, rank=8, c=64, parts=[24], pad=4, lead=8)
    out_store = torch.full((40 * 40,), 3.0, dtype=BF16, device="cuda")
    out = out_store[100:100 + 30 * 28].view(30, 28)[:, :24]
    for starts in ([0, 30, 0, 30], [-5, 100, 7, 1 << 30], [1 << 30, -(1 << 31), 5, 3], [30, 30, 30, 30]):
        t = dict(s, row_start=torch.tensor(starts, dtype=torch.int32).cuda(), adapter=torch.tensor([1 << 30, -7, 2], dtype=torch.int32).cuda())
        apply(t, out=out)
        rest = out_store.clone()
        rest[100:100 + 30 * 28].view(30, 28)[:, :24] = 3.0
        assert (rest == 3.0).all()


@gpu
def test_adapter_with_another_plan_does_nothing():
    s = make_adapters(news=[4], names=[0], n_adapters=2, rank=8, c=64, parts=[24])
    b = binding()
    ad = b.DeviceAdapters(s["A"], s["B"], s["scale"], s["ranks"], s["parts"])
    ws = torch.empty(b.qllm_adapter_workspace_bytes(ad, 4), dtype=torch.uint8, device="cuda")
    out = torch.full_like(s["y"], 3.0)
    b.qllm_adapter_apply(s["x"], ad, b.DeviceAdapterPlan(4, 2), s["y"], out, ws)      # never filled
    assert (out == 3.0).all()


@gpu
def test_adapter_loaded_into_its_place():
    """Writing a place of the pool is loading an adapter: nothing is kept between calls."""
    s = make_adapters(news=[3, 3], names=[0, 1], n_adapters=2, rank=8, c=64, parts=[24], yd=F32)
    first, (ad, plan, ws) = apply(s)
    s["A"][1], s["B"][1], s["scale"][1] = s["A"][0].clone(), s["B"][0].clone(), s["scale"][0].clone()
    s["x"][3:], s["y"][3:] = s["x"][:3].clone(), s["y"][:3].clone()
    out = torch.empty_like(s["y"])
    binding().qllm_adapter_apply(s["x"], ad, plan, s["y"], out, ws)
    assert torch.equal(out[:3], first[:3]) and torch.equal(out[3:], first[:3])


@gpu
def test_adapter_many_sequences_and_adapters():
    n = 3000
    rng = np.random.default_rng(0)
    names = rng.integers(-1, 700, n).tolist()
    check_adapters(news=[1] * n, names=names, n_adapters=700, rank=8, c=40, parts=[16], single=True)
    news = rng.integers(0, 3, n).tolist()
    check_adapters(news=news, names=names, n_adapters=700, rank=8, c=40, parts=[16], yd=F32, tail=1)


@gpu
@pytest.mark.parametrize("c", [16385, 16640, 20001, 28672, 32768, 32769])
def test_adapter_few_rows_of_long_inputs(c):
    """As many slices as the second product adds up by itself, some of several turns, the last one shorter or none."""
    check_adapters(news=[1, 3], names=[2, 0], n_adapters=3, rank=16, c=c, parts=[72, 40])
    check_adapters(news=[1], names=[0], n_adapters=1, rank=24, c=c, parts=[33], xd=F32, wd=F32, yd=F32)


@gpu
def test_adapter_long_inputs():
    check_adapters(news=[1, 2, 40], names=[0, 1, 1], n_adapters=2, rank=64, c=28672, parts=[64])
    check_adapters(news=[130], names=[1], n_adapters=2, rank=16, c=13824, parts=[40], xd=F32, wd=F32, yd=F32)


@gpu
def test_adapter_largest_pool():
    check_adapters(news=[1] * 40, names=[(i * 997) % 8192 for i in range(39)] + [8191], n_adapters=8192, rank=8, c=24, parts=[16], single=True)


@gpu
def test_adapter_many_rows():
    check_adapters(news=[30000, 1, 0, 9000], names=[1, 0, 0, -1], n_adapters=2, rank=8, c=40, parts=[24], tail=3)


@gpu
def test_adapter_rows_far_apart():
    b = binding()
    s = make_adapters(news=[1, 1], names=[1, 0], n_adapters=2, rank=16, c=300, parts=[200])
    near, (ad, plan, ws) = apply(s)
    x, y, out = far_rows(300, 1), far_rows(200, 2), far_rows(200, 3)
    x.copy_(s["x"]), y.copy_(s["y"])
    b.qllm_adapter_apply(x, ad, plan, y, out, ws)
    assert torch.equal(out, near)
    b.qllm_adapter_apply(x, ad, plan, y, y, ws)
    assert torch.equal(y, near)


@gpu
def test_adapter_on_two_streams_at_once():
    """One plan and one pool, a workspace each."""
    b = binding()
    s = make_adapters(news=[40, 3, 90], names=[0, 1, 2], n_adapters=3, rank=32, c=2000, parts=[500, 300], yd=F32)
    want, (ad, plan, ws) = apply(s)
    sets = [(torch.cuda.Stream(), torch.empty_like(ws), torch.empty_like(want)) for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, w, out in sets:
            b.qllm_adapter_apply(s["x"], ad, plan, s["y"], out, w, stream=st)
        torch.cuda.synchronize()
        for _, _, out in sets:
            assert torch.equal(out, want)
            out.zero_()
        torch.cuda.synchronize()


@gpu
def test_adapter_another_batch_in_a_captured_step():
    """A graph of the plan and the call serves whatever the arrays hold at the replay."""
    b = binding()
    s = make_adapters(news=[1] * 30, names=[0] * 30, n_adapters=4, rank=16, c=256, parts=[128], yd=F32)
    ad = b.DeviceAdapters(s["A"], s["B"], s["scale"], None, s["parts"])
    plan, out = b.DeviceAdapterPlan(30, 4), torch.empty_like(s["y"])
    ws = torch.empty(b.qllm_adapter_workspace_bytes(ad, 30), dtype=torch.uint8, device="cuda")

    def step():
        b.qllm_adapter_plan(plan, s["adapter"])
        b.qllm_adapter_apply(s["x"], ad, plan, s["y"], out, ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        names = [(i * (k + 3) + k) % 6 - 1 for i in range(30)]
        s["adapter"].copy_(torch.tensor(names, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want, bound = adapters_reference(s, [(slice(i, i + 1), a) for i, a in enumerate(names)])
        assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got)


# ---------------------------------------------------------------- together

@gpu
def test_step_between_two_layers_on_a_stream_and_as_a_graph():
    """A layer's output joins the residual, is normalised and quantized, goes through a shared projection and each request's adapter."""
    b = binding()
    n, c, o, bits = 24, 512, 384, 8
    rng = np.random.default_rng(11)
    csr = random_csr_map(rng, c, 520, 17)
    k = 520
    W = rng.standard_normal((c, o)).astype(np.float32) * 0.02
    q = b.qllm_quantize_weight_host(W, csr[0], csr[1], bits)
    dw = b.DeviceWeight(q["codes"], q["scale"], q["zero"], q["colsum"], k, bits)
    gather = b.DeviceGather(*csr, c)
    gamma = torch.from_numpy(rng.uniform(0.5, 1.5, c).astype(np.float32)).cuda()
    x, r = torch.from_numpy(draw(rng, n, c, BF16)).cuda().bfloat16(), torch.from_numpy(draw(rng, n, c, BF16)).cuda().bfloat16()
    s = make_adapters(news=[1] * n, names=[i % 5 - 1 for i in range(n)], n_adapters=4, rank=16, c=c, parts=[256, 128])
    ad = b.DeviceAdapters(s["A"], s["B"], s["scale"], None, s["parts"])
    plan = b.DeviceAdapterPlan(n, 4)
    act, total, normed = b.DeviceQAct(n, k, bits), torch.empty_like(r), torch.empty_like(r)
    y = torch.empty((n, o), dtype=BF16, device="cuda")
    gws = torch.empty(max(16, b.qllm_gemm_workspace_bytes(n, k, o, bits)), dtype=torch.uint8, device="cuda")
    ws = torch.empty(b.qllm_adapter_workspace_bytes(ad, n), dtype=torch.uint8, device="cuda")

    def step():
        b.qllm_adapter_plan(plan, s["adapter"])
        b.qllm_add_norm_quant(x, r, total, 2, gamma, None, 1e-5, act, bits, gather=gather, y_out=normed)
        b.qllm_int_gemm(act, dw, y, workspace=gws)
        b.qllm_adapter_apply(normed, ad, plan, y, y, ws)

    step()
    torch.cuda.synchronize()
    e = expected(x.float().cpu().numpy(), r.float().cpu().numpy(), BF16, "rms", gamma.cpu().numpy(), None, 1e-5, csr, bits)
    acc = e["codes"].astype(np.float64) - e["zero"][:, None]
    wv = orc.unpack_codes(q["codes"], k, bits).astype(np.float64) - q["zero"][:, None]
    base = e["alpha"][:, None].astype(np.float64) * (acc @ wv.T) * q["scale"]
    shared = torch.empty_like(y)
    b.qllm_int_gemm(act, dw, shared, workspace=gws)
    off = np.abs(shared.double().cpu().numpy() - base)
    assert (off <= 2.0 ** -8 * np.abs(base) + 2.0 ** -20 * np.abs(base).max()).all()      # rounded to bf16, behind three roundings to fp32
    want, bound = adapters_reference(dict(s, x=normed, y=shared), s["of"])
    assert (np.abs(y.double().cpu().numpy() - want) <= bound).all()
    eager = [t.clone() for t in (total, normed, act.codes, act.scale, y)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        step()
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(eager, (total, normed, act.codes, act.scale, y)))

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for t in (total, normed, act.codes, y):
            t.zero_()
        x.copy_(x.flip(0)), r.copy_(r.flip(0))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (total, normed, act.codes, act.scale, y)]
        for t in (total, normed, act.codes, y):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(want, (total, normed, act.codes, act.scale, y))), i
    assert all(torch.equal(u, v) for u, v in zip(eager, want))       # flipped an even number of times


# ---------------------------------------------------------------- adapters, sums of whole numbers: every result is one number

def differences(rank, c, o, yd, seed, rows=45):
    """A step whose adapter takes the difference of ranks 2 j and 2 j + 1: h is a whole number of 18 to 23 bits that differs between the
    two in its last few, so out = y + a small whole number.  Three channels are not zero."""
    rng = np.random.default_rng([seed, rank, c])
    s = make_adapters(news=[1, rows - 1], names=[1, 0], n_adapters=2, rank=rank, c=c, parts=[o], yd=yd, scale=False)
    at = [0, c // 2, c - 1]
    x, A = np.zeros((rows, c), np.int64), np.zeros((2, rank, c), np.int64)
    x[:, at] = rng.integers(1, 4, (rows, 3)) * np.array([1 << 13, 1 << 6, 1])
    A[:, ::2, at] = rng.integers(32, 128, (2, rank // 2, 3))
    A[:, 1::2] = A[:, ::2]
    A[:, 1::2, c - 1] = 64 + rng.integers(0, 4, (2, rank // 2))
    A[:, ::2, c - 1] = 64 + rng.integers(0, 4, (2, rank // 2))
    B = np.zeros((2, o, rank), np.int64)
    B[:, :, ::2] = rng.choice([-1, 1], (2, o, rank // 2))
    B[:, :, 1::2] = -B[:, :, ::2]
    y = rng.integers(-4, 5, (rows, o))
    for name, v in (("x", x), ("A", A), ("B", B), ("y", y)):
        s[name].copy_(torch.from_numpy(v.astype(np.float32)))
    h = np.stack([x[n] @ A[1 if n == 0 else 0].T for n in range(rows)])
    return s, y + np.stack([B[1 if n == 0 else 0] @ h[n] for n in range(rows)])


@gpu
@pytest.mark.parametrize("rank", [8, 24, 64, 136, 256])
@pytest.mark.parametrize("yd", [BF16, F32])
def test_adapter_ranks_that_nearly_cancel(rank, yd):
    """What h loses on its way to B shows where two ranks cancel.  Every product and sum here is a whole number below 2^24 times the step
    of its part, so out is the whole number rounded once."""
    for c, o in ((96, 70), (300, 300)):
        s, want = differences(rank, c, o, yd, seed=1)
        out, _ = apply(s)
        assert torch.equal(out.cpu(), torch.from_numpy(want.astype(np.float32)).to(yd))


@gpu
@pytest.mark.parametrize("wd", [BF16, F32])
@pytest.mark.parametrize("yd", [BF16, F32])
def test_adapter_sums_near_the_largest_float(wd, yd):
    """h between the largest bf16 and the largest fp32 number, either sign, against a small B: x's only channel times 2^-100, once rounded."""
    s = make_adapters(news=[1, 40], names=[0, 0], n_adapters=1, rank=8, c=70, parts=[33], xd=F32, wd=wd, yd=yd, scale=False, ranks=[1], junk=False)
    for name in ("x", "A", "B", "y"):
        s[name].zero_()
    top = torch.tensor(np.linspace(3.3896e38, 3.4028e38, 41).astype(np.float32)) * torch.tensor([1.0, -1.0]).repeat(21)[:41]
    s["x"][:, 69], s["A"][0, 0, 69], s["B"][0, :, 0] = top.cuda(), 1.0, 2.0 ** -100
    out, _ = apply(s)
    assert torch.equal(out.cpu(), (top.double() * 2.0 ** -100).to(yd)[:, None].expand(41, 33))


def whole_numbers(rows, n_adapters, rank, c, o, seed):
    """x, A, B and y of small whole numbers, none of x, A and B 0, so that every sum is a whole number below 2^24, exact in whatever order
    it is made, and one channel that is left out of it shows.  A [adapters, rank, c]."""
    assert 3 * 3 * 2 * 2 * c * rank < 1 << 24
    rng = np.random.default_rng([seed, rows, rank, c, o])
    sign = lambda *s: rng.choice([-1, 1], s)  # noqa: E731
    return (sign(rows, c) * rng.integers(1, 4, (rows, c)), sign(n_adapters, rank, c) * rng.integers(1, 4, (n_adapters, rank, c)),
            sign(n_adapters, o, rank) * rng.integers(1, 3, (n_adapters, o, rank)), rng.integers(-9, 10, (rows, o)))


def whole_result(x, A, B, y, of, without=None):
    """out, exact: of: (rows, adapter) pairs, adapter a's scale 1 + a % 2; without: a channel that is left out."""
    out = y.astype(np.float64)
    for rs, a in of:
        if 0 <= a < A.shape[0]:
            xa, Aa = x[rs].astype(np.float64), A[a].astype(np.float64)
            if without is not None:
                xa[:, without] = 0.0
            out[rs] += (1 + a % 2) * (xa @ Aa.T) @ B[a].astype(np.float64).T
    return out


def check_whole_numbers(news, names, n_adapters, rank, c, o, xd=BF16, wd=BF16, yd=F32, seed=0, **kw):
    s = make_adapters(news=news, names=names, n_adapters=n_adapters, rank=rank, c=c, parts=[o], xd=xd, wd=wd, yd=yd, **kw)
    x, A, B, y = whole_numbers(sum(news), n_adapters, rank, c, o, seed)
    for name, v in (("x", x), ("A", A), ("B", B), ("y", y)):
        s[name].copy_(torch.from_numpy(v.astype(np.float32)))
    s["scale"].copy_(torch.tensor([1.0 + a % 2 for a in range(n_adapters)]))
    out, _ = apply(s)
    assert torch.equal(out.cpu(), torch.from_numpy(whole_result(x, A, B, y, s["of"])).to(yd))


LONG = [1, 9, 63, 65, 255, 257, 1025, 4097, 8193, 16385, 16640, 20001, 28672, 32768, 32769]


@gpu
@pytest.mark.parametrize("c", LONG)
def test_adapter_whole_numbers(c):
    """Equality, however long the inputs: the last slice of one channel, one wave's last block, a slice of the sum are each seen."""
    for yd in (F32, BF16):
        check_whole_numbers([1, 3], [2, 1], 3, 8, c, 40, yd=yd)
        check_whole_numbers([1], [0], 1, 8, c, 33, xd=F32, wd=F32, yd=yd, pad=1, lead=1)
        check_whole_numbers([2, 17], [0, 1], 2, 8, c, 24, xd=F32, wd=BF16, yd=yd)
        check_whole_numbers([70, 40, 1], [1, 0, 1], 2, 8, c, 24, yd=yd)
        check_whole_numbers([70, 2], [1, 0], 2, 8, c, 24, xd=F32, wd=F32, yd=yd)


@gpu
@pytest.mark.parametrize("rank", [16, 40, 64])
def test_adapter_whole_numbers_of_more_ranks(rank):
    for c in (4097, 7169):
        check_whole_numbers([1, 9], [1, 0], 2, rank, c, 40)
        check_whole_numbers([80], [0], 2, rank, c, 40, xd=F32, wd=F32)


@gpu
def test_norm_rows_far_apart_of_every_output():
    """The normalised rows and what the codes stand for, with rows past 2^32 bytes apart, are those of rows next to each other."""
    b = binding()
    c, k = 1000, 1003
    rng = np.random.default_rng(8)
    csr = random_csr_map(rng, c, k, 9)
    x, r, g = far_rows(c, 1), far_rows(c, 2), torch.rand(c, device="cuda") + 0.5
    for gather, n in ((None, c), (b.DeviceGather(*csr, c), k)):
        near = dict(s=torch.empty((2, c), dtype=BF16, device="cuda"), y=torch.empty((2, c), dtype=BF16, device="cuda"), v=torch.empty((2, n), dtype=BF16, device="cuda"))
        far = dict(s=far_rows(c, 3), y=far_rows(c, 4), v=far_rows(n, 5))
        q = b.DeviceQAct(2, n, 8), b.DeviceQAct(2, n, 8)
        for t in far.values():
            t.fill_(float("nan"))
        b.qllm_add_norm_quant(x.contiguous(), r.contiguous(), near["s"], 2, g, None, 1e-5, q[0], 8, gather=gather, y_out=near["y"], values_out=near["v"])
        b.qllm_add_norm_quant(x, r, far["s"], 2, g, None, 1e-5, q[1], 8, gather=gather, y_out=far["y"], values_out=far["v"])
        for name in far:
            assert torch.equal(far[name], near[name]), name
        assert torch.equal(q[0].codes, q[1].codes) and torch.equal(q[0].rowsum, q[1].rowsum)
        del far


@gpu
@pytest.mark.parametrize("yd", [BF16, F32])
def test_adapter_sequences_in_another_order(yd):
    """The same sequences in another order of rows: each row's bits are the same."""
    news, names = [5, 30, 1, 64, 2, 17, 90], [2, 1, 2, 2, -1, 0, 1]
    s = make_adapters(news=news, names=names, n_adapters=3, rank=16, c=700, parts=[100, 60], yd=yd, ranks=[16, 9, 3])
    out, _ = apply(s)
    rows = [list(range(sum(news[:i]), sum(news[:i + 1]))) for i in range(len(news))]
    for order in ([6, 5, 4, 3, 2, 1, 0], [3, 0, 6, 1, 5, 2, 4], [2, 3, 0, 4, 1, 6, 5]):
        at = torch.tensor([n for i in order for n in rows[i]], device="cuda")
        starts = np.cumsum([0] + [news[i] for i in order])
        moved, _ = apply(dict(s, x=s["x"][at], y=s["y"][at], row_start=torch.tensor(starts, dtype=torch.int32).cuda(),
                              adapter=torch.tensor([names[i] for i in order], dtype=torch.int32).cuda()))
        assert torch.equal(moved, out[at]), order


def guarded(size):
    """Exactly `size` bytes between two guards of 4096, all of one pattern; the bytes and a check of the guards."""
    store = torch.full((size + 8192,), 0xA5, dtype=torch.uint8, device="cuda")

    def kept():
        return bool((store[:4096] == 0xA5).all()) and bool((store[4096 + size:] == 0xA5).all())

    return store[4096:4096 + size], kept


def apply_guarded(s, out, single=False):
    """apply() with a plan and a workspace of exactly the bytes asked for, through the C entries; both hold whatever was there before."""
    b = binding()
    ad = b.DeviceAdapters(s["A"], s["B"], s["scale"], s["ranks"], s["parts"])
    rows, here = s["rows"], torch.cuda.current_stream().cuda_stream
    plan, plan_kept = guarded(b.qllm_adapter_plan_bytes(rows, s["n_adapters"]))
    ws, ws_kept = guarded(b.qllm_adapter_workspace_bytes(ad, rows))
    code = {F32: b.F32, BF16: b.BF16}
    for _ in range(2):
        assert 0 == b.raw().qllm_adapter_plan(rows, s["adapter"].numel(), None if single else s["row_start"].data_ptr(), s["adapter"].data_ptr(), s["n_adapters"],
                                              plan.data_ptr(), plan.numel(), here)
        assert 0 == b.raw().qllm_adapter_apply(s["x"].data_ptr(), code[s["x"].dtype], s["x"].stride(0), rows, ad.ref, plan.data_ptr(), plan.numel(),
                                               s["y"].data_ptr(), s["y"].stride(0), out.data_ptr(), out.stride(0), code[s["y"].dtype], ws.data_ptr(), ws.numel(), here)
        torch.cuda.synchronize()
        assert plan_kept() and ws_kept()
    return out


@gpu
def test_adapter_guards_of_plan_and_workspace():
    """Many slices, many adapters, many ranks, many rows, one row: nothing is written beside the bytes that the sizes name."""
    for kw, single in ((dict(news=[1] * 16, names=[i % 3 for i in range(16)], n_adapters=3, rank=24, c=32768, parts=[40]), True),
                       (dict(news=[3, 1], names=[0, 1], n_adapters=2, rank=8, c=200001, parts=[24], xd=F32, wd=F32, yd=F32), False),
                       (dict(news=[1] * 40, names=[(i * 997) % 8192 for i in range(40)], n_adapters=8192, rank=8, c=24, parts=[16]), True),
                       (dict(news=[65, 64, 63, 1], names=[0, 1, 2, 0], n_adapters=3, rank=256, c=4096, parts=[24, 24]), False),
                       (dict(news=[1000, 3000, 200], names=[1, 0, 5], n_adapters=2, rank=16, c=5000, parts=[24], tail=3), False),
                       (dict(news=[1], names=[0], n_adapters=1, rank=8, c=1, parts=[1]), True)):
        s = make_adapters(**kw)
        want, _ = apply(s, single=single)
        assert torch.equal(apply_guarded(s, torch.full_like(s["y"], 3.0), single=single), want)


@gpu
@pytest.mark.parametrize("starts", [[0, 30, 0, 30], [-5, 100, 7, 1 << 30], [1 << 30, -(1 << 31), 5, 3], [30, 30, 30, 30], [0, 70, 0, 70], [-1, -1, 70, 0]])
def test_adapter_guards_with_contradictory_arrays(starts):
    for names in ([1 << 30, -7, 2], [0, 0, 0], [2, 1, 2]):
        s = make_adapters(news=[10, 10, 10], names=[0, 1, 2], n_adapters=3, rank=8, c=70, parts=[24], pad=4, lead=8)
        s = dict(s, row_start=torch.tensor(starts, dtype=torch.int32).cuda(), adapter=torch.tensor(names, dtype=torch.int32).cuda())
        out_store = torch.full((40 * 40,), 3.0, dtype=BF16, device="cuda")
        out = out_store[100:100 + 30 * 28].view(30, 28)[:, :24]
        apply_guarded(s, out)
        out.fill_(3.0)
        assert (out_store == 3.0).all()


@gpu
def test_adapter_guards_with_many_sequences_on_the_same_rows():
    """3000 sequences of all rows each, on one adapter and on many: every count and place goes past what the plan has room for."""
    n = 3000
    s = make_adapters(news=[100], names=[0], n_adapters=50, rank=8, c=40, parts=[16], yd=F32)
    starts = torch.tensor([0, 100] * (n // 2) + [0], dtype=torch.int32).cuda()
    for names in ([7] * n, [i % 50 for i in range(n)]):
        t = dict(s, row_start=starts, adapter=torch.tensor(names, dtype=torch.int32).cuda())
        out = apply_guarded(t, torch.full_like(s["y"], 3.0))
        assert torch.isfinite(out).all()


def whole_step(rows, n_adapters, rank, c, parts, yd, a_of, seed=0, live=None):
    """A step made on the device, a row a sequence, of small whole numbers as above; live: the channels of x that are not 0 (None: all).
    a_of: each row's adapter."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    one = lambda most, *s: (torch.randint(1, most + 1, s, generator=g, device="cuda", dtype=torch.int8) * (2 * torch.randint(0, 2, s, generator=g, device="cuda", dtype=torch.int8) - 1)).to(BF16)  # noqa: E731
    o = sum(parts)
    x = one(3, rows, c)
    if live is not None:
        keep = torch.zeros(c, dtype=torch.bool, device="cuda")
        keep[live] = True
        x *= keep
    A, B = one(3, n_adapters, len(parts) * rank, c), torch.empty((n_adapters, o, rank), dtype=BF16, device="cuda")
    for a in range(n_adapters):
        B[a] = one(2, o, rank)
    return dict(x=x, A=A, B=B, y=one(9, rows, o).to(yd), scale=None, ranks=None, parts=parts, rank=rank, n_adapters=n_adapters, rows=rows, c=c,
                adapter=torch.tensor(a_of, dtype=torch.int32).cuda())


def check_whole_step(s, live=None):
    """In place, against products in 64 bits, a row at a time where rows are long."""
    y = s["y"].clone()
    apply(s, out=s["y"], single=True)
    at = slice(None) if live is None else live
    o = sum(s["parts"])
    for a in sorted(set(s["adapter"].tolist())):
        rows = torch.nonzero(s["adapter"] == a)[:, 0]
        for some in rows.split(max(1, (1 << 25) // o)):
            want = y[some].double()
            if 0 <= a < s["n_adapters"]:
                col = 0
                for p, width in enumerate(s["parts"]):
                    h = s["x"][some][:, at].double() @ s["A"][a, p * s["rank"]:(p + 1) * s["rank"]][:, at].double().T.contiguous()
                    want[:, col:col + width] += h @ s["B"][a, col:col + width].double().T.contiguous()
                    col += width
            assert torch.equal(s["y"][some], want.to(y.dtype)), a


@gpu
@pytest.mark.parametrize("yd", [BF16, F32])
@pytest.mark.parametrize("rows,parts", [(256, [4096, 4096, 4096]), (256, [4095, 2, 8190]), (4200, [13824, 13824]), (4200, [27000]), (1100, [12288, 1]), (60, [40000])])
def test_adapter_blocks_of_many_columns(rows, parts, yd):
    """Workgroups of the second product that take more than 256 columns, in tiles of few and of many rows, of whole and of other widths."""
    few = [(i * 7) % 17 - 1 for i in range(rows)] if rows <= 256 else [i // 1500 for i in range(rows)]
    s = whole_step(rows, 16 if rows <= 256 else 2, 16, 72, parts, yd, few)
    check_whole_step(s)


@gpu
def test_adapter_more_slices_than_the_short_division_takes():
    """4 tiles of 32768 slices of the longest input: 2^32 and more in the product that the multiplication in place of a division stands for."""
    c = (1 << 24) - 1
    live = torch.tensor([0, 1, 63, 255, 256, 511, 512, 513, 8191, 1 << 20, (1 << 23) + 5, c - 513, c - 256, c - 255, c - 2, c - 1], device="cuda")
    s = whole_step(5, 4, 8, c, [40], F32, [3, 1, -1, 0, 2], live=live)
    check_whole_step(s, live)


@gpu
def test_adapter_more_columns_than_the_short_division_takes():
    """65 tiles of 8192 blocks of 2048 columns: as above, for the second product."""
    s = whole_step(64, 63, 8, 16, [(1 << 24) - 1], BF16, list(range(63)) + [-1])
    check_whole_step(s)
    torch.cuda.empty_cache()


@gpu
def test_adapter_sums_near_the_smallest_float():
    """h of 24 bits whose last one is the smallest bf16 number, 2^-133: all of them reach B; of h below, what is 2^-133 and more."""
    s = make_adapters(news=[1, 40], names=[0, 0], n_adapters=1, rank=8, c=70, parts=[33], xd=F32, yd=F32, scale=False, ranks=[1], junk=False)
    for name in ("x", "A", "B", "y"):
        s[name].zero_()
    s["A"][0, 0, 69], s["B"][0, :, 0] = 1.0, 2.0 ** 100
    for lowest, most in ((1 << 23, 1 << 24), (1, 1 << 16)):
        h = torch.from_numpy(np.random.default_rng(0).integers(lowest, most, 41).astype(np.float64) * 2.0 ** -133)
        s["x"][:, 69] = h.float().cuda()
        out, _ = apply(s)
        assert torch.equal(out.cpu(), (h * 2.0 ** 100).float()[:, None].expand(41, 33))


@gpu
def test_norm_without_x_leaves_sum_out():
    """Nothing is added, and sum_out is not written."""
    b = binding()
    r, s = torch.randn(5, 300, device="cuda"), torch.full((5, 300), 7.0, device="cuda")
    q, w = b.DeviceQAct(5, 300, 8), b.DeviceQAct(5, 300, 8)
    g = torch.ones(300, device="cuda")
    b.qllm_add_norm_quant(None, r, s, 2, g, None, 1e-5, q, 8)
    b.qllm_add_norm_quant(None, r, None, 2, g, None, 1e-5, w, 8)
    assert (s == 7.0).all() and torch.equal(q.codes, w.codes) and torch.equal(q.scale, w.scale)
