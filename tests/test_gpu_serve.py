"""Serving-layer operators on the GPU against their plain forms in 64 bits."""
import math

import pytest
import torch

from paper_2504_18547_amd import vitq
from tests import serve_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16, F8 = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _codes(m):
    return m.data[:, :m.cols].contiguous().view(F8).cpu().double()


def _within(got, want, bound, what=""):
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = got == want
    off = torch.where(same | torch.isnan(want), torch.zeros_like(want), (got - want).abs())
    bad = ~(off <= bound) & ~torch.isnan(want)
    assert not bool(bad.any()), "%s: %d of %d outside, worst %g against %g" % (
        what, int(bad.sum()), bad.numel(), float(off.max()), float(bound[bad].max()) if torch.is_tensor(bound) else bound)


# ---- quantizer ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 7), (17, 129), (128, 128), (130, 257), (257, 1000), (16, 4096)])
def test_quantize_codes_and_scales(rows, cols, dtype, block_rows):
    x = (torch.randn(rows, cols, generator=_gen(rows * 7 + cols)) * 3).to(dtype)
    m = vitq.FMat.empty(rows, cols, block_rows)
    m.data.fill_(0xA5)
    vitq.vq_quantize_e4m3(x.cuda(), m)
    codes, scales = ref.quantize(x, block_rows)
    assert torch.equal(_codes(m), codes)
    assert torch.equal(m.scales.cpu(), scales)
    assert not bool(m.data[:, cols:].any())                          # the padding of a row is written as zeros


def test_quantize_many_blocks_and_strides():
    big = torch.randn(700, 33 * 130, generator=_gen(5)).to(BF16).cuda()
    for view in (big, big[:, 1:-2], big[::3, :4000], big[:, ::2].contiguous()[:, 3:]):
        m = vitq.FMat.empty(view.shape[0], view.shape[1], 1)
        vitq.vq_quantize_e4m3(view, m)
        codes, scales = ref.quantize(view.cpu(), 1)
        assert torch.equal(_codes(m), codes) and torch.equal(m.scales.cpu(), scales)
    wide = torch.randn(2100, 4 * 2048, generator=_gen(6)).cuda()      # past the size where a workgroup takes four blocks
    m = vitq.FMat.empty(2100, 8192, 1)
    vitq.vq_quantize_e4m3(wide, m)
    at = torch.tensor([0, 1, 1000, 2099])
    codes, scales = ref.quantize(wide.cpu()[at], 1)
    assert torch.equal(_codes(m)[at], codes) and torch.equal(m.scales.cpu()[:, at], scales)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_extreme_values(block_rows):
    x = torch.zeros(5, 128 * 6)
    x[0, 0:128] = torch.linspace(-1, 1, 128)
    x[1, 128:256] = 1e-38                                            # below the smallest scale
    x[2, 256] = 3.0e38
    x[2, 257] = 1.0
    x[3, 384:512] = 1.0
    x[3, 390] = float("nan")
    x[4, 512] = float("inf")
    x[4, 513] = -2.0
    x[0, 640:768] = torch.arange(128) * 448.0 / 127                  # ties and every binade
    m = vitq.FMat.empty(5, x.shape[1], block_rows)
    vitq.vq_quantize_e4m3(x.cuda(), m)
    got, scales = _codes(m), m.scales.cpu()
    rows = 5 if block_rows == 1 else 1
    for j in range(6):
        for i in range(rows):
            at = (slice(i, i + 1) if block_rows == 1 else slice(0, 5), slice(j * 128, j * 128 + 128))
            b, g, s = x[at], got[at], float(scales[j, i])
            if torch.isnan(b).any():
                assert math.isnan(s) and bool(torch.isnan(g).all())
            elif torch.isinf(b).any():
                assert math.isinf(s) and bool((g[~torch.isinf(b)] == 0).all()) and bool(torch.isnan(g[torch.isinf(b)]).all())
            else:
                codes, want = ref.quantize(b, 128 if block_rows == 128 else 1)
                assert torch.equal(g, codes) and s == float(want[0, 0])


# ---- linear -----------------------------------------------------------------------------------------------------

def _coded(x, block_rows, extra=0):
    """FMat of the reference's codes with `extra` more bytes per row than it needs."""
    codes, scales = ref.quantize(x, block_rows)
    stride = (x.shape[1] + 15) // 16 * 16
    data = torch.zeros(x.shape[0], stride, dtype=torch.uint8)
    data[:, :x.shape[1]] = codes.float().to(F8).view(torch.uint8)
    if extra:
        data = torch.cat((data, torch.full((x.shape[0], extra), 0x7E, dtype=torch.uint8)), dim=1)
    return vitq.FMat(data.cuda(), scales.cuda(), x.shape[1], block_rows), ref.dequantize(codes, scales, block_rows)


def _check_linear(M, K, N, out, act, bias, seed=0, extra=0, pad=0):
    g = _gen(seed + M * 31 + K * 7 + N)
    x = torch.randn(M, K, generator=g) * (1 + 10 * (torch.rand(K, generator=g) < 0.02))
    w = torch.randn(N, K, generator=g) * 0.05
    xm, xd = _coded(x, 1, extra)
    wm, wd = _coded(w, 128, extra)
    b = torch.randn(N, generator=g) if bias else None
    room = torch.full((M, N + pad), 7.0, dtype=out, device="cuda")
    y = room[:, :N]
    vitq.vq_linear_e4m3(xm, wm, b.cuda() if bias else None, act, y)
    want, size, peak = ref.linear(xd, wd, b, act)
    _within(y, want, ref.linear_bound(want, size, peak, K, out), "linear %d %d %d" % (M, K, N))
    assert bool((room[:, N:] == 7.0).all())
    return xm, wm, y


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 128, 16), (1, 4096, 256), (2, 100, 33), (16, 384, 130), (17, 256, 128),
                                   (33, 129, 65), (64, 1024, 512), (100, 640, 384), (197, 384, 1152), (130, 257, 259),
                                   (300, 1000, 1001)])
def test_linear_sizes(M, K, N, out):
    _check_linear(M, K, N, out, act=0, bias=True)


@pytest.mark.parametrize("M,K,N", [(5, 200, 48), (128, 128, 128), (256, 512, 256), (385, 896, 640), (777, 300, 515)])
def test_linear_gelu_strides(M, K, N):
    _check_linear(M, K, N, BF16, act=1, bias=True, extra=48, pad=3)
    _check_linear(M, K, N, F32, act=1, bias=False, extra=0, pad=8)
    _check_linear(M, K, N, F16, act=0, bias=False, extra=16, pad=4)


@pytest.mark.parametrize("M,K,N", [(2048, 512, 1024), (1000, 2048, 1100), (4096, 256, 4096), (520, 8192, 300)])
def test_linear_large_sampled(M, K, N):
    """Sizes of the tiled forms, checked on sampled rows and columns against 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda") * 0.05
    xm, wm = vitq.FMat.empty(M, K, 1), vitq.FMat.empty(N, K, 128)
    vitq.vq_quantize_e4m3(x, xm)
    vitq.vq_quantize_e4m3(w, wm)
    b = torch.randn(N, generator=g, device="cuda")
    xd = ref.dequantize(_codes(xm), xm.scales.cpu(), 1)
    wd = ref.dequantize(_codes(wm), wm.scales.cpu(), 128)
    rows = torch.unique(torch.cat((torch.arange(0, M, max(1, M // 97)), torch.tensor([M - 1]))))
    want, size, peak = ref.linear(xd[rows], wd, b.cpu(), 0)
    for out in (F32, BF16):
        y = torch.full((M, N), float("nan"), dtype=out, device="cuda")
        vitq.vq_linear_e4m3(xm, wm, b, 0, y)
        _within(y[rows.cuda()], want, ref.linear_bound(want, size, peak, K, out), "large")
        assert not bool(torch.isnan(y).any())
        again = torch.empty_like(y)
        vitq.vq_linear_e4m3(xm, wm, b, 0, again)
        assert torch.equal(y, again)


def test_linear_empty_and_nan():
    xm, _ = _coded(torch.randn(4, 256, generator=_gen(1)), 1)
    wm, _ = _coded(torch.randn(32, 256, generator=_gen(2)), 128)
    y = torch.full((0, 32), 1.0, device="cuda")
    vitq.vq_linear_e4m3(vitq.FMat.empty(0, 256, 1), wm, None, 0, y)
    xm.data[1, 3] = 0x7F
    xm.scales[1, 2] = float("inf")
    y = torch.empty(4, 32, device="cuda")
    vitq.vq_linear_e4m3(xm, wm, None, 0, y)
    y = y.cpu()
    assert bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[2]).any()) and bool(torch.isfinite(y[[0, 3]]).all())


# ---- norm + rotation + append ---------------------------------------------------------------------------------------

def _check_rotate(T, Hq, Hk, D, dtype=BF16, cache=BF16, norm="rms", rot=None, interleaved=False, page=16, layout=0,
                  per_head=False, seed=0, pad=0):
    g = _gen(seed + T * 11 + D + Hq)
    rot = D if rot is None else rot
    width = (Hq + 2 * Hk) * D
    room = (torch.randn(T, width + pad, generator=g) * 2 + 0.3).to(dtype)
    qkv = room.cuda()[:, :width]
    rows = max(4 * T, 64)
    angle = torch.rand(rows, max(rot // 2, 1), generator=g) * 6.3
    cos, sin = (angle.cos().cuda(), angle.sin().cuda()) if rot else (None, None)
    pos = torch.randint(0, rows, (T,), generator=g).int()
    gam = [1 + 0.3 * torch.randn(h, D, generator=g) if per_head else 1 + 0.3 * torch.randn(D, generator=g) for h in (Hq, Hk)]
    bet = [0.2 * torch.randn_like(t) for t in gam] if norm == "layer" else [None, None]
    pages = -(-T // page) + 2
    slots = torch.randperm(pages * page, generator=g)[:T]
    if T > 3:
        slots[T // 2] = -1
        slots[1] = pages * page
        if rot:
            pos[2] = rows
    fresh = lambda: torch.randint(0, 100, (pages, Hk, page, D) if layout == 0 else (pages, page, Hk, D), generator=g).to(torch.uint8)
    store = [fresh().float().to(cache) for _ in range(2)]
    kd, vd = [(t.cuda() if layout == 0 else t.cuda().transpose(1, 2)) for t in store]
    unit = 0.05 if cache == F8 else 1.0
    c = vitq.KvCache(kd, vd, unit, 2 * unit if cache == F8 else 1.0)
    up = lambda t: None if t is None else t.cuda()
    desc = vitq.make_rotate_desc(Hq, Hk, D, norm, *(up(t) if norm != "none" else None for t in (gam[0], bet[0], gam[1], bet[1])), 1e-5,
                                 cos, sin, interleaved)
    q_type = F16 if dtype == F16 else BF16
    q_room = torch.full((T, Hq * D + 8), 5.0, dtype=q_type, device="cuda")
    vitq.vq_qkv_norm_rotate(desc, qkv, pos.cuda(), q_room[:, :Hq * D], c, slots.cuda())

    x = room[:, :width].double().view(T, Hq + 2 * Hk, D)
    ok = torch.ones(T, dtype=torch.bool) if not rot else (pos >= 0) & (pos < rows)
    at = pos.long().clamp(0, rows - 1)
    args = lambda i: (norm, gam[i], bet[i], 1e-5, cos.cpu()[at] if rot else None, sin.cpu()[at] if rot else None, interleaved)
    q, qs = ref.norm_rotate(x[:, :Hq], *args(0))
    k, ks = ref.norm_rotate(x[:, Hq:Hq + Hk], *args(1))
    v = x[:, Hq + Hk:]
    # fewer than 2^3 roundings of 2^-24 each on the statistics' way, sums of D squares among them (2^-24 D / 2 relative)
    slack = 2.0 ** -20 + D * 2.0 ** -24
    got = q_room[:, :Hq * D].cpu().double().view(T, Hq, D)
    _within(got[ok], q[ok], ref.HALF[q_type] * q[ok].abs() + slack * qs[ok] + ref.tiny(q_type), "q")
    assert bool((q_room[:, Hq * D:] == 5.0).all()) and bool((got[~ok] == 5.0).all())
    write = ok & (slots >= 0) & (slots < pages * page)
    for name, dev, raw, val, size, u in (("k", kd, store[0], k, ks, unit), ("v", vd, store[1], v, v.abs(), c._c.v_scale)):
        raw = (raw if layout == 0 else raw.transpose(1, 2)).double()
        want, bound = raw.clone(), torch.zeros_like(raw)
        t, e = (val / u), (size / u)
        if cache == F8:
            t = t.clamp(-448, 448)
        pg, pl = slots[write] // page, slots[write] % page
        want[pg, :, pl] = t[write]
        small = 2.0 ** -10 if cache == F8 else ref.tiny(cache)
        bound[pg, :, pl] = ref.HALF[cache] * t[write].abs() + (slack if name == "k" or cache == F8 else 0) * e[write] + small
        _within(dev.cpu().double(), want, bound, name)
    return desc, qkv, pos.cuda(), c, slots.cuda()


@pytest.mark.parametrize("T,Hq,Hk,D", [(1, 32, 8, 128), (1, 1, 1, 8), (5, 7, 1, 64), (33, 12, 12, 64), (70, 28, 4, 128),
                                       (3, 6, 2, 256), (9, 5, 5, 80), (130, 16, 2, 96), (900, 32, 8, 128)])
def test_rotate_heads(T, Hq, Hk, D):
    _check_rotate(T, Hq, Hk, D, rot=D // 16 * 16)


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("dtype,cache", [(F32, BF16), (F32, F8), (BF16, F8), (F16, F16), (F16, F8), (BF16, F16)])
def test_rotate_types(dtype, cache, norm):
    _check_rotate(21, 6, 2, 64, dtype, cache, norm, rot=32, interleaved=True, page=7, layout=1)
    _check_rotate(21, 4, 4, 128, dtype, cache, norm, rot=96, page=64, per_head=norm != "none", pad=16)
    _check_rotate(2, 4, 4, 128, dtype, cache, norm, rot=0)


def test_rotate_outputs_on_request():
    desc, qkv, pos, c, slots = _check_rotate(6, 4, 2, 64)
    k0 = c.k.clone()
    q = torch.empty(6, 4 * 64, dtype=BF16, device="cuda")
    vitq.vq_qkv_norm_rotate(desc, qkv, pos, q, None, None)
    assert torch.equal(c.k, k0)
    c.k.zero_()
    vitq.vq_qkv_norm_rotate(desc, qkv, pos, None, c, slots)
    written = (k0 != 0).any(dim=(1, 3)) & (c.k != 0).any(dim=(1, 3))
    assert bool(written.any()) and torch.equal(c.k.transpose(1, 2)[written], k0.transpose(1, 2)[written])


def test_rotate_limits_to_the_largest_code():
    D = 64
    qkv = torch.zeros(2, 3 * D, dtype=F32)
    qkv[:, 2 * D:] = torch.linspace(-1000, 1000, D)
    qkv[1, 2 * D + 5] = float("nan")
    k = torch.zeros(1, 1, 16, D, dtype=torch.float32, device="cuda").to(F8)
    c = vitq.KvCache(k, k.clone(), 1.0, 1.0)
    desc = vitq.make_rotate_desc(1, 1, D, "none")
    vitq.vq_qkv_norm_rotate(desc, qkv.cuda(), None, None, c, torch.tensor([3, 4]).cuda())
    got = c.v[0, 0, 3:5].cpu().double()
    want = ref.e4m3_round(qkv[:, 2 * D:].double().clamp(-448, 448))
    assert torch.equal(got[0], want[0]) and math.isnan(float(got[1, 5])) and torch.equal(got[1, 6:], want[1, 6:])


# ---- attention over the pages -----------------------------------------------------------------------------------------

def _paged(lengths, Hq, Hk, D, dtype, cache, page, layout, seed, spare=2, bad=()):
    """Device inputs and their doubles: q, offsets, lens, table, cache object, per-sequence keys and values."""
    g = _gen(seed)
    T = sum(n for n, _ in lengths)
    q = torch.randn(T, Hq * D, generator=g).to(dtype)
    per = [-(-n // page) for _, n in lengths]
    pages = sum(per) + spare
    unit = 0.05 if cache == F8 else 1.0
    shape = (pages, Hk, page, D) if layout == 0 else (pages, page, Hk, D)
    store = [(torch.randn(*shape, generator=g) / unit).to(cache) for _ in range(2)]
    order = torch.randperm(pages, generator=g)
    cols = max(max(per), 1)
    table = torch.full((len(lengths), cols), -7, dtype=torch.int32)
    at = 0
    for s, c in enumerate(per):
        table[s, :c] = order[at:at + c].int()
        at += c
    kd, vd = [(t.cuda() if layout == 0 else t.cuda().transpose(1, 2)) for t in store]
    obj = vitq.KvCache(kd, vd, unit, unit)
    views = [(t if layout == 0 else t.transpose(1, 2)).double() * obj._c.k_scale for t in store]
    visible = []
    for s, c in bad:
        table[s, c] = pages + 3 if c % 2 else -1
    keys, values = [], []
    for s, c in enumerate(per):
        sel = table[s, :c].long()
        ok = (sel >= 0) & (sel < pages)
        visible.append(ok.repeat_interleave(page))
        take = lambda t: t[sel.clamp(0, pages - 1)].transpose(1, 2).reshape(c * page, Hk, D)
        keys.append(take(views[0]))
        values.append(take(views[1]))
    offsets = torch.tensor([0] + [n for n, _ in lengths]).cumsum(0).int()
    lens = torch.tensor([n for _, n in lengths]).int()
    return q, offsets, lens, table, obj, keys, values, visible


def _gather(obj, table, lengths):
    """Keys and values of every sequence as they are in the cache."""
    out = []
    for cache, unit in ((obj.k, obj._c.k_scale), (obj.v, obj._c.v_scale)):
        pages, heads, page, dim = cache.shape
        store = cache.cpu().double() * unit
        per = []
        for s, (_, n) in enumerate(lengths):
            c = -(-n // page)
            sel = table[s, :c].long().clamp(0, pages - 1)
            per.append(store[sel].transpose(1, 2).reshape(c * page, heads, dim))
        out.append(per)
    return out


def _check_attention(lengths, Hq, Hk, D, dtype=BF16, cache=None, page=16, layout=0, causal=True, window=0, seed=0, scale=None,
                     max_kv=None, bad=(), edit=None):
    cache = dtype if cache is None else cache
    q, offsets, lens, table, obj, keys, values, visible = _paged(lengths, Hq, Hk, D, dtype, cache, page, layout, seed, bad=bad)
    scale = 1 / math.sqrt(D) if scale is None else scale
    T = q.shape[0]
    if edit is not None:
        edit(obj, table)
        keys, values = _gather(obj, table, lengths)
    longest = max(n for _, n in lengths) if max_kv is None else max_kv
    ws = torch.full((vitq.vq_attention_paged_workspace(T, len(lengths), Hq, obj, longest),), 0xFF, dtype=torch.uint8, device="cuda")
    q_room = torch.zeros(T, Hq * D + 16, dtype=dtype, device="cuda")
    q_room[:, :Hq * D] = q.cuda()
    out_room = torch.full((T + 1, Hq * D + 8), 9.0, dtype=dtype, device="cuda")
    out, lse = out_room[:T, :Hq * D], torch.full((T, Hq), 9.0, device="cuda")
    args = (q_room[:, :Hq * D], offsets.cuda(), lens.cuda(), table.cuda(), obj, scale, causal, window, longest)
    vitq.vq_attention_paged(*args, out, lse, ws)
    assert bool((out_room[T:] == 9.0).all()) and bool((out_room[:, Hq * D:] == 9.0).all())
    at = 0
    for s, (n, kv) in enumerate(lengths):
        qs = q[at:at + n].double().view(n, Hq, D)
        place = torch.arange(kv - n, kv)
        vis = visible[s][:max(kv, 0)] if len(visible[s]) else torch.zeros(0, dtype=torch.bool)
        o, l, mass, reach, tv = ref.attention(qs, keys[s][:kv], values[s][:kv], place, scale, causal, window, kv, vis)
        ob, lb = ref.attention_bounds(o, l, mass, reach, tv, dtype, D, kv)
        _within(out[at:at + n].view(n, Hq, D), o, ob, "out of sequence %d" % s)
        _within(lse[at:at + n], l, lb, "lse of sequence %d" % s)
        at += n
    again, ws2 = torch.empty_like(out), torch.zeros_like(ws)
    vitq.vq_attention_paged(*args, again, None, ws2)
    assert torch.equal(again.view(torch.int16), out.contiguous().view(torch.int16))
    return args, out, lse


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, F8), (F16, F8)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (4, 4), (8, 2), (7, 1), (32, 1)])
def test_attention_single_tokens(Hq, Hk, D, dtype, cache):
    _check_attention([(1, 1), (1, 2), (1, 31), (1, 33), (1, 200), (1, 700)], Hq, Hk, D, dtype, cache, page=16, layout=Hq % 2)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5), (True, 100), (False, 64), (True, 1)])
@pytest.mark.parametrize("Hq,Hk,D", [(4, 2, 64), (3, 1, 128), (8, 8, 64)])
def test_attention_chunks(Hq, Hk, D, causal, window):
    _check_attention([(5, 5), (1, 77), (64, 200), (33, 33), (130, 131)], Hq, Hk, D, BF16, page=32, causal=causal, window=window)


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, F8), (F16, F8)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 90)])
def test_attention_long_chunks(D, dtype, cache, causal, window):
    _check_attention([(300, 700), (1, 600), (257, 257), (0, 40), (90, 1000)], 4, 1, D, dtype, cache, page=64, causal=causal,
                     window=window, layout=1)


@pytest.mark.parametrize("page", [1, 3, 16, 61, 128, 200])
def test_attention_page_sizes(page):
    _check_attention([(1, 130), (17, 150), (70, 403)], 4, 2, 64, BF16, page=page, layout=page % 2)
    _check_attention([(1, 130), (17, 150), (70, 403)], 4, 2, 128, F16, F8, page=page)


def test_attention_rows_that_see_nothing():
    # more new tokens than keys, an empty history, and no tokens at all
    _check_attention([(5, 2), (3, 0), (0, 0), (0, 9), (40, 3), (1, 1)], 4, 2, 64, BF16)
    _check_attention([(200, 30)], 8, 2, 128, BF16)


def test_attention_pages_outside_the_cache():
    _check_attention([(1, 100), (20, 100), (1, 16), (200, 400)], 4, 2, 64, BF16, page=16, bad=((0, 1), (0, 4), (1, 2), (2, 0), (3, 7)))
    _check_attention([(1, 100), (20, 100), (1, 16), (200, 400)], 4, 2, 128, BF16, F8, page=16, bad=((0, 1), (0, 4), (1, 2), (2, 0), (3, 7)))


@pytest.mark.parametrize("cache", [BF16, F8])
@pytest.mark.parametrize("lengths", [[(1, 5)], [(1, 50), (1, 33)], [(6, 37)], [(150, 150)], [(100, 260)]])
def test_attention_what_lies_behind_the_last_key(lengths, cache):
    """NaN in the unused rest of the pages and in pages of nobody."""
    def spoil(obj, table):
        page = obj.k.shape[2]
        used = torch.zeros(obj.k.shape[0], page, dtype=torch.bool)
        for s, (_, n) in enumerate(lengths):
            for j in range(n):
                used[int(table[s, j // page]), j % page] = True
        for t in (obj.k, obj.v):
            raw = t.view(torch.uint8) if cache == F8 else t
            raw.permute(0, 2, 1, 3)[~used.cuda()] = 0x7F if cache == F8 else float("nan")
    _check_attention(lengths, 4, 2, 64, BF16, cache, page=16, edit=spoil)
    _check_attention(lengths, 4, 2, 128, BF16, cache, page=16, window=20, edit=spoil)


@pytest.mark.parametrize("cache", [BF16, F8])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_values_that_are_not_finite(D, cache):
    """An infinity or NaN among the values of a key reaches the rows that see the key, and no other."""
    lengths = [(6, 37), (1, 90), (150, 200), (3, 3), (300, 300)]
    def plant(obj, table):
        page = obj.v.shape[2]
        raw = obj.v.view(torch.uint8) if cache == F8 else obj.v
        for s, key, head, c in ((0, 36, 0, 3), (0, 33, 1, 7), (1, 89, 0, 0), (2, 180, 1, 60), (2, 199, 0, 5), (3, 1, 0, 63), (4, 299, 1, 2), (4, 130, 0, 9)):
            raw[int(table[s, key // page]), head, key % page, c] = 0x7F if cache == F8 else float("nan" if key % 2 else "-inf")
    for causal, window in ((True, 0), (True, 25), (False, 0)):
        _check_attention(lengths, 4, 2, D, BF16, cache, page=16, causal=causal, window=window, edit=plant)
    _check_attention([(6, 37)] + lengths[1:2], 4, 2, D, BF16, cache, page=16, edit=lambda o, t: plant_two(o, t, cache))


def plant_two(obj, table, cache):
    raw = obj.v.view(torch.uint8) if cache == F8 else obj.v
    raw[int(table[0, 2]), 1, 1, 4] = 0x7F if cache == F8 else float("inf")


def test_attention_a_chunk_beside_single_tokens():
    """A batch that both forms of the kernel share."""
    lengths = [(1, 40 + 13 * i) for i in range(15)] + [(300, 700)] + [(1, 600 - 11 * i) for i in range(15)] + [(0, 5), (20, 100)]
    for D, dtype, cache in ((64, BF16, BF16), (128, F16, F8)):
        _check_attention(lengths, 4, 1, D, dtype, cache, page=16)
        _check_attention(lengths, 4, 1, D, dtype, cache, page=16, window=100)


def test_attention_split_over_workgroups():
    for D, dtype, cache in ((128, BF16, BF16), (64, F16, F8)):
        _check_attention([(1, 5000)], 8, 2, D, dtype, cache, page=64)
        _check_attention([(1, 3000), (3, 100), (2, 4097), (1, 0)], 4, 1, D, dtype, cache, page=16, window=3500)
        _check_attention([(40, 2500)], 4, 1, D, dtype, cache, page=16)
        _check_attention([(1, 900)], 4, 1, D, dtype, cache, page=16, max_kv=4)           # a hint that is too small
        _check_attention([(1, 90)], 4, 1, D, dtype, cache, page=16, max_kv=100000)


def test_attention_strong_scores():
    _check_attention([(1, 300), (20, 90)], 4, 2, 64, BF16, scale=3.0)
    _check_attention([(1, 300), (20, 90)], 4, 2, 64, BF16, scale=-0.5)
    _check_attention([(1, 300), (20, 90)], 4, 2, 64, BF16, scale=0.0)


def test_attention_rows_outside_every_sequence_and_cut_lengths():
    args, out, lse = _check_attention([(3, 40), (70, 300), (1, 1200)], 4, 2, 64, BF16)
    q, offsets, lens, table, obj, scale, causal, window, longest = args
    part = torch.tensor([3, 73, 73, 73], dtype=torch.int32).cuda()       # the first three rows and the last belong to nobody
    o2, l2 = torch.full_like(out, 4.0), torch.full_like(lse, 4.0)
    ws = torch.empty(vitq.vq_attention_paged_workspace(74, 3, 4, obj, longest), dtype=torch.uint8, device="cuda")
    lens2 = torch.tensor([300, 0, 0], dtype=torch.int32).cuda()
    table2 = table[[1, 0, 2]].contiguous()
    vitq.vq_attention_paged(q, part, lens2, table2, obj, scale, causal, window, longest, o2, l2, ws)
    assert bool((o2[:3] == 4.0).all()) and bool((o2[73:] == 4.0).all()) and bool((l2[:3] == 4.0).all())
    # (another position in the batch may share its keys among workgroups otherwise, so bits are not compared)
    assert float((o2[3:73].float() - out[3:73].float()).abs().max()) <= 2.0 ** -7 * float(out[3:73].float().abs().max())
    # a length beyond the table is cut at the table
    width = table.shape[1] * 16
    long, cut = (torch.tensor([40, 300, n], dtype=torch.int32).cuda() for n in (width + 1000, width))
    table[table < 0] = 0
    o3, o4 = torch.empty_like(out), torch.empty_like(out)
    vitq.vq_attention_paged(q, offsets, long, table, obj, scale, causal, window, longest, o3, None, ws)
    vitq.vq_attention_paged(q, offsets, cut, table, obj, scale, causal, window, longest, o4, None, ws)
    assert torch.equal(o3, o4)


def test_attention_hints_and_windows_past_every_length():
    _check_attention([(1, 300), (8, 3), (70, 90)], 4, 2, 64, BF16, causal=False, window=2 ** 31 - 1, max_kv=2 ** 40)
    _check_attention([(1, 300), (8, 3), (70, 90)], 4, 2, 64, BF16, window=2 ** 31 - 1)
    args, out, _ = _check_attention([(1, 300), (8, 3), (70, 90)], 4, 2, 64, BF16)
    empty = args[3][:, :0].contiguous()                               # a table without columns: nobody sees anything
    o, lse = torch.empty_like(out), torch.empty(79, 4, device="cuda")
    vitq.vq_attention_paged(*args[:3], empty, *args[4:], o, lse, None)
    assert not bool(o.any()) and bool((lse == -math.inf).all())


def test_tensors_elsewhere_are_refused():
    m = vitq.FMat.empty(4, 128)
    with pytest.raises(ValueError):
        vitq.vq_quantize_e4m3(torch.zeros(4, 128), m)
    with pytest.raises(ValueError):
        vitq.vq_quantize_e4m3(torch.zeros(4, 128, device="cuda"), vitq.FMat.empty(4, 128, device="cpu"))
    args, out, _ = _check_attention([(1, 30)], 4, 2, 64, BF16)
    with pytest.raises(ValueError):
        vitq.vq_attention_paged(*args[:2], args[2].cpu(), *args[3:], out, None, None)
    with pytest.raises(ValueError):
        vitq.vq_attention_paged(*args[:2], args[2].long(), *args[3:], out, None, None)
    with pytest.raises(vitq.VitqError):                               # more splits than the workspace has room for
        long = torch.zeros(1, 4096, dtype=torch.int32, device="cuda")
        vitq.vq_attention_paged(args[0], args[1], args[2], long, args[4], 0.1, True, 0, 65536, out, None, torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_attention_in_place():
    args, out, _ = _check_attention([(3, 40), (70, 300), (1, 1200)], 4, 2, 64, F16)
    q = args[0].clone()
    ws = torch.empty(vitq.vq_attention_paged_workspace(74, 3, 4, args[4], args[8]), dtype=torch.uint8, device="cuda")
    vitq.vq_attention_paged(q, *args[1:], q, None, ws)
    assert torch.equal(q, out)


# ---- all of them as one layer --------------------------------------------------------------------------------------------

class _Layer:
    """Attention half of a layer: quantize, Q K V linear, norm + rotation + append, attention, quantize, output linear."""

    def __init__(self, lengths, D_model, Hq, Hk, D, cache, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.Hq, self.Hk, self.D = Hq, Hk, D
        T = sum(n for n, _ in lengths)
        self.lengths = lengths
        self.x = r(T, D_model).to(BF16)
        self.w = [vitq.FMat.empty((Hq + 2 * Hk) * D, D_model, 128), vitq.FMat.empty(D_model, Hq * D, 128)]
        self.w_f = [r((Hq + 2 * Hk) * D, D_model) * 0.05, r(D_model, Hq * D) * 0.05]
        for w, m in zip(self.w_f, self.w):
            vitq.vq_quantize_e4m3(w, m)
        self.xq, self.oq = vitq.FMat.empty(T, D_model, 1), vitq.FMat.empty(T, Hq * D, 1)
        self.qkv = torch.empty(T, (Hq + 2 * Hk) * D, dtype=BF16, device="cuda")
        page = 16
        per = [-(-n // page) for _, n in lengths]
        pages = sum(per)
        kv = [(r(pages, Hk, page, D) * (20 if cache == F8 else 1)).to(cache) for _ in range(2)]
        self.cache = vitq.KvCache(kv[0], kv[1], *((0.05, 0.05) if cache == F8 else (1.0, 1.0)))
        self.table = torch.zeros(len(lengths), max(per), dtype=torch.int32)
        order, at = torch.randperm(pages), 0
        slots, pos = [], []
        for s, (n, kv_len) in enumerate(lengths):
            self.table[s, :per[s]] = order[at:at + per[s]].int()
            at += per[s]
            p = torch.arange(kv_len - n, kv_len)
            pos.append(p)
            slots.append(self.table[s][p // page].long() * page + p % page)
        self.slots, self.pos = torch.cat(slots).cuda(), torch.cat(pos).int().cuda()
        self.table = self.table.cuda()
        self.offsets = torch.tensor([0] + [n for n, _ in lengths]).cumsum(0).int().cuda()
        self.lens = torch.tensor([n for _, n in lengths]).int().cuda()
        inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
        ang = torch.arange(4096, dtype=torch.float64)[:, None] * inv
        gam = [1 + 0.1 * r(D), 1 + 0.1 * r(D)]
        self.desc = vitq.make_rotate_desc(Hq, Hk, D, "rms", gam[0], None, gam[1], None, 1e-6, ang.cos().float().cuda(), ang.sin().float().cuda())
        self.q, self.o = torch.empty(T, Hq * D, dtype=BF16, device="cuda"), torch.empty(T, Hq * D, dtype=BF16, device="cuda")
        self.y = torch.empty(T, D_model, dtype=F32, device="cuda")
        self.longest = max(n for _, n in lengths)
        self.ws = torch.empty(vitq.vq_attention_paged_workspace(T, len(lengths), Hq, self.cache, self.longest), dtype=torch.uint8, device="cuda")

    def run(self):
        vitq.vq_quantize_e4m3(self.x, self.xq)
        vitq.vq_linear_e4m3(self.xq, self.w[0], None, 0, self.qkv)
        vitq.vq_qkv_norm_rotate(self.desc, self.qkv, self.pos, self.q, self.cache, self.slots)
        vitq.vq_attention_paged(self.q, self.offsets, self.lens, self.table, self.cache, self.D ** -0.5, True, 0, self.longest, self.o, None, self.ws)
        vitq.vq_quantize_e4m3(self.o, self.oq)
        vitq.vq_linear_e4m3(self.oq, self.w[1], None, 0, self.y)


@pytest.mark.parametrize("cache", [BF16, F8])
@pytest.mark.parametrize("lengths", [[(1, 700), (1, 90), (1, 1)], [(150, 200), (1, 333), (20, 20)]])
def test_layer_of_all(lengths, cache):
    """The chain's result against 64 bits from the same weights' codes: each stage rounds (E4M3 twice, bf16 thrice), so the whole
    is compared in the 2-norm; the stages are bounded by their own tests."""
    L = _Layer(lengths, 512, 8, 2, 64, cache, 3)
    k0, v0 = L.cache.k.cpu().double() * L.cache._c.k_scale, L.cache.v.cpu().double() * L.cache._c.v_scale
    L.run()
    torch.cuda.synchronize()
    xd = ref.dequantize(*ref.quantize(L.x.cpu(), 1), 1)
    wd = [ref.dequantize(_codes(m), m.scales.cpu(), 128) for m in L.w]
    T = xd.shape[0]
    qkv = (xd @ wd[0].t()).view(T, 12, 64)
    g_q, g_k, cos, sin = (t.cpu() for t in L.desc._keep)
    at = L.pos.long().cpu()
    cos, sin = cos[at], sin[at]
    q, _ = ref.norm_rotate(qkv[:, :8], "rms", g_q, None, 1e-6, cos, sin, False)
    k, _ = ref.norm_rotate(qkv[:, 8:10], "rms", g_k, None, 1e-6, cos, sin, False)
    slots = L.slots.cpu()
    k0[slots // 16, :, slots % 16], v0[slots // 16, :, slots % 16] = k, qkv[:, 10:]
    outs, first = [], 0
    for s, (n, kv) in enumerate(lengths):
        sel = L.table[s].long().cpu()
        take = lambda t: t[sel].transpose(1, 2).reshape(-1, 2, 64)[:kv]
        outs.append(ref.attention(q[first:first + n], take(k0), take(v0), torch.arange(kv - n, kv), 0.125, True, 0, kv)[0])
        first += n
    y = torch.cat(outs).reshape(T, 512) @ wd[1].t()
    rel = float((L.y.cpu().double() - y).norm() / y.norm())
    # an E4M3 rounding is off by at most 2^-4 of a value; keys, values and the attention's output take one each
    assert rel <= (3 if cache == F8 else 1) * 2.0 ** -4, rel


@pytest.mark.parametrize("cache", [BF16, F8])
def test_layer_captured_and_replayed(cache):
    """Graphs of two layers that share one stream order, replayed between eager work, give the eager results each time."""
    layers = [_Layer([(1, 700), (3, 90), (1, 1)], 512, 8, 2, 64, cache, 4), _Layer([(150, 200), (1, 333)], 256, 4, 4, 64, cache, 5)]
    eager = []
    for L in layers:
        L.run()
        torch.cuda.synchronize()
        eager.append((L.y.clone(), L.cache.k.clone().view(torch.uint8)))
    graphs = []
    for L in layers:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            L.run()
        torch.cuda.current_stream().wait_stream(side)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            L.run()
        graphs.append(gr)
    for turn in range(3):
        for L, gr, want in zip(layers, graphs, eager):
            L.y.fill_(float("nan"))
            L.ws.fill_(0xFF)
            gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(L.y, want[0]) and torch.equal(L.cache.k.view(torch.uint8), want[1])
            L.run()
            torch.cuda.synchronize()
            assert torch.equal(L.y, want[0])


def test_layer_on_another_stream():
    L = _Layer([(1, 700), (33, 90)], 512, 8, 2, 64, BF16, 6)
    L.run()
    torch.cuda.synchronize()
    want = L.y.clone()
    side = torch.cuda.Stream()
    L.y.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        L.run()
    side.synchronize()
    assert torch.equal(L.y, want)
