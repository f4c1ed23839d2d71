"""Every form of the serving layer's linear and attention at sizes, strides and masks that are not whole tiles."""
import math

import pytest
import torch

from paper_2504_18547_amd import vitq
from tests import serve_reference as ref
from tests.test_gpu_serve import BF16, F16, F32, F8, _check_attention, _codes

pytestmark = pytest.mark.gpu


# ---- linear -----------------------------------------------------------------------------------------------------

# The forms: K shared by a workgroup's waves, blocks of 16 x 16, 16 x 32 and 32 x 32 (in one and in two rounds of K); tiles of
# 64 x 128, 128 x 128, and 256 x 256 (fp32: 128 x 128 on four waves).
SIZES = [(5, 9000, 300), (24, 9000, 300), (24, 100, 515), (60, 5000, 257), (520, 100, 2050), (520, 129, 2048), (300, 1000, 5000),
         (1025, 1000, 4100), (1025, 129, 4104), (1300, 100, 2999), (4100, 300, 4111), (4097, 129, 4352), (4351, 60, 4100)]


def _within_here(got, want, bound, what):
    """As _within, on the device."""
    off = (got.double() - want).abs()
    bad = ~(off <= bound)                                              # (a NaN is none)
    assert not bool(bad.any()), "%s: %d of %d outside, worst %g" % (what, int(bad.sum()), bad.numel(), float(off.nan_to_num(math.inf).max()))


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_linear_forms(M, K, N, out):
    g = torch.Generator(device="cuda").manual_seed(M + K + N)
    x = torch.randn(M, K, generator=g, device="cuda") * (1 + 10 * (torch.rand(K, generator=g, device="cuda") < 0.02))
    w = torch.randn(N, K, generator=g, device="cuda") * 0.05
    b = torch.randn(N, generator=g, device="cuda")
    xm, wm = vitq.FMat.empty(M, K, 1), vitq.FMat.empty(N, K, 128)
    vitq.vq_quantize_e4m3(x, xm)
    vitq.vq_quantize_e4m3(w, wm)
    xd = ref.dequantize(_codes(xm), xm.scales.cpu(), 1).cuda()
    wd = ref.dequantize(_codes(wm), wm.scales.cpu(), 128).cuda()
    raw, size, peak = ref.linear(xd, wd, None, 0)
    for act, bias, pad in ((0, None, 0), (1, b, 3), (0, b, 8), (1, None, 5)):
        room = torch.full((M + 1, N + pad), float("nan"), dtype=out, device="cuda")
        vitq.vq_linear_e4m3(xm, wm, bias, act, room[:M, :N])
        want, big = (raw, size) if bias is None else (raw + b.double(), size + b.double().abs())
        want = ref.gelu(want) if act else want
        _within_here(room[:M, :N], want, ref.linear_bound(want, big, peak, K, out), "linear %d %d %d act %d pad %d" % (M, K, N, act, pad))
        assert bool(torch.isnan(room[M:]).all()) and bool(torch.isnan(room[:, N:]).all())
        again = torch.empty_like(room)
        vitq.vq_linear_e4m3(xm, wm, bias, act, again[:M, :N])
        assert torch.equal(again[:M, :N], room[:M, :N])


# ---- attention over the pages: the form of 256 rows a workgroup -------------------------------------------------------

TILES = [(70, 403), (257, 700), (3, 90)]                               # (with four rows a token more than 64 rows a sequence)


@pytest.mark.parametrize("page", [1, 3, 17, 48, 100, 200])
def test_attention_tiles_page_sizes(page):
    _check_attention(TILES, 4, 1, 64, BF16, page=page, layout=page % 2)
    _check_attention(TILES, 4, 1, 128, F16, F8, page=page)
    _check_attention(TILES, 8, 2, 128, BF16, page=page, causal=False, window=70, bad=((0, 1), (1, 2)))
    _check_attention(TILES, 8, 2, 64, F16, F8, page=page, layout=1, window=70)


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F16, F16), (BF16, F8)])
@pytest.mark.parametrize("scale", [3.0, -0.5, 0.0])
def test_attention_tiles_strong_scores(scale, dtype, cache):
    for D in (64, 128):
        _check_attention(TILES, 4, 1, D, dtype, cache, page=16, scale=scale)
        _check_attention(TILES, 4, 1, D, dtype, cache, page=16, scale=scale, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lengths", [TILES, [(1, 700), (2, 403)]])
def test_attention_scores_that_grow_along_the_keys(lengths, D, dtype):
    """The largest score moves on with nearly every step, by less than what makes the sums follow at once, and by more."""
    for gain in (2.0, 12.0):
        def grow(obj, table):
            page = obj.k.shape[2]
            for s, (_, n) in enumerate(lengths):
                for c in range(-(-n // page)):
                    obj.k[int(table[s, c])] *= 0.2 + gain * c * page / n
        for causal in (True, False):
            _check_attention(lengths, 4, 1, D, dtype, page=16, causal=causal, edit=grow)


def test_attention_tiles_in_place():
    for dtype, D in ((F16, 64), (BF16, 128)):
        args, out, _ = _check_attention(TILES, 4, 1, D, dtype, page=16)
        q = args[0].clone()
        ws = torch.empty(vitq.vq_attention_paged_workspace(q.shape[0], 3, 4, args[4], args[8]), dtype=torch.uint8, device="cuda")
        vitq.vq_attention_paged(q, *args[1:], q, None, ws)
        assert torch.equal(q, out)
        vitq.vq_attention_paged(q.copy_(args[0]), *args[1:8], 4, q, None, None)           # one piece: no workspace between
        # each is off by half a step of the probabilities and of the result, both at most half a step of the largest value, and by
        # 2^-13 of it for fp32 sums over up to 700 keys (the other test's bound)
        assert float((q.float() - out.float()).abs().max()) <= 2 * (2 * ref.HALF[dtype] + 2.0 ** -13) * float(args[4].v.float().abs().max())


def test_attention_tiles_hints_and_windows_past_every_length():
    _check_attention(TILES, 4, 1, 64, BF16, causal=False, window=2 ** 31 - 1, max_kv=2 ** 40)
    _check_attention(TILES, 4, 1, 128, F16, F8, max_kv=5)
    _check_attention(TILES, 4, 1, 128, F16, causal=False, window=30, max_kv=100000)
    _check_attention([(300, 20), (0, 5), (200, 0)], 4, 1, 128, BF16, window=7)


def test_attention_many_sequences():
    """Row tiles are found by a search over the sequences: two and three levels of it, sequences without tokens among them."""
    g = torch.Generator().manual_seed(11)
    lengths = [(int(n), int(n + extra)) for n, extra in zip(torch.randint(0, 4, (4200,), generator=g), torch.randint(0, 30, (4200,), generator=g))]
    _check_attention(lengths, 2, 1, 64, BF16, page=16)
    lengths = [(int(n), int(n + extra)) for n, extra in zip(torch.randint(0, 60, (300,), generator=g), torch.randint(0, 90, (300,), generator=g))]
    _check_attention(lengths, 4, 1, 128, F16, F8, page=16)


# ---- a cache of more than 2^31 units of 16 bytes ----------------------------------------------------------------------

@pytest.fixture(scope="module")
def storage():
    room = torch.empty(36 << 30, dtype=torch.uint8, device="cuda")
    yield room
    del room
    torch.cuda.empty_cache()


@pytest.mark.parametrize("page", [16, 10])
@pytest.mark.parametrize("cache", [BF16, F8])
def test_cache_past_32_bits(storage, cache, page):
    """Pages spread over 36 GiB, first at its start and last at its end: append by the rotation, then read by both forms."""
    Hq, Hk, D, n = 4, 2, 64, 400
    room = storage.view(cache)
    pages = 64
    step = room.numel() // pages // 16 * 16
    # [page, head, place, channel], keys and values of a place side by side
    k, v = [room[first:].as_strided((pages, Hk, page, D), (step, D, 2 * Hk * D, 1)) for first in (0, Hk * D)]
    unit = 0.05 if cache == F8 else 1.0
    obj = vitq.KvCache(k, v, unit, unit)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(page))[:-(-n // page)].int()
    assert int(table.max()) * step * room.element_size() > 2 ** 35
    place = torch.arange(n)
    slots = table[place // page].long() * page + place % page
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn(n, (Hq + 2 * Hk) * D, generator=g).to(BF16)
    q = torch.empty(n, Hq * D, dtype=BF16, device="cuda")
    vitq.vq_qkv_norm_rotate(vitq.make_rotate_desc(Hq, Hk, D, "none"), qkv.cuda(), None, q, obj, slots.cuda())
    x = qkv.view(n, Hq + 2 * Hk, D)
    assert torch.equal(q.cpu(), x[:, :Hq].reshape(n, Hq * D))
    want = [x[:, Hq + i * Hk:Hq + (i + 1) * Hk].double() for i in range(2)]
    got = [torch.stack([t[int(s) // page, :, int(s) % page] for s in slots]).cpu().double() * obj._c.k_scale for t in (k, v)]
    for a, b in zip(got, want):
        # a BF16 cache holds the values as they are; a code is off by half a step (a hair more for the product with 1/unit), the
        # smallest ones by half of 2^-9
        assert bool(((a - b).abs() <= (0.0 if cache == BF16 else 1.001 * (ref.HALF[F8] * b.abs() + 2.0 ** -10 * unit))).all())
    for first in (0, n - 3):                                           # all rows (tiles), then the last three alone
        rows = n - first
        off, lens = torch.tensor([0, rows]).int().cuda(), torch.tensor([n]).int().cuda()
        out = torch.empty(rows, Hq * D, dtype=BF16, device="cuda")
        ws = torch.empty(vitq.vq_attention_paged_workspace(rows, 1, Hq, obj, n), dtype=torch.uint8, device="cuda")
        vitq.vq_attention_paged(q[first:], off, lens, table.view(1, -1).cuda(), obj, 0.125, True, 0, n, out, None, ws)
        res = ref.attention(x[first:, :Hq].double(), got[0], got[1], torch.arange(first, n), 0.125, True, 0, n)
        bound, _ = ref.attention_bounds(*res, BF16, D, n)
        _within_here(out.view(rows, Hq, D).cpu(), res[0], bound, "rows from %d" % first)
