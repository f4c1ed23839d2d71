"""Host-side checks of the serving-layer operators: every refusal comes before a launch (CPU only)."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2504_18547_amd import vitq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E = {n[3:]: i for i, n in enumerate(vitq.STATUS_NAMES)}
P = 0x10000                                     # an address that no call here may reach


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(vitq.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return vitq.lib()


def _with(d, **kw):
    d = type(d).from_buffer_copy(d)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_struct_layouts_match_the_header(lib, tmp_path):
    want = [(vitq.vq_fmat, "vq_fmat", ("scales", "cols", "scale_stride")), (vitq.vq_kv_cache, "vq_kv_cache", ("dtype", "pages", "token_stride", "v_scale")),
            (vitq.vq_rotate_desc, "vq_rotate_desc", ("rot_dim", "q_gamma", "gamma_head_stride", "table_rows", "eps"))]
    lines = ["printf(\"%%zu\\n\", sizeof(%s));" % n for _, n, _ in want]
    lines += ["printf(\"%%zu\\n\", offsetof(%s, %s));" % (n, f) for _, n, fs in want for f in fs]
    src = tmp_path / "sz.c"
    src.write_text('#include "vitq.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(){' + "".join(lines) + "}")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sz")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "sz")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(c) for c, _, _ in want] + [getattr(c, f).offset for c, _, fs in want for f in fs]


def _fmat(rows=4, cols=200, block_rows=1, **kw):
    nb = -(-rows // block_rows)
    return _with(vitq.vq_fmat(P, P, block_rows, 0, rows, cols, (cols + 15) // 16 * 16, nb), **kw)


BAD_FMAT = [(dict(data=None), "ERR_NULL"), (dict(scales=None), "ERR_NULL"), (dict(block_rows=64), "ERR_UNSUPPORTED"),
            (dict(rows=-1), "ERR_SHAPE"), (dict(cols=0), "ERR_SHAPE"), (dict(rows=1 << 28), "ERR_SHAPE"),
            (dict(row_stride=199), "ERR_STRIDE"), (dict(row_stride=192), "ERR_STRIDE"), (dict(data=P + 8), "ERR_STRIDE"),
            (dict(scale_stride=3), "ERR_STRIDE"), (dict(scales=P + 2), "ERR_STRIDE")]


@pytest.mark.parametrize("change,status", BAD_FMAT)
def test_matrix_descriptions(lib, change, status):
    m, w = _fmat(**change), _fmat(32, 200, 128)
    # (the quantizer compares its sizes with the description's only after the description itself)
    assert lib.vq_quantize_e4m3(P, vitq.VQ_F32, 4, 200, 200, C.byref(m), None) == E[status]
    assert lib.vq_linear_e4m3(C.byref(m), C.byref(w), None, 0, P, vitq.VQ_F32, 32, None) == E[status]


def test_quantizer_and_linear_refusals(lib):
    m, x, w = _fmat(), _fmat(), _fmat(32, 200, 128)
    q = lambda p=P, t=vitq.VQ_BF16, r=4, c=200, ld=200, o=m: lib.vq_quantize_e4m3(p, t, r, c, ld, None if o is None else C.byref(o), None)
    assert q(o=None) == E["ERR_NULL"] and q(p=None) == E["ERR_NULL"]
    assert q(t=vitq.VQ_E4M3) == E["ERR_BITS"] and q(t=-1) == E["ERR_BITS"] and q(t=17) == E["ERR_BITS"]
    assert q(r=5) == E["ERR_SHAPE"] and q(c=199) == E["ERR_SHAPE"] and q(ld=199) == E["ERR_SHAPE"]
    assert q(p=P + 1) == E["ERR_STRIDE"] and q(r=0, o=_fmat(0)) == E["OK"]
    f = lambda a=x, b=w, bias=None, act=0, y=P, t=vitq.VQ_BF16, ld=32: lib.vq_linear_e4m3(C.byref(a), C.byref(b), bias, act, y, t, ld, None)
    assert f(y=None) == E["ERR_NULL"] and f(act=2) == E["ERR_UNSUPPORTED"] and f(t=vitq.VQ_E4M3) == E["ERR_BITS"]
    assert f(ld=31) == E["ERR_STRIDE"] and f(y=P + 1) == E["ERR_STRIDE"] and f(bias=P + 2) == E["ERR_STRIDE"]
    assert f(b=_fmat(32, 199, 128)) == E["ERR_SHAPE"] and f(a=_fmat(4, 200, 128)) == E["ERR_UNSUPPORTED"]
    assert f(b=_fmat(32, 200, 1)) == E["ERR_UNSUPPORTED"]
    big = _fmat(4, 65537), _fmat(32, 65537, 128)
    assert f(*big) == E["ERR_SHAPE"]
    assert f(a=_fmat(row_stride=1 << 24)) == E["ERR_STRIDE"]
    assert f(a=_fmat(0)) == E["OK"] and f(b=_fmat(0, 200, 128), ld=0) == E["OK"]


def _cache(**kw):
    return _with(vitq.vq_kv_cache(P, P, vitq.VQ_BF16, 2, 64, 16, 10, 2 * 16 * 64, 16 * 64, 64, 1.0, 1.0), **kw)


BAD_CACHE = [(dict(k=None), "ERR_NULL"), (dict(v=None), "ERR_NULL"), (dict(dtype=vitq.VQ_F32), "ERR_BITS"), (dict(dtype=9), "ERR_BITS"),
             (dict(pages=0), "ERR_SHAPE"), (dict(page_size=0), "ERR_SHAPE"), (dict(page_size=-4), "ERR_SHAPE"), (dict(pages=1 << 31), "ERR_SHAPE"),
             (dict(pages=1 << 28), "ERR_SHAPE"), (dict(token_stride=60), "ERR_STRIDE"), (dict(token_stride=68), "ERR_STRIDE"),
             (dict(page_stride=-2048), "ERR_STRIDE"), (dict(page_stride=1 << 60), "ERR_STRIDE"), (dict(page_stride=1 << 34), "ERR_SHAPE"),
             (dict(k=P + 8), "ERR_STRIDE"), (dict(v=P + 2), "ERR_STRIDE"), (dict(k_scale=2.0), "ERR_STEP"), (dict(v_scale=float("nan")), "ERR_STEP"),
             (dict(dtype=vitq.VQ_E4M3, k_scale=0.0), "ERR_STEP"), (dict(dtype=vitq.VQ_E4M3, v_scale=-1.0), "ERR_STEP")]


def _rotate(lib, d=None, c=None, **kw):
    d = d if d is not None else _desc()
    c = c if c is not None else _cache()
    a = dict(qkv=P, dtype=vitq.VQ_BF16, tokens=3, ld=8 * 64, positions=P, q_out=P, q_dtype=vitq.VQ_BF16, q_ld=4 * 64, cache=C.byref(c), slots=P)
    a.update(kw)
    return lib.vq_qkv_norm_rotate(C.byref(d), a["qkv"], a["dtype"], a["tokens"], a["ld"], a["positions"], a["q_out"], a["q_dtype"],
                                  a["q_ld"], a["cache"], a["slots"], None)


def _desc(**kw):
    return _with(vitq.vq_rotate_desc(4, 2, 64, 1, 64, 0, P, None, P, None, 0, P, P, 100, 1e-6, 0), **kw)


def _attend(lib, c=None, **kw):
    c = c if c is not None else _cache()
    a = dict(q=P, dtype=vitq.VQ_BF16, tokens=3, q_ld=256, q_heads=4, offsets=P, lens=P, seqs=2, table=P, ts=4, tc=4, scale=0.1, causal=1,
             window=0, max_kv=64, out=P, out_ld=256, lse=None, ws=None, wb=0)
    a.update(kw)
    return lib.vq_attention_paged(a["q"], a["dtype"], a["tokens"], a["q_ld"], a["q_heads"], a["offsets"], a["lens"], a["seqs"], a["table"],
                                  a["ts"], a["tc"], C.byref(c), a["scale"], a["causal"], a["window"], a["max_kv"], a["out"], a["out_ld"],
                                  a["lse"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_cache_descriptions(lib, change, status):
    c, n = _cache(**change), C.c_size_t()
    assert _rotate(lib, c=c) == E[status]
    assert _attend(lib, c=c) == E[status]
    assert lib.vq_attention_paged_workspace(3, 2, 4, C.byref(c), 64, C.byref(n)) == E[status]


@pytest.mark.parametrize("change,status", [
    (dict(q_heads=0), "ERR_SHAPE"), (dict(kv_heads=3), "ERR_STRIDE"), (dict(head_dim=60), "ERR_SHAPE"), (dict(head_dim=264), "ERR_SHAPE"),
    (dict(head_dim=56), "ERR_SHAPE"), (dict(norm=3), "ERR_UNSUPPORTED"), (dict(rot_dim=8), "ERR_SHAPE"), (dict(rot_dim=80), "ERR_SHAPE"),
    (dict(q_gamma=None), "ERR_NULL"), (dict(k_gamma=None), "ERR_NULL"), (dict(q_gamma=P + 4), "ERR_STRIDE"), (dict(k_beta=P + 4), "ERR_STRIDE"),
    (dict(eps=-1.0), "ERR_STEP"), (dict(eps=float("inf")), "ERR_STEP"), (dict(gamma_head_stride=32), "ERR_STRIDE"), (dict(gamma_head_stride=66), "ERR_STRIDE"),
    (dict(cos_table=None), "ERR_NULL"), (dict(sin_table=P + 8), "ERR_STRIDE"), (dict(table_rows=0), "ERR_SHAPE")])
def test_rotate_descriptions(lib, change, status):
    assert _rotate(lib, _desc(**change)) == E[status]


@pytest.mark.parametrize("change,status", [
    (dict(qkv=None), "ERR_NULL"), (dict(qkv=P + 8), "ERR_STRIDE"), (dict(ld=500), "ERR_STRIDE"), (dict(ld=516), "ERR_STRIDE"), (dict(dtype=vitq.VQ_E4M3), "ERR_BITS"),
    (dict(q_dtype=vitq.VQ_F32), "ERR_BITS"), (dict(q_ld=252), "ERR_STRIDE"), (dict(positions=None), "ERR_NULL"), (dict(slots=None), "ERR_NULL"),
    (dict(cache=None), "ERR_NULL"), (dict(q_out=None, cache=None, slots=None), "ERR_NULL"), (dict(tokens=-1), "ERR_SHAPE"), (dict(tokens=1 << 24), "ERR_SHAPE"),
    (dict(tokens=0), "OK")])
def test_rotate_arguments(lib, change, status):
    assert _rotate(lib, **change) == E[status]


@pytest.mark.parametrize("change,status", [
    (dict(q=None), "ERR_NULL"), (dict(out=None), "ERR_NULL"), (dict(offsets=None), "ERR_NULL"), (dict(lens=None), "ERR_NULL"), (dict(table=None), "ERR_NULL"),
    (dict(dtype=vitq.VQ_F16), "ERR_BITS"), (dict(dtype=vitq.VQ_F32), "ERR_BITS"), (dict(q_heads=3), "ERR_SHAPE"), (dict(q_heads=0), "ERR_SHAPE"),
    (dict(tokens=-1), "ERR_SHAPE"), (dict(seqs=-1), "ERR_SHAPE"), (dict(tokens=1 << 23), "ERR_SHAPE"), (dict(q_ld=252), "ERR_STRIDE"),
    (dict(out_ld=260), "ERR_STRIDE"), (dict(q=P + 2), "ERR_STRIDE"), (dict(ts=3), "ERR_STRIDE"), (dict(window=-1), "ERR_SHAPE"),
    (dict(tc=1 << 28, ts=1 << 28), "ERR_SHAPE"), (dict(scale=float("nan")), "ERR_STEP"), (dict(max_kv=-1), "ERR_SHAPE"),
    (dict(max_kv=0, tc=8192, ts=8192), "ERR_WORKSPACE"), (dict(max_kv=100000, tc=8192, ts=8192, ws=P, wb=16), "ERR_WORKSPACE"),
    (dict(max_kv=100000, tc=8192, ts=8192, ws=P + 4, wb=1 << 40), "ERR_STRIDE"),
    (dict(lens=P + 2), "ERR_STRIDE"), (dict(out_ld=264), "ERR_STRIDE"), (dict(tokens=0), "OK"), (dict(seqs=0), "OK")])
def test_attention_arguments(lib, change, status):
    assert _attend(lib, **change) == E[status]


def test_attention_head_dims_and_workspace(lib):
    assert _attend(lib, _cache(head_dim=32), q_ld=128, out_ld=128) == E["ERR_UNSUPPORTED"]
    n, m = C.c_size_t(), C.c_size_t()
    c = _cache(pages=100000, page_stride=2048)
    assert lib.vq_attention_paged_workspace(3, 2, 4, C.byref(c), 100, None) == E["ERR_NULL"]
    assert lib.vq_attention_paged_workspace(0, 2, 4, C.byref(c), 100, C.byref(n)) == E["OK"] and n.value == 0
    assert lib.vq_attention_paged_workspace(1, 1, 4, C.byref(c), 0, C.byref(n)) == E["OK"]
    for kv in (1, 100, 1000, 5000, 100000, 1 << 30):
        assert lib.vq_attention_paged_workspace(1, 1, 4, C.byref(c), kv, C.byref(m)) == E["OK"]
        assert m.value <= n.value


def test_binding_refuses_what_the_library_cannot_see(lib):
    x = torch.zeros(4, 128)
    with pytest.raises(ValueError):
        vitq.FMat(x, torch.zeros(1, 4), 128, 1)                       # codes are bytes
    with pytest.raises(ValueError):
        vitq.FMat(torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(1, 4), 256, 1)
    with pytest.raises(ValueError):
        vitq.vq_quantize_e4m3(x.t(), vitq.FMat.empty(128, 4, 1, device="cpu"))
    with pytest.raises(ValueError):
        vitq.vq_quantize_e4m3(x.to(torch.int32), vitq.FMat.empty(4, 128, 1, device="cpu"))
    k = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        vitq.KvCache(k, k.transpose(1, 2))
    with pytest.raises(ValueError):
        vitq.KvCache(k.transpose(2, 3), k.transpose(2, 3))
    with pytest.raises(ValueError):
        vitq.make_rotate_desc(4, 2, 64, "rms", q_gamma=torch.ones(32))
    with pytest.raises(ValueError):
        vitq.make_rotate_desc(4, 2, 64, "rms", cos=torch.ones(4, 32))
