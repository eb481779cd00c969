"""Host side of rotation, caches of 8 bits and shared prefixes: sizes and refusals, no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild

P = 0x1000      # stands for any aligned address: these calls end before it is used
BAD = nb.NP_E_INVAL


@pytest.fixture(scope="module")
def lib():
    nbuild.build()
    return nb.load()


def _with(s, kw):
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _desc(**kw):
    return _with(nb.make_kv_desc(torch.bfloat16, 2, 4, 128, 64, 100, 8, 50, e4m3=kw.pop("e4m3", False)), kw)


def _tables(**kw):
    return _with(nb.np_kv_tables(P, P, P, P, P), kw)


def _rows(**kw):
    return _with(nb.np_rows(P, 4 * 128, 128), kw)


def _rotation(**kw):
    return _with(nb.np_rotation(P, P, P, 128, nb.NP_ROT_HALVES, 1e-6), kw)


def _b(x):
    return None if x is None else C.byref(x)


def _said(lib, word):
    return word in lib.np_attn_last_error().decode()


def test_struct_size_matches_the_header():
    assert C.sizeof(nb.np_rotation) == 3 * 8 + 6 * 4


@pytest.mark.parametrize("hd", [64, 128])
def test_sizes_of_a_cache_of_8_bits(lib, hd):
    d = _desc(e4m3=True, head_dim=hd)
    s, t = nb.np_kv_sizes(d), nb.np_kv_sizes(_desc(head_dim=hd))
    assert d.dtype == nb.NP_T_BF16 | nb.NP_KV_E4M3
    assert s.page_bytes == 2 * 4 * 64 * (hd + 1) and s.cache_bytes == 2 * 100 * s.page_bytes and s.page_bytes % 16 == 0
    assert s.table_bytes == t.table_bytes and s.scratch_bytes == t.scratch_bytes
    small = _desc(e4m3=True, head_dim=hd, n_kv_heads=1, page_tokens=16)
    assert nb.np_kv_sizes(small).page_bytes == 32 * (hd + 1)
    assert nb.np_attn_workspace_bytes(d, 8, 3) == nb.np_attn_workspace_bytes(_desc(head_dim=hd), 8, 3)


@pytest.mark.parametrize("dtype", [2, 3, 18, 32, 48, -16, -1, 1 << 20])
def test_no_other_types(lib, dtype):
    with pytest.raises(nb.NpError) as e:
        nb.np_kv_sizes(_desc(dtype=dtype))
    assert e.value.code == BAD


def test_workspace_of_shared_prefixes(lib):
    d = _desc()
    a, plain = nb.np_attn_shared_workspace_bytes(d, 8, 4), nb.np_attn_workspace_bytes(d, 8, 4)
    assert a > plain and nb.np_attn_shared_workspace_bytes(d, 8, 1024) > a and nb.np_attn_shared_workspace_bytes(d, 512, 4) > a
    for heads, n in ((6, 1), (0, 1), (4 * 129, 1), (8, -1), (8, 1025)):
        with pytest.raises(nb.NpError) as e:
            nb.np_attn_shared_workspace_bytes(d, heads, n)
        assert e.value.code == BAD
    assert lib.np_attn_shared_workspace_bytes(_b(d), 8, 4, None) == BAD


@pytest.mark.parametrize("field,value", [("rot_dim", -16), ("rot_dim", 144), ("rot_dim", 8), ("rot_dim", 24), ("pairs", 2), ("pairs", -1), ("eps", 0.0), ("eps", -1.0),
                                         ("eps", 1e-40), ("eps", float("inf")), ("eps", float("nan")), ("freq", None), ("freq", P + 4), ("q_gain", P + 8), ("k_gain", P + 4)])
def test_rotations_that_are_none(lib, field, value):
    r = _rotation(**{field: value})
    shape, x = nb.np_attn_shape(0, 8, 4, 128), _rows()
    assert lib.np_attn_rotate(_b(shape), _b(r), _b(x), _b(x), _b(x), _b(x), 3, P, P, 2, None) == BAD
    assert lib.np_kv_append_rotated(_b(_desc()), P, 0, _b(_tables()), _b(r), _b(x), 8, _b(x), _b(x), _b(x), 3, None, P, P, 2, None) == BAD
    assert lib.np_attn_last_error()


def test_rotate_refuses_bad_arguments(lib):
    def call(dtype=0, hq=8, hkv=4, hd=128, rot=_rotation(), q=_rows(), k=_rows(), qo=_rows(), ko=_rows(), tokens=9, cu=P, start=P, n=2, **kw):
        s = _with(nb.np_attn_shape(dtype, hq, hkv, hd), kw)
        return lib.np_attn_rotate(_b(s), _b(rot), _b(q), _b(k), _b(qo), _b(ko), tokens, cu, start, n, None)

    assert lib.np_attn_rotate(None, _b(_rotation()), *[_b(_rows())] * 4, 9, P, P, 2, None) == BAD
    assert call(dtype=2) == BAD and call(dtype=16) == BAD and call(hd=96) == BAD and call(hq=0) == BAD and call(hkv=0) == BAD and call(hkv=1025) == BAD
    assert call(rot=None) == BAD and call(tokens=-1) == BAD and call(n=-1) == BAD and call(start=None) == BAD
    assert call(cu=None) == BAD and _said(lib, "one token for each")
    assert call(n=1025) == BAD and _said(lib, "NP_KV_MAX_SEQS")
    for name in ("q", "k", "qo", "ko"):
        for field, value in (("data", None), ("data", P + 8), ("token_stride", 12), ("head_stride", -8)):
            assert call(**{name: _rows(**{field: value})}) == BAD
    for name in ("qo", "ko"):
        assert call(**{name: _rows(token_stride=0)}) == BAD and call(**{name: _rows(head_stride=0)}) == BAD and _said(lib, "above 0")
    assert call(hd=64, rot=_rotation()) == BAD                 # more values turn than a head has
    assert call(tokens=1 << 30) == BAD and _said(lib, "too many rows")
    bad = nb.np_attn_shape(0, 8, 4, 128)
    bad.reserved[2] = 1
    assert lib.np_attn_rotate(_b(bad), _b(_rotation()), *[_b(_rows())] * 4, 9, P, P, 2, None) == BAD
    r = _rotation()
    r.reserved[1] = 1
    assert call(rot=r) == BAD
    # nothing to do is no error, and nothing is looked at
    assert call(tokens=0, q=None, start=None) == 0 and call(n=0, q=None) == 0


def test_append_rotated_and_read_refuse_bad_arguments(lib):
    for d in (_desc(), _desc(e4m3=True)):
        def rotated(cache=P, layer=0, t=_tables(), rot=_rotation(), q=_rows(), heads=8, k=_rows(), v=_rows(), qo=_rows(), tokens=3, cu=P, start=P, n=2):
            return lib.np_kv_append_rotated(_b(d), cache, layer, _b(t), _b(rot), _b(q), heads, _b(k), _b(v), _b(qo), tokens, None, cu, start, n, None)

        def read(cache=P, layer=0, t=_tables(), k=_rows(), v=_rows(), tokens=3, cu=P, start=P, n=2):
            return lib.np_kv_read(_b(d), cache, layer, _b(t), _b(k), _b(v), tokens, None, cu, start, n, None)

        for call in (rotated, read):
            assert call(layer=-1) == BAD and call(layer=2) == BAD and call(tokens=-1) == BAD and call(n=9) == BAD and call(n=-1) == BAD
            assert call(cu=None) == BAD and _said(lib, "one token for each")
            assert call(start=None) == BAD and call(cache=None) == BAD and call(cache=P + 8) == BAD
            assert call(t=None) == BAD and call(t=_tables(lens=None)) == BAD and call(t=_tables(status=None)) == BAD
            assert call(k=_rows(data=None)) == BAD and call(v=_rows(token_stride=4)) == BAD
            assert call(tokens=0) == 0 and call(n=0, tokens=0, cu=None) == 0
        assert rotated(heads=0) == BAD and rotated(heads=1 << 18) == BAD and rotated(rot=None) == BAD and rotated(q=_rows(data=P + 2)) == BAD
        assert rotated(qo=_rows(token_stride=0)) == BAD and rotated(qo=_rows(head_stride=0)) == BAD
        assert read(k=_rows(token_stride=0)) == BAD and read(v=_rows(head_stride=0)) == BAD and _said(lib, "above 0")


def test_shared_refuses_bad_arguments(lib):
    d = _desc()

    def held(t=_tables(), seqs=P, n=3, cu=P, groups=1, out=P):
        return lib.np_kv_shared(_b(d), _b(t), seqs, n, cu, groups, out, None)

    assert held(t=None) == BAD and held(t=_tables(page_table=None)) == BAD and held(n=-1) == BAD and held(n=1025) == BAD and held(n=9, seqs=None) == BAD
    assert held(groups=-1) == BAD and held(groups=1025) == BAD and held(cu=None) == BAD and held(out=None) == BAD
    assert held(groups=0, cu=None, out=None) == 0

    def call(layer=0, q=_rows(), heads=8, seqs=P, n=2, cu=P, shared=P, groups=1, scale=0.1, out=_rows(), ws=P, size=1 << 40, cache=P, tables=_tables()):
        return lib.np_attn_decode_shared(_b(d), cache, layer, _b(tables), _b(q), heads, seqs, n, cu, shared, groups, scale, _b(out), None, ws, size, None)

    assert call(size=nb.np_attn_shared_workspace_bytes(d, 8, 2) - 1) == BAD and _said(lib, "workspace")
    assert call(heads=6) == BAD and call(heads=0) == BAD and call(heads=4 * 129) == BAD and call(n=-1) == BAD and call(n=1025) == BAD and call(n=9, seqs=None) == BAD
    assert call(groups=-1) == BAD and call(groups=1025) == BAD and call(cu=None) == BAD and call(shared=None) == BAD
    assert call(layer=2) == BAD and call(cache=None) == BAD and call(ws=None) == BAD and call(ws=P + 4) == BAD
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=s) == BAD
    assert call(q=_rows(data=P + 2)) == BAD and call(out=_rows(head_stride=4)) == BAD and call(out=_rows(token_stride=0)) == BAD
    assert call(tables=_tables(lens=None)) == BAD
    assert call(n=0) == 0


def test_without_a_device_calls_fail(lib):
    if torch.cuda.is_available():
        pytest.skip("a device is there")
    x, r, t = _b(_rows()), _b(_rotation()), _b(_tables())
    shape = nb.np_attn_shape(0, 8, 4, 128)
    assert lib.np_attn_rotate(_b(shape), r, x, x, x, x, 3, P, P, 2, None) == nb.NP_E_CUDA
    for d in (_desc(), _desc(e4m3=True)):
        assert lib.np_kv_append_rotated(_b(d), P, 0, t, r, x, 8, x, x, x, 3, None, P, P, 2, None) == nb.NP_E_CUDA
        assert lib.np_kv_append(_b(d), P, 0, t, x, x, 3, None, P, P, 2, None) == nb.NP_E_CUDA
        assert lib.np_kv_read(_b(d), P, 0, t, x, x, 3, None, P, P, 2, None) == nb.NP_E_CUDA
        assert lib.np_attn_decode_shared(_b(d), P, 0, t, x, 8, P, 2, P, P, 1, 0.1, x, None, P, 1 << 40, None) == nb.NP_E_CUDA
    assert lib.np_kv_shared(_b(_desc()), t, P, 3, P, 1, P, None) == nb.NP_E_CUDA


def test_binding_refuses_what_does_not_fit(lib):
    z = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    none = nb.make_rotation(None)
    for call in (lambda: nb.np_attn_rotate(none, z, z, z, z, None, i), lambda: nb.make_rotation(torch.zeros(32, dtype=torch.float64)),
                 lambda: nb.np_kv_append_rotated(_desc(), z, 0, _tables(), none, z, z, z, z, i, None, i), lambda: nb.np_kv_read(_desc(), z, 0, _tables(), z, z, i, None, i),
                 lambda: nb.np_kv_read(_desc(e4m3=True), z, 0, _tables(), z, z, i, None, i), lambda: nb.np_kv_shared(_desc(), _tables(), i, i, i),
                 lambda: nb.np_attn_decode_shared(_desc(), z, 0, _tables(), z, z, i, i, i)):
        with pytest.raises(nb.NpError) as e:
            call()
        assert e.value.code == BAD
