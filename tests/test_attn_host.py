"""Host side of the cache and attention entry points: sizes and refusals, no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2608_22643_b200 import binding as nb
from paper_2608_22643_b200 import build as nbuild

P = 0x1000      # stands for any aligned address: these calls end before it is used


@pytest.fixture(scope="module")
def lib():
    nbuild.build()
    return nb.load()


def _desc(**kw):
    d = nb.make_kv_desc(torch.bfloat16, 2, 4, 128, 64, 100, 8, 50)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _tables(**kw):
    t = nb.np_kv_tables(P, P, P, P, P)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def _rows(**kw):
    r = nb.np_rows(P, 4 * 128, 128)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def test_struct_sizes_match_the_header():
    assert C.sizeof(nb.np_kv_desc) == 12 * 4 and C.sizeof(nb.np_kv_tables) == 5 * 8 and C.sizeof(nb.np_kv_sizes_out) == 4 * 8
    assert C.sizeof(nb.np_rows) == 24 and C.sizeof(nb.np_attn_shape) == 8 * 4


def test_sizes(lib):
    s = nb.np_kv_sizes(_desc())
    assert s.page_bytes == 2 * 4 * 64 * 128 * 2 and s.cache_bytes == 2 * 100 * s.page_bytes and s.table_bytes == 8 * 50 * 4
    assert s.scratch_bytes >= 4 * (100 + 2 * 1024)
    big = _desc(n_pages=1 << 22, max_pages=1 << 22, page_tokens=16, n_layers=80)
    assert nb.np_kv_sizes(big).cache_bytes == 80 * (1 << 22) * 2 * 4 * 16 * 128 * 2      # past 32 bits by far


def test_workspace_grows_with_rows_and_heads(lib):
    a = nb.np_attn_workspace_bytes(_desc(), 4, 1)
    assert a > 0 and nb.np_attn_workspace_bytes(_desc(), 4, 1024) > a and nb.np_attn_workspace_bytes(_desc(), 256, 1) > a


@pytest.mark.parametrize("field,value", [
    ("dtype", 2), ("dtype", -1), ("n_layers", 0), ("n_kv_heads", 0), ("n_kv_heads", 1025), ("head_dim", 96), ("head_dim", 256),
    ("page_tokens", 8), ("page_tokens", 48), ("page_tokens", 512), ("n_pages", 0), ("n_pages", (1 << 22) + 1), ("max_seqs", 0),
    ("max_seqs", 1025), ("max_pages", 0), ("max_pages", 101),
])
def test_bad_descriptions_are_refused(lib, field, value):
    with pytest.raises(nb.NpError) as e:
        nb.np_kv_sizes(_desc(**{field: value}))
    assert e.value.code == nb.NP_E_INVAL and str(e.value)


def test_reserved_fields_are_refused(lib):
    d = _desc()
    d.reserved[3] = 1
    with pytest.raises(nb.NpError):
        nb.np_kv_sizes(d)
    s = nb.np_attn_shape(0, 4, 4, 128)
    s.reserved[0] = 1
    r = C.byref(_rows())
    assert lib.np_attn_prompt(C.byref(s), r, r, r, P, 1, 5, 1.0, r, None, P, None) == nb.NP_E_INVAL


def _b(x):
    return C.byref(x)


def test_table_calls_refuse_bad_arguments(lib):
    d, t = _desc(), _tables()
    bad = nb.NP_E_INVAL
    assert lib.np_kv_reset(None, _b(t), None) == bad and lib.np_kv_reset(_b(d), None, None) == bad
    for name, _ in nb.np_kv_tables._fields_:
        assert lib.np_kv_reset(_b(d), _b(_tables(**{name: None})), None) == bad
    for n in (-1, 9):
        assert lib.np_kv_reserve(_b(d), _b(t), P, P, n, None, None) == bad
        assert lib.np_kv_fork(_b(d), P, _b(t), P, P, n, None) == bad
        assert lib.np_kv_free(_b(d), _b(t), P, n, None) == bad
    assert lib.np_kv_reserve(_b(d), _b(t), P, None, 2, None, None) == bad
    assert lib.np_kv_fork(_b(d), None, _b(t), P, P, 2, None) == bad
    assert lib.np_kv_fork(_b(d), P + 8, _b(t), P, P, 2, None) == bad and "aligned" in lib.np_attn_last_error().decode()
    assert lib.np_kv_fork(_b(d), P, _b(t), None, P, 2, None) == bad and lib.np_kv_fork(_b(d), P, _b(t), P, None, 2, None) == bad
    assert lib.np_kv_compact(_b(d), P, _b(t), None, None, None) == bad
    mixed = _tables(refs=2 * P)
    assert lib.np_kv_compact(_b(d), P, _b(t), _b(mixed), None, None) == bad and "three others" in lib.np_attn_last_error().decode()
    assert lib.np_kv_copy_pages(_b(d), P, P, P, P, 101, P, None) == bad and lib.np_kv_copy_pages(_b(d), P, P, P, P, 1, None, None) == bad
    # nothing to do is no error, and nothing is looked at
    assert lib.np_kv_reserve(_b(d), _b(t), None, None, 0, None, None) == 0 and lib.np_kv_free(_b(d), _b(t), None, 0, None) == 0
    assert lib.np_kv_fork(_b(d), None, _b(t), None, None, 0, None) == 0


def test_append_refuses_bad_arguments(lib):
    d, t, bad = _desc(), _tables(), nb.NP_E_INVAL

    def call(layer=0, k=_rows(), v=_rows(), tokens=3, cu=P, start=P, n=2, cache=P):
        return lib.np_kv_append(_b(d), cache, layer, _b(t), _b(k), _b(v), tokens, None, cu, start, n, None)

    assert call(layer=-1) == bad and call(layer=2) == bad and call(tokens=-1) == bad and call(n=9) == bad
    assert call(cu=None) == bad and "one token for each" in lib.np_attn_last_error().decode()
    assert call(start=None) == bad and call(cache=None) == bad and call(cache=P + 2) == bad
    assert call(k=_rows(data=None)) == bad and call(v=_rows(data=P + 8)) == bad
    assert call(k=_rows(token_stride=12)) == bad and call(v=_rows(head_stride=-8)) == bad
    assert call(tokens=0) == 0 and call(n=0, tokens=0, cu=None) == 0


def test_decode_refuses_bad_arguments(lib):
    d, t, bad = _desc(), _tables(), nb.NP_E_INVAL

    def call(layer=0, q=_rows(), heads=8, seqs=P, n=2, scale=0.1, out=_rows(), ws=P, size=1 << 40, cache=P, tables=t):
        return lib.np_attn_decode(_b(d), cache, layer, _b(tables), _b(q), heads, seqs, n, scale, _b(out), None, ws, size, None)

    assert call(size=nb.np_attn_workspace_bytes(d, 8, 2) - 1) == bad and "workspace" in lib.np_attn_last_error().decode()
    assert call(heads=6) == bad and call(heads=0) == bad and call(n=-1) == bad and call(n=1025) == bad and call(n=9, seqs=None) == bad
    assert call(layer=2) == bad and call(cache=None) == bad and call(ws=None) == bad and call(ws=P + 4) == bad
    for s in (0.0, -1.0, float("inf"), float("nan")):
        assert call(scale=s) == bad
    assert call(q=_rows(data=P + 2)) == bad and call(out=_rows(head_stride=4)) == bad
    assert call(tables=_tables(lens=None)) == bad
    assert call(n=0) == 0


def test_prompt_refuses_bad_arguments(lib):
    bad = nb.NP_E_INVAL

    def call(dtype=0, hq=8, hkv=4, hd=128, q=_rows(), k=_rows(), v=_rows(), out=_rows(), cu=P, n=2, tokens=9, scale=0.1, status=P):
        s = nb.np_attn_shape(dtype, hq, hkv, hd)
        return lib.np_attn_prompt(_b(s), _b(q), _b(k), _b(v), cu, n, tokens, scale, _b(out), None, status, None)

    assert call(dtype=3) == bad and call(hq=6) == bad and call(hkv=0) == bad and call(hd=80) == bad and call(n=0) == bad and call(n=1025) == bad
    assert call(hq=129, hkv=1) == bad and "NP_ATTN_MAX_GROUP" in lib.np_attn_last_error().decode()
    assert call(tokens=-1) == bad and call(scale=0.0) == bad and call(scale=float("nan")) == bad and call(cu=None) == bad and call(status=None) == bad
    for name in ("q", "k", "v", "out"):
        assert call(**{name: _rows(data=None)}) == bad and call(**{name: _rows(token_stride=4)}) == bad
        assert call(**{name: _rows(token_stride=0)}) == bad and call(**{name: _rows(head_stride=0)}) == bad
    assert call(tokens=0, cu=None) == 0


def test_without_a_device_calls_fail(lib):
    if torch.cuda.is_available():
        pytest.skip("a device is there")
    d, t = _desc(), _tables()
    assert lib.np_kv_free(_b(d), _b(t), P, 2, None) == nb.NP_E_CUDA
    assert lib.np_attn_decode(_b(d), P, 0, _b(t), _b(_rows()), 8, P, 2, 0.1, _b(_rows()), None, P, 1 << 40, None) == nb.NP_E_CUDA


def test_binding_refuses_host_tensors_and_other_types(lib):
    z = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(nb.NpError) as e:
        nb.np_attn_prompt(z, z, z, torch.zeros(2, dtype=torch.int32), z, torch.zeros(1, dtype=torch.int32))
    assert e.value.code == nb.NP_E_INVAL
    with pytest.raises(nb.NpError):
        nb.make_kv_desc(torch.float32, 1, 1, 64, 16, 1, 1)


def test_binding_refuses_a_cache_of_no_type(lib):
    """A description made by hand with a type that there is none of: a refusal, not an IndexError."""
    d = _desc(dtype=7)
    z = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(nb.NpError) as e:
        nb.np_kv_fork(d, z, _tables(), torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    assert e.value.code == nb.NP_E_INVAL


@pytest.mark.parametrize("short", range(5))
def test_binding_refuses_tables_that_are_too_small_or_elsewhere(lib, short):
    """Tables that would be written past their ends, or that belong to another device than the call."""
    d = _desc()
    room = [torch.cuda.current_device() if torch.cuda.is_available() else -2, d.max_seqs * d.max_pages, d.max_seqs, d.n_pages,
            nb.np_kv_sizes(d).scratch_bytes // 4]
    t = _tables()
    if not torch.cuda.is_available():
        t.room = tuple(room)
        with pytest.raises(nb.NpError) as e:
            nb.np_kv_reset(d, t)
        assert e.value.code == nb.NP_E_CUDA          # nothing to refuse but the missing device
    t.room = tuple(r - (i == short) for i, r in enumerate(room))
    with pytest.raises(nb.NpError) as e:
        nb.np_kv_reset(d, t)
    assert e.value.code == nb.NP_E_INVAL and "tables on device" in str(e.value)


def test_decode_refuses_results_on_top_of_each_other(lib):
    d, t, bad = _desc(), _tables(), nb.NP_E_INVAL

    def call(out, n):
        return lib.np_attn_decode(_b(d), P, 0, _b(t), _b(_rows()), 8, P, n, 0.1, _b(out), None, P, 1 << 40, None)

    assert call(_rows(token_stride=0), 2) == bad and call(_rows(head_stride=0), 2) == bad and "above 0" in lib.np_attn_last_error().decode()
