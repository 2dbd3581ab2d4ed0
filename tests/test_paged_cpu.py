"""Refusals of the paged K/V operators: arguments are checked on the host, so none of this needs a GPU."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2511_21759_amd import binding as B                        # noqa: E402


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2511_21759_amd.build import build_library
        build_library()
    return B.lib()


INVALID = -1
A = [0x10000 * (i + 1) for i in range(24)]                # addresses that are only compared, never followed


def tables_args(**kw):
    a = dict(held=A[0], wanted=A[1], n=4, page_size=16, tables=A[2], columns=8, free_pages=A[3], n_pages=64, n_free=A[4], row_first=A[5],
             row_count=A[6], len=A[7], cu_rows=A[8], slots=A[9], positions=A[10], rows_cap=100, state=A[11])
    a.update(kw)
    return [*a.values(), None]


@pytest.mark.parametrize("kw", [dict(held=None), dict(state=None), dict(positions=None), dict(n=0), dict(n=4097), dict(page_size=8), dict(page_size=24),
                                dict(page_size=8192), dict(columns=0), dict(columns=1 << 27), dict(n_pages=0), dict(n_pages=1 << 27), dict(rows_cap=0),
                                dict(rows_cap=(1 << 24) + 1), dict(len=A[0]), dict(len=A[0] + 12), dict(state=A[4]), dict(cu_rows=A[7] + 12),
                                dict(slots=A[10]), dict(tables=A[3] + 252), dict(row_first=A[9] + 396)])
def test_page_tables_refuses(lib, kw):
    assert lib.odb_page_tables(*tables_args(**kw)) == INVALID
    assert b"page_tables" in lib.odb_last_error()


@pytest.mark.parametrize("n_pos,rot,rope", [
    (0, 64, {}), ((1 << 22) + 1, 64, {}), (10, 0, {}), (10, 63, {}), (10, 258, {}), (10, 64, dict(base=1.0)), (10, 64, dict(base=float("nan"))),
    (10, 64, dict(scaling=4)), (10, 64, dict(scaling=-1)), (10, 64, dict(scaling=1, factor=0.5)), (10, 64, dict(scaling=2, factor=float("inf"))),
    (10, 64, dict(scaling=3, factor=2.0)), (10, 64, dict(scaling=3, factor=2.0, original_len=100, beta_fast=1.0)),
    (10, 64, dict(scaling=3, factor=2.0, original_len=100, beta_slow=-1.0)), (10, 64, dict(magnitude=-1.0)), (10, 64, dict(magnitude=float("nan")))])
def test_rope_table_refuses(lib, n_pos, rot, rope):
    r = B.odb_rope(**dict(dict(base=10000.0, scaling=0, factor=1.0, original_len=0, beta_fast=32.0, beta_slow=1.0, magnitude=0.0), **rope))
    assert lib.odb_rope_table(A[0], n_pos, rot, ctypes.byref(r), None) == INVALID
    assert lib.odb_rope_table(None, 10, 64, ctypes.byref(r), None) == INVALID
    assert lib.odb_rope_table(A[0], 10, 64, None, None) == INVALID


def pages(**kw):
    a = dict(k=A[0], v=A[1], n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, dtype=0, page_stride=2048, head_stride=1024, pos_stride=64)
    a.update(kw)
    return B.odb_pages(**a)


BAD_PAGES = [dict(k=None), dict(v=A[1] + 8), dict(n_pages=0), dict(page_size=20), dict(n_kv_heads=0), dict(head_dim=96), dict(dtype=2), dict(dtype=-1),
             dict(page_stride=-8), dict(head_stride=4), dict(pos_stride=1 << 24)]


def qk_rows(**kw):
    big = 1 << 30
    a = dict(q=big, k=2 * big, v=3 * big, in_dtype=0, rows=5, n_heads=4, q_row=256, k_row=128, v_row=128, q_gain=A[2], k_gain=A[3], eps=1e-5, table=A[4],
             n_pos=100, rot_dim=64, interleaved=0, positions=A[5], slots=A[6], q_out=4 * big, q_out_row=256)
    a.update(kw)
    return B.odb_qk_rows(**a)


@pytest.mark.parametrize("kw", [dict(q=None), dict(k=None), dict(v=(3 << 30) + 2), dict(q_out=None), dict(in_dtype=1), dict(in_dtype=3), dict(rows=-1),
                                dict(rows=(1 << 24) + 1), dict(rows=1 << 24, n_heads=200), dict(n_heads=0), dict(q_row=248), dict(k_row=132), dict(v_row=120), dict(q_out_row=-256),
                                dict(q_gain=None), dict(k_gain=A[3] + 4), dict(eps=-1.0), dict(eps=float("nan")), dict(table=None), dict(n_pos=0),
                                dict(rot_dim=8), dict(rot_dim=72), dict(rot_dim=24), dict(positions=None), dict(slots=None), dict(q_out=(1 << 30) + 256),
                                dict(q_out=2 << 30), dict(q_out=(3 << 30) - 2048), dict(q_out=1 << 30, in_dtype=2), dict(q_out=1 << 30, q_out_row=264)])
def test_qk_norm_rope_refuses(lib, kw):
    assert lib.odb_qk_norm_rope(ctypes.byref(qk_rows(**kw)), ctypes.byref(pages()), None) == INVALID
    assert b"qk_norm_rope" in lib.odb_last_error()


def attention(**kw):
    a = dict(q=1 << 30, out=2 << 30, q_row=256, out_row=256, cu_rows=A[2], first_pos=None, kv_len=A[3], tables=A[4], columns=8, n=3, rows=5, n_heads=4,
             scale=0.125, causal=1, window=0, sinks=0, max_rows=0, max_len=0, workspace=None, workspace_bytes=0)
    a.update(kw)
    return B.odb_attention(**a)


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(kv_len=None), dict(tables=None), dict(q=(1 << 30) + 4), dict(q_row=8), dict(out_row=260),
                                dict(n=0), dict(n=4097), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(n_heads=3), dict(n_heads=0), dict(columns=0),
                                dict(columns=1 << 28), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38),
                                dict(window=-1), dict(sinks=-1), dict(window=(1 << 30) + 1), dict(max_rows=-1), dict(max_len=-1), dict(out=(1 << 30) + 512),
                                dict(cu_rows=None), dict(columns=4000), dict(columns=4000, workspace=A[5] + 16, workspace_bytes=1 << 30),
                                dict(columns=4000, workspace=A[5], workspace_bytes=100)])
def test_paged_attention_refuses(lib, kw):
    assert lib.odb_paged_attention(ctypes.byref(attention(**kw)), ctypes.byref(pages()), None) == INVALID
    assert b"paged_attention" in lib.odb_last_error()


@pytest.mark.parametrize("kw", BAD_PAGES)
def test_pools_that_are_refused(lib, kw):
    p = pages(**kw)
    assert lib.odb_paged_attention(ctypes.byref(attention()), ctypes.byref(p), None) == INVALID
    assert lib.odb_qk_norm_rope(ctypes.byref(qk_rows()), ctypes.byref(p), None) == INVALID
    if not {"k", "v"} & set(kw):
        assert lib.odb_paged_attention_workspace(ctypes.byref(attention()), ctypes.byref(p)) == INVALID


def test_null_structures(lib):
    assert lib.odb_paged_attention(None, ctypes.byref(pages()), None) == INVALID
    assert lib.odb_paged_attention(ctypes.byref(attention()), None, None) == INVALID
    assert lib.odb_qk_norm_rope(None, ctypes.byref(pages()), None) == INVALID
    assert lib.odb_qk_norm_rope(ctypes.byref(qk_rows()), None, None) == INVALID
    assert lib.odb_paged_attention_workspace(None, None) == INVALID
    assert lib.odb_step_paged(None, None, ctypes.byref(pages()), None) == INVALID


def test_launches_of_too_many_threads_are_refused(lib):
    # a launch has fewer than 2^32 threads
    size = lambda **kw: lib.odb_paged_attention_workspace(ctypes.byref(attention(rows=1 << 24, **kw)), ctypes.byref(pages()))        # noqa: E731
    assert size(n_heads=64) == 0
    for kw in (dict(n_heads=66), dict(n_heads=100), dict(n_heads=60, max_rows=1)):
        assert size(**kw) == INVALID
        assert b"too many for one launch" in lib.odb_last_error()
    wide = dict(rows=1 << 24, n_heads=60, q_row=3840, q_out=1 << 30, q_out_row=3840)          # four waves a row
    assert lib.odb_qk_norm_rope(ctypes.byref(qk_rows(**wide)), ctypes.byref(pages()), None) == INVALID
    assert b"too many for one launch" in lib.odb_last_error()


def test_no_rows_need_no_workspace(lib):
    assert lib.odb_paged_attention_workspace(ctypes.byref(attention(columns=4000, rows=0)), ctypes.byref(pages())) == 0
    assert lib.odb_paged_attention(ctypes.byref(attention(columns=4000, rows=0)), ctypes.byref(pages()), None) == 0
    assert lib.odb_qk_norm_rope(ctypes.byref(qk_rows(rows=0)), ctypes.byref(pages()), None) == 0


def test_workspace_grows_with_rows_and_is_none_for_short_keys(lib):
    size = lambda **kw: lib.odb_paged_attention_workspace(ctypes.byref(attention(**kw)), ctypes.byref(pages()))        # noqa: E731
    assert size(columns=8) == 0 and size(columns=4000, max_len=100) == 0
    assert 0 < size(columns=4000) <= size(columns=4000, rows=400, max_rows=3)
    assert size(columns=4000, rows=1 << 24) == 0                     # row tiles enough for every CU: no split


def test_binding_refuses_tensors():
    q = torch.zeros(3, 4, 64, dtype=torch.float16)
    k = torch.zeros(5, 2, 16, 64, dtype=torch.float16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)               # noqa: E731
    ok = dict(q=q, k_pages=k, v_pages=k.clone(), tables=i32(3, 4), kv_len=i32(3), causal=True)
    with pytest.raises(B.OdbError, match="CUDA"):                    # well-formed, but not on a GPU
        B.odb_paged_attention(**ok)
    for kw in (dict(q=q.bfloat16()), dict(q=q[:, :, ::2]), dict(k_pages=k[:, :, :, ::2]), dict(v_pages=k.bfloat16()), dict(tables=i32(3)),
               dict(kv_len=i32(4)), dict(kv_len=torch.zeros(3)), dict(cu_rows=i32(3)), dict(first_pos=i32(3, 1)), dict(tables=i32(4, 3).t()),
               dict(out=q.float()), dict(out=torch.zeros(3, 4, 128, dtype=torch.float16)), dict(workspace=i32(9))):
        with pytest.raises(TypeError):
            B.odb_paged_attention(**dict(ok, **kw))
    with pytest.raises(ValueError):
        B.odb_paged_attention(**dict(ok, tables=i32(2, 4), kv_len=i32(2)))
    rows = dict(q=q, k=q[:, :2], v=q[:, 2:], k_pages=k, v_pages=k.clone(), table=torch.zeros(9, 32, 2), positions=i32(3), slots=i32(3))
    with pytest.raises(B.OdbError, match="CUDA"):
        B.odb_qk_norm_rope(**rows)
    for kw in (dict(k=q[:, :3]), dict(v=q[:, 2:].float()), dict(table=torch.zeros(9, 32)), dict(table=torch.zeros(9, 32, 2).double()), dict(positions=i32(4)),
               dict(slots=torch.zeros(3)), dict(q_gain=torch.zeros(32)), dict(out=q.float()), dict(q=q.double(), k=q[:, :2].double(), v=q[:, 2:].double())):
        with pytest.raises(TypeError):
            B.odb_qk_norm_rope(**dict(rows, **kw))
    with pytest.raises(ValueError):
        B.odb_rope_table(8, 64, 10000.0, scaling="other", device="cpu")
    with pytest.raises(TypeError):
        B.odb_rope_table(8, 64, 10000.0, out=torch.zeros(8, 64))
    tables = dict(held=i32(3), wanted=i32(3), tables=i32(3, 4), free_pages=i32(9), n_free=i32(1), page_size=16, n_pages=9, rows_cap=5)
    with pytest.raises(B.OdbError, match="CUDA"):
        B.odb_page_tables(**tables)
    for kw in (dict(wanted=i32(4)), dict(tables=i32(4, 4)), dict(tables=i32(3)), dict(free_pages=i32(8)), dict(n_free=i32(2)), dict(row_first=i32(1)),
               dict(row_count=torch.zeros(3)), dict(slots=i32(5), positions=i32(6)), dict(held=i32(3, 1))):
        with pytest.raises(TypeError):
            B.odb_page_tables(**dict(tables, **kw))
