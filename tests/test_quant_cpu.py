"""Refusals of the paged K/V operators in 8 bits: arguments are checked on the host, so none of this needs a GPU."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2511_21759_amd import binding as B                        # noqa: E402

INVALID = -1
A = [0x10000 * (i + 1) for i in range(24)]                # addresses that are only compared, never followed
BIG = 1 << 30


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2511_21759_amd.build import build_library
        build_library()
    return B.lib()


def pages(**kw):
    a = dict(k=A[0], v=A[1], k_scale=A[2], v_scale=A[3], n_pages=10, page_size=32, n_kv_heads=2, head_dim=64, codes=3, group=16, dtype=0, page_stride=4096,
             head_stride=2048, pos_stride=64, scale_page_stride=4, scale_head_stride=2)
    a.update(kw)
    return B.odb_quant_pages(**a)


def rows(**kw):
    """Heads 4 over 2 of 64, in place in a fused buffer of 512 elements a row."""
    a = dict(q=BIG, k=BIG + 2 * 256, v=BIG + 2 * 384, in_dtype=0, rows=5, n_heads=4, q_row=512, k_row=512, v_row=512, q_gain=None, k_gain=None, eps=1e-5,
             table=A[4], n_pos=100, rot_dim=64, interleaved=0, positions=A[5], q_out=BIG, q_out_row=512, cu_rows=A[6], first_pos=None, kv_len=A[7],
             tables=A[8], columns=4, n=3, odd=None)
    a.update(kw)
    return B.odb_quant_rows(**a)


def attention(**kw):
    a = dict(q=BIG, out=2 * BIG, q_row=256, out_row=256, cu_rows=A[6], first_pos=None, kv_len=A[7], tables=A[8], columns=4, n=3, rows=5, n_heads=4,
             scale=0.125, causal=1, window=0, sinks=0, max_rows=0, max_len=0, workspace=None, workspace_bytes=0)
    a.update(kw)
    return B.odb_attention(**a)


BAD_PAGES = [dict(k=None), dict(v=A[1] + 8), dict(k_scale=None), dict(v_scale=A[3] + 4), dict(n_pages=0), dict(page_size=20), dict(page_size=8), dict(n_kv_heads=0),
             dict(head_dim=96), dict(codes=2), dict(codes=5), dict(dtype=2), dict(group=0), dict(group=8), dict(group=64), dict(group=24), dict(page_stride=-16),
             dict(head_stride=8), dict(pos_stride=72), dict(pos_stride=1 << 24), dict(scale_page_stride=-4), dict(group=1, scale_page_stride=66, scale_head_stride=32)]


@pytest.mark.parametrize("kw", BAD_PAGES)
def test_pages_that_are_refused(lib, kw):
    p = ctypes.byref(pages(**kw))
    assert lib.odb_qk_norm_rope_quant(ctypes.byref(rows()), p, None) == INVALID and b"qk_norm_rope_quant" in lib.odb_last_error()
    assert lib.odb_paged_attention_quant(ctypes.byref(attention()), p, None) == INVALID and b"paged_attention_quant" in lib.odb_last_error()
    if "dtype" not in kw:
        assert lib.odb_paged_read_quant(p, A[9], 3, 0, BIG, 2 * BIG, 128, 128, None) == INVALID and b"paged_read_quant" in lib.odb_last_error()


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=(1 << 24) + 1), dict(n_heads=0), dict(n_heads=65537), dict(in_dtype=1), dict(in_dtype=3), dict(q=None), dict(k=BIG + 4),
                                dict(q_row=255), dict(k_row=120), dict(v_row=516), dict(q_out=None), dict(table=None), dict(positions=None), dict(q_gain=A[9]),
                                dict(q_gain=A[9], k_gain=A[9] + 4), dict(q_gain=A[9], k_gain=A[10], eps=-1.0), dict(n_pos=0), dict(n_pos=(1 << 22) + 1), dict(rot_dim=0),
                                dict(rot_dim=24), dict(rot_dim=80), dict(q_out=BIG + 512), dict(k=BIG), dict(v=BIG + 2 * 440), dict(n=0), dict(n=4097),
                                dict(cu_rows=None), dict(kv_len=None), dict(tables=None), dict(columns=0), dict(columns=1 << 26)])
def test_rows_that_are_refused(lib, kw):
    assert lib.odb_qk_norm_rope_quant(ctypes.byref(rows(**kw)), ctypes.byref(pages()), None) == INVALID
    assert b"qk_norm_rope_quant" in lib.odb_last_error()


@pytest.mark.parametrize("kw", [dict(n=0), dict(n=4097), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(n_heads=3), dict(n_heads=0), dict(columns=0), dict(columns=1 << 26),
                                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=3e38), dict(window=-1), dict(sinks=-1), dict(sinks=(1 << 30) + 1),
                                dict(max_rows=-1), dict(max_len=-1), dict(q=None), dict(out=BIG + 8), dict(q_row=252), dict(out_row=100), dict(out=BIG + 1024),
                                dict(kv_len=None), dict(tables=None), dict(cu_rows=None)])
def test_attention_that_is_refused(lib, kw):
    assert lib.odb_paged_attention_quant(ctypes.byref(attention(**kw)), ctypes.byref(pages()), None) == INVALID
    assert b"paged_attention_quant" in lib.odb_last_error()


@pytest.mark.parametrize("args", [(None, 3, 0, BIG, 2 * BIG, 128, 128), (A[9], -1, 0, BIG, 2 * BIG, 128, 128), (A[9], (1 << 24) + 1, 0, BIG, 2 * BIG, 128, 128),
                                  (A[9], 3, 3, BIG, 2 * BIG, 128, 128), (A[9], 3, -1, BIG, 2 * BIG, 128, 128), (A[9], 3, 0, None, 2 * BIG, 128, 128),
                                  (A[9], 3, 0, BIG, 2 * BIG + 8, 128, 128), (A[9], 3, 0, BIG, 2 * BIG, 120, 128), (A[9], 3, 0, BIG, 2 * BIG, 128, 130),
                                  (A[9], 3, 0, BIG, BIG, 128, 128), (A[9], 3, 0, BIG, BIG + 2 * 120, 256, 256), (A[9], 3, 0, BIG, BIG + 2 * 136, 256, 256),
                                  (A[9], 3, 2, BIG, BIG + 512, 256, 264), (A[9], 1, 0, BIG, BIG + 128, 256, 256)])
def test_read_back_that_is_refused(lib, args):
    assert lib.odb_paged_read_quant(ctypes.byref(pages()), *args, None) == INVALID
    assert b"paged_read_quant" in lib.odb_last_error()


def test_null_arguments_and_launches_of_too_many_threads(lib):
    assert lib.odb_qk_norm_rope_quant(None, ctypes.byref(pages()), None) == INVALID
    assert lib.odb_qk_norm_rope_quant(ctypes.byref(rows()), None, None) == INVALID
    assert lib.odb_paged_attention_quant(None, ctypes.byref(pages()), None) == INVALID
    assert lib.odb_paged_attention_quant(ctypes.byref(attention()), None, None) == INVALID
    assert lib.odb_paged_attention_quant_workspace(None, None) == INVALID
    assert lib.odb_paged_read_quant(None, A[9], 3, 0, BIG, 2 * BIG, 128, 128, None) == INVALID
    wide = dict(rows=1 << 24, n_heads=96, q_row=8192, k_row=8192, v_row=8192, q_out=1 << 60, q_out_row=6144)
    assert lib.odb_qk_norm_rope_quant(ctypes.byref(rows(**wide)), ctypes.byref(pages()), None) == INVALID
    assert b"too many for one launch" in lib.odb_last_error()
    many = pages(n_kv_heads=8192, head_dim=256, page_stride=1 << 28, head_stride=1 << 13, pos_stride=256, scale_page_stride=1 << 14, scale_head_stride=2)
    assert lib.odb_paged_read_quant(ctypes.byref(many), A[9], 1 << 13, 0, BIG, 1 << 50, 8192 * 256, 8192 * 256, None) == INVALID
    assert b"too many for one launch" in lib.odb_last_error()
    lots = lambda **kw: lib.odb_paged_attention_quant_workspace(ctypes.byref(attention(rows=1 << 24, **kw)), ctypes.byref(pages()))        # noqa: E731
    assert lots(n_heads=64) == 0 and lots(n_heads=66) == INVALID


def test_no_rows_need_no_workspace_and_launch_nothing(lib):
    assert lib.odb_paged_attention_quant_workspace(ctypes.byref(attention(rows=0, columns=1 << 20, n=1)), ctypes.byref(pages())) == 0
    assert lib.odb_paged_attention_quant(ctypes.byref(attention(rows=0)), ctypes.byref(pages()), None) == 0
    assert lib.odb_qk_norm_rope_quant(ctypes.byref(rows(rows=0)), ctypes.byref(pages()), None) == 0
    assert lib.odb_paged_read_quant(ctypes.byref(pages()), A[9], 0, 0, BIG, 2 * BIG, 128, 128, None) == 0


def test_a_workspace_that_is_too_small(lib):
    long = dict(rows=1, n=1, columns=1 << 15, max_rows=1)
    need = lib.odb_paged_attention_quant_workspace(ctypes.byref(attention(**long)), ctypes.byref(pages()))
    assert need > 0
    for kw in (dict(), dict(workspace=A[9], workspace_bytes=need - 1), dict(workspace=A[9] + 128, workspace_bytes=need + 256)):
        assert lib.odb_paged_attention_quant(ctypes.byref(attention(**long, **kw)), ctypes.byref(pages()), None) == INVALID
        assert b"workspace" in lib.odb_last_error()


def test_packed_structures_are_as_long_as_the_declared_ones():
    for pack, fields, struct in ((B._PACK_QUANT_PAGES, 16, B.odb_quant_pages), (B._PACK_QUANT_ROWS, 26, B.odb_quant_rows)):
        assert len(struct._fields_) == fields and len(pack(*[1] * fields)) == ctypes.sizeof(struct)
        there = struct.from_buffer_copy(pack(*range(1, fields + 1)))
        assert [int(getattr(there, name)) for name, _ in struct._fields_] == list(range(1, fields + 1))


def good(codes=torch.int8):
    i32, q = torch.int32, torch.zeros(3, 4, 64, dtype=torch.float16)
    pool, scale = torch.zeros(5, 2, 32, 64, dtype=torch.int8).view(codes), torch.zeros(5, 2, 2)
    pools = dict(k_pages=pool, v_pages=pool.clone(), k_scale=scale, v_scale=scale.clone())
    return q, pools, dict(tables=torch.zeros(2, 4, dtype=i32), kv_len=torch.zeros(2, dtype=i32), cu_rows=torch.zeros(3, dtype=i32))


@pytest.mark.parametrize("codes", [torch.int8, torch.float8_e4m3fn])
def test_tensors_that_do_not_fit_are_refused(codes):
    q, pools, requests = good(codes)
    rope = dict(table=torch.zeros(9, 32, 2), positions=torch.zeros(3, dtype=torch.int32))
    store = lambda q=q, **kw: B.odb_qk_norm_rope_quant(q, q[:, :2], q[:, 2:], **{**pools, **requests, **rope, **kw})       # noqa: E731
    attend = lambda q=q, **kw: B.odb_paged_attention_quant(q, **{**pools, **requests, **kw}, causal=True)                 # noqa: E731
    read = lambda slots=torch.zeros(3, dtype=torch.int32), **kw: B.odb_paged_read_quant(**{**pools, **kw}, slots=slots)   # noqa: E731
    for call in (store, attend, read):
        with pytest.raises(B.OdbError, match="CUDA"):                    # well-formed, but not on a GPU
            call()
        for bad in (dict(k_pages=pools["k_pages"].float()), dict(v_pages=pools["v_pages"][:, :, :16]), dict(k_scale=pools["k_scale"].double()),
                    dict(v_scale=pools["v_scale"][:, :, :1]), dict(k_scale=pools["k_scale"][..., None]), dict(k_scale=torch.zeros(5, 2, 0), v_scale=torch.zeros(5, 2, 0)),
                    dict(k_scale=torch.zeros(5, 2, 3), v_scale=torch.zeros(5, 2, 3)), dict(k_pages=pools["k_pages"].view(torch.uint8))):
            with pytest.raises(TypeError):
                call(**bad)
    with pytest.raises(TypeError):
        attend(q.float())
    with pytest.raises(TypeError, match="dtype"):
        store(q.float())
    for bad in (dict(kv_len=torch.zeros(3, dtype=torch.int32)), dict(tables=torch.zeros(8, dtype=torch.int32)), dict(cu_rows=torch.zeros(2, dtype=torch.int32)),
                dict(tables=torch.zeros(2, 4, dtype=torch.int64))):
        for call in (store, attend):
            with pytest.raises(TypeError):
                call(**bad)
    for call in (store, attend):
        with pytest.raises(ValueError, match="cu_rows"):
            call(cu_rows=None)
    for bad in (torch.zeros(2, dtype=torch.int32), torch.zeros(1), torch.zeros((), dtype=torch.int32)):
        with pytest.raises(TypeError):
            store(odd=bad)
    with pytest.raises(TypeError):
        read(dtype=torch.int8)
    with pytest.raises(TypeError):
        read(torch.zeros(3, dtype=torch.int64))
    with pytest.raises(TypeError):
        read(out=(torch.zeros(3, 2, 64), torch.zeros(3, 2, 32)))
