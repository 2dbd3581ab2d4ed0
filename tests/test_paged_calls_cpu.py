"""More of the paged K/V operators' boundary that needs no GPU: structures that the binding packs, arguments that came later."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2511_21759_amd import binding as B                        # noqa: E402


def test_packed_structures_are_as_long_as_the_declared_ones():
    for pack, fields, struct in ((B._PACK_PAGES, 10, B.odb_pages), (B._PACK_QK_ROWS, 21, B.odb_qk_rows), (B._PACK_ATTENTION, 20, B.odb_attention)):
        assert len(struct._fields_) == fields and len(pack(*[1] * fields)) == ctypes.sizeof(struct)
        there = struct.from_buffer_copy(pack(*range(1, fields + 1)))
        assert [int(getattr(there, name)) for name, _ in struct._fields_] == list(range(1, fields + 1))


def test_row_end_is_one_number_on_the_device_of_the_others():
    q, k, i32 = torch.zeros(3, 4, 64, dtype=torch.float16), torch.zeros(5, 2, 16, 64, dtype=torch.float16), torch.int32
    rows = dict(q=q, k=q[:, :2], v=q[:, 2:], k_pages=k, v_pages=k.clone(), table=torch.zeros(9, 32, 2), positions=torch.zeros(3, dtype=i32),
                slots=torch.zeros(3, dtype=i32))
    with pytest.raises(B.OdbError, match="CUDA"):                    # well-formed, but not on a GPU
        B.odb_qk_norm_rope(**rows, row_end=torch.zeros(4, dtype=i32)[3:])
    for bad in (torch.zeros(2, dtype=i32), torch.zeros((), dtype=i32), torch.zeros(1), torch.zeros(1, dtype=torch.int64)):
        with pytest.raises(TypeError):
            B.odb_qk_norm_rope(**rows, row_end=bad)


INVALID = -1


def qk_rows(**kw):
    """Heads 4 over 2 of 64, in place in a fused buffer of 512 elements a row."""
    big = 1 << 30
    a = dict(q=big, k=big + 2 * 256, v=big + 2 * 384, in_dtype=0, rows=5, n_heads=4, q_row=512, k_row=512, v_row=512, q_gain=None, k_gain=None, eps=1e-5,
             table=0x10000, n_pos=100, rot_dim=64, interleaved=0, positions=0x20000, slots=0x30000, q_out=big, q_out_row=512)
    a.update(kw)
    return B.odb_qk_rows(**a)


@pytest.mark.parametrize("kw", [dict(k=1 << 30), dict(v=1 << 30), dict(k=(1 << 30) + 2 * 192), dict(v=(1 << 30) + 2 * 248), dict(k=(1 << 30) - 2 * 64),
                                dict(v=(1 << 30) + 2 * 448), dict(k=(1 << 30) + 2 * 512), dict(k=(1 << 30) + 2 * 256, k_row=520), dict(v=(1 << 30) + 2 * 384, v_row=1024)])
def test_keys_and_values_that_share_elements_with_queries_in_place_are_refused(kw):
    lib, pages = B.lib(), B.odb_pages(k=0x10000, v=0x20000, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, dtype=0, page_stride=2048, head_stride=1024, pos_stride=64)
    assert lib.odb_qk_norm_rope(ctypes.byref(qk_rows(**kw)), ctypes.byref(pages), None) == INVALID
    assert b"in place" in lib.odb_last_error()
