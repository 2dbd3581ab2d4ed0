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
