"""odb_step_paged where it leaves the ordinary: values beyond the binary16 range, pools of another model, many rows and requests.  Bars
are those of test_gpu_paged_model.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import odb_oracle as o                                   # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402
from paper_2511_21759_amd import workloads as W                      # noqa: E402
from test_gpu_paged_model import KV_TOL, LOG_CONF, Paged, ints       # noqa: E402

pytestmark = pytest.mark.gpu


def test_pools_of_another_number_of_layers_are_refused():
    """Pools of fewer layers than the model has (a part of them, or those of another model) would be left behind their end."""
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        pg = Paged(dict(shape, n_layers=3), model, 1, 4, 16, 5)
        args = dict(tokens=ints([[1, 2]]), tables=ints([[0, 1, 2, 3]]), first_pos=ints([0]), kv_len=ints([2]), positions=ints([0, 1]), slots=ints([0, 1]), table=pg.table)
        for layers in (1, 3):
            before = [x[:layers].clone() for x in (pg.k, pg.v)]
            with pytest.raises(B.OdbError, match="%d layers; the model has 2" % layers):
                B.odb_step_paged(model, k_pages=pg.k[:layers], v_pages=pg.v[:layers], **args)
            torch.cuda.synchronize()
            for x, y in zip(before, (pg.k, pg.v)):
                assert torch.equal(x.nan_to_num(7.0), y[:layers].nan_to_num(7.0))
        B.odb_step_paged(model, k_pages=pg.k[:2], v_pages=pg.v[:2], **args)
        assert not pg.k[:2, 0, :, :2].isnan().any() and pg.k[2].isnan().all()
    finally:
        B.odb_model_destroy(model)
