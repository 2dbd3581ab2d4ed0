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


@pytest.mark.parametrize("tensor", ["WQ", "WK", "WV"])
@pytest.mark.parametrize("sign", [1, -1])
def test_values_beyond_binary16_are_clamped_and_reported_as_in_the_dense_calls(tensor, sign):
    """One position sees itself alone.  Where K overflows, Q has the opposite sign in that channel: the score is minus infinity if
    K is not clamped, and nothing else shows that it was."""
    shape = dict(W.MODEL_SHAPES["tiny"], n_layers=1)
    cfg, model = o.Config(**shape), B.odb_model_create(shape)
    try:
        w = o.Weights(cfg, W.WEIGHT_SEED, W.WEIGHT_STD)
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        pg, token = Paged(shape, model, 1, 4, 16, 5), np.array([[5]])
        pg.forward(token, [0], [1], tau=0.5)
        B.odb_model_status(model)                                    # in range: clean
        big = w.f64(getattr(o, "T_" + tensor), 0).copy()
        big[0] *= 2.0 ** 19                                          # the first channel of head 0, which position 0 does not turn
        w.set_values(getattr(o, "T_" + tensor), 0, big)
        B.odb_model_set_tensor(model, getattr(B, "T_" + tensor), 0, w.bits(getattr(o, "T_" + tensor), 0))
        if tensor == "WK":
            other = w.f64(o.T_WQ, 0).copy()
            other[0] = sign * big[0] * 2.0 ** -20
            w.set_values(o.T_WQ, 0, other)
            B.odb_model_set_tensor(model, B.T_WQ, 0, w.bits(o.T_WQ, 0))
        emb = w.f64(o.T_EMBED, 0)[5]
        hidden = emb / np.sqrt(np.mean(emb * emb) + cfg.rms_eps)
        assert abs(hidden @ w.f64(getattr(o, "T_" + tensor), 0)[0]) > 70000
        dense = B.odb_cache_create(model, 1, 1)
        B.odb_prefill(model, dense, ints(token), 0)
        with pytest.raises(B.OdbError, match="binary16"):
            B.odb_model_status(model)
        pg.forward(token, [0], [1], tau=0.5)
        with pytest.raises(B.OdbError, match="binary16"):
            B.odb_model_status(model)
        B.odb_model_status(model)                                    # cleared by the check
        for kv in (0, 1):
            want, got = B.odb_cache_read(dense, 0, kv, 0, 0, 1, cfg.n_heads, cfg.head_dim), pg.keys(0, 0, kv, 1)
            assert np.isfinite(got).all() and np.abs(got - want).max() <= KV_TOL * np.abs(want).max()
        if tensor != "WQ":
            assert np.abs(pg.keys(0, 0, tensor == "WV", 1)).max() == 65504.0
        B.odb_cache_destroy(dense)
    finally:
        B.odb_model_destroy(model)


def test_padding_rows_report_nothing():
    """What a padding row holds means nothing, so it reports nothing: its token's K would leave the binary16 range."""
    shape = dict(W.MODEL_SHAPES["tiny"], n_layers=1)
    cfg, model = o.Config(**shape), B.odb_model_create(shape)
    try:
        w = o.Weights(cfg, W.WEIGHT_SEED, W.WEIGHT_STD)
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        big = w.f64(o.T_WK, 0).copy()
        big[0] = 0.0
        emb = w.f64(o.T_EMBED, 0)
        apart = emb[5] - emb[9] * (emb[5] @ emb[9]) / (emb[9] @ emb[9])
        big[0] = apart / np.abs(apart).max() * 60000                 # (nearly) nothing of token 9
        w.set_values(o.T_WK, 0, big)
        B.odb_model_set_tensor(model, B.T_WK, 0, w.bits(o.T_WK, 0))
        k = [float((e / np.sqrt(np.mean(e * e) + cfg.rms_eps)) @ w.f64(o.T_WK, 0)[0]) for e in (emb[5], emb[9])]
        assert abs(k[0]) > 100000 and abs(k[1]) < 30000
        pg = Paged(shape, model, 2, 4, 16, 9)
        pg.forward(np.array([[9], [9]]), [0, 0], [1, 1], head=False)
        B.odb_model_status(model)
        B.odb_step_paged(model, ints([[9], [5]]), pg.k, pg.v, pg.tables, ints([0, 0]), ints([1, 0]), ints([0, -1]), ints([int(pg.tables[0, 0]) * 16, -1]), pg.table,
                         tau=0.5)
        B.odb_model_status(model)
        pg.forward(np.array([[9], [5]]), [0, 0], [1, 1], tau=0.5)
        with pytest.raises(B.OdbError, match="binary16"):
            B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)
