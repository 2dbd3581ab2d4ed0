"""odb_step_paged_quant where it leaves the ordinary: values beyond the binary16 range, keys that are not finite, padding, captured steps."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import quant_plain as quant                                          # noqa: E402
from oracle import odb_oracle as o                                   # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402
from paper_2511_21759_amd import workloads as W                      # noqa: E402
from test_gpu_quant_model import LOG_CONF, Pages, ints               # noqa: E402

pytestmark = pytest.mark.gpu


def one_layer():
    shape = dict(W.MODEL_SHAPES["tiny"], n_layers=1)
    model, w = B.odb_model_create(shape), o.Weights(o.Config(**shape), W.WEIGHT_SEED, W.WEIGHT_STD)
    B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)

    def put(tensor, values):
        w.set_values(getattr(o, "T_" + tensor), 0, values)
        B.odb_model_set_tensor(model, getattr(B, "T_" + tensor), 0, w.bits(getattr(o, "T_" + tensor), 0))
    emb = w.f64(o.T_EMBED, 0)[5]
    return shape, model, w, put, emb / np.sqrt(np.mean(emb * emb) + o.Config(**shape).rms_eps)


@pytest.mark.parametrize("kind,group", [("int8", 16), ("e4m3", 1)])
def test_queries_beyond_binary16_are_clamped_and_reported(kind, group):
    """One position sees itself alone, so its answer is the same whatever its query is, as long as that is a number - but for the roundings of one probability p: the
    row is fl(p s) / fl(p) of V, with p between 2^7 and 2^9 as the rounding of the reference has it, and each fl within 2^-11.  That is far inside the bar of
    confidences."""
    shape, model, w, put, hidden = one_layer()
    try:
        pg, token = Pages(shape, model, kind, group, [1, 1], 16), np.array([[5]])
        conf, argmax, _ = (x.clone() for x in pg.step(token, [0], [0], tau=0.5))
        B.odb_model_status(model)                                    # in range: clean
        big = w.f64(o.T_WQ, 0).copy()
        big[0] *= 2.0 ** 19
        put("WQ", big)
        assert abs(hidden @ w.f64(o.T_WQ, 0)[0]) > 70000
        again = pg.step(token, [0], [0], tau=0.5)
        assert (again[0].log() - conf.log()).abs().max() <= LOG_CONF
        with pytest.raises(B.OdbError, match="binary16"):
            B.odb_model_status(model)
        B.odb_model_status(model)                                    # cleared by the check
        # as a padding row it reports nothing, and is not stored
        before = [t.view(torch.int8 if t.dtype != torch.float32 else torch.int32).clone() for t in pg.codes + pg.scales]
        B.odb_step_paged_quant(model, ints(token), *pg.codes, *pg.scales, ints(pg.tables[:1]), ints([0]), ints([1]), ints([-1]), pg.table, tau=0.5)
        B.odb_model_status(model)
        for x, y in zip(before, pg.codes + pg.scales):
            assert torch.equal(x, y.view(x.dtype))
    finally:
        B.odb_model_destroy(model)


@pytest.mark.parametrize("kind,group", [("int8", 16), ("e4m3", 1)])
@pytest.mark.parametrize("tensor", ["WK", "WV"])
def test_keys_and_values_beyond_binary16_are_stored_as_they_are(tensor, kind, group):
    """Scales are 32-bit: what is beyond binary16 and finite is stored.  Nothing is reported, but that answers which values of V make too large leave binary16."""
    shape, model, w, put, hidden = one_layer()
    try:
        pg, token = Pages(shape, model, kind, group, [1], 16), np.array([[5]])
        big = w.f64(getattr(o, "T_" + tensor), 0).copy()
        big[0] *= 2.0 ** 19
        put(tensor, big)
        want = hidden @ w.f64(getattr(o, "T_" + tensor), 0)[0]       # (position 0 is not turned)
        assert abs(want) > 70000
        pg.step(token, [0], [0], head=False)
        if tensor == "WV":
            with pytest.raises(B.OdbError, match="binary16"):
                B.odb_model_status(model)
        B.odb_model_status(model)
        page, i = int(pg.tables[0, 0]), 1 if tensor == "WV" else 0
        value = quant.values(pg.codes[i][0].cpu(), pg.scales[i][0].cpu())[page, 0, 0, 0].item()
        assert abs(value - want) <= 1e-2 * abs(want)                 # (the bar of K/V; the group's largest has the largest code)
    finally:
        B.odb_model_destroy(model)


@pytest.mark.parametrize("kind,group", [("int8", 16), ("e4m3", 1)])
def test_keys_that_are_not_finite_are_reported(kind, group):
    """A table of angles so large that turned keys overflow 32 bits; queries are zero, so nothing else is out of range."""
    shape, model, w, put, hidden = one_layer()
    try:
        pg, token = Pages(shape, model, kind, group, [1], 16), np.array([[5]])
        put("WQ", np.zeros_like(w.f64(o.T_WQ, 0)))
        key = w.f64(o.T_WK, 0).copy()
        key[0] *= 100 / (hidden @ key[0])
        put("WK", key)
        assert hidden @ w.f64(o.T_WK, 0)[0] > 50
        pg.step(token, [0], [0], tau=0.5)
        B.odb_model_status(model)
        pg.table = pg.table * 3e37                                   # 50 times that is beyond 32 bits, ten times is not
        conf, argmax, unmask = pg.step(token, [0], [0], head=True)
        with pytest.raises(B.OdbError, match="binary16"):
            B.odb_model_status(model)
        page = int(pg.tables[0, 0])
        assert quant.numbers(pg.codes[0][0, page, 0, 0].cpu())[0] == quant.MOST[kind]
        assert torch.isfinite(pg.scales[0][0, page, :, 0]).all()
    finally:
        B.odb_model_destroy(model)


@pytest.mark.filterwarnings("ignore:The CUDA Graph is empty")       # (of the capture that is refused)
@pytest.mark.parametrize("kind,group", [("int8", 16), ("e4m3", 1)])
def test_captured_steps_outlive_larger_calls(kind, group):
    """A graph holds the address of the scratch that its step uses; a larger call takes new scratch, and the graph is replayed again."""
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        lens, first, b, rng = [70, 33, 129], [40, 17, 100], 16, np.random.default_rng(4)
        pg = Pages(shape, model, kind, group, lens, 16)
        tokens = ints(rng.integers(0, shape["vocab"], (3, b)))
        args = [ints(pg.tables), ints(first), ints(lens), ints(pg.positions(first, b))]
        cache = B.odb_cache_create(model, 1, 1200)

        def step(pools):
            return B.odb_step_paged_quant(model, tokens, *pools, *args, pg.table, tau=0.5)
        mine = pg.codes + pg.scales
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(B.OdbError, match="captured"):             # nothing was allocated yet
            with torch.cuda.graph(graph):
                step(mine)
        graph = torch.cuda.CUDAGraph()
        for r in range(3):                                            # all positions hold numbers
            pg.step(rng.integers(0, shape["vocab"], (1, lens[r])), [0], [r], head=False)
        step(mine)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            out = step(mine)
        large = W.decode_workload(shape, 500, 700, b, 1, 5)
        for turn in range(4):
            tokens.copy_(ints(rng.integers(0, shape["vocab"], (3, b))))
            if turn in (1, 3):                                        # takes more scratch than everything before
                B.odb_prefill(model, cache, ints(large.tokens[:, :400 * turn]), 0)
                fill = [torch.full((1 << 24,), float("nan"), device="cuda") for _ in range(4)]       # what was freed would be written over
            eager = [t.view(torch.int8).clone().view(t.dtype) for t in mine]
            graph.replay()
            torch.cuda.synchronize()
            got = [x.clone() for x in out]
            for x, y in zip(got, step(eager)):
                assert torch.equal(x, y), turn
            for x, y in zip(mine, eager):
                assert torch.equal(x.view(torch.int8), y.view(torch.int8)), turn
        del fill
        B.odb_model_status(model)
        B.odb_cache_destroy(cache)
    finally:
        B.odb_model_destroy(model)
