"""odb_step_paged where it leaves the ordinary: values beyond the binary16 range, pools of another model, many rows and requests, further
turns.  Bars are those of test_gpu_paged_model.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import odb_oracle as o                                   # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402
from paper_2511_21759_amd import workloads as W                      # noqa: E402
from test_gpu_paged_model import KV_TOL, LOG_CONF, MARGIN, Paged, decide, ints       # noqa: E402

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


# ---- many rows and requests -----------------------------------------------------------------------------------------------

def random_pages(shape, model, lens, page, seed):
    """Requests of those lengths over pools of random numbers."""
    columns = -(-max(lens) // page)
    need = [-(-x // page) for x in lens]
    pg = Paged(shape, model, len(lens), columns, page, sum(need) + 1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for pool in (pg.k, pg.v):
        pool.copy_(0.4 * torch.randn(pool.shape, generator=g, device="cuda"))
    ids, tables, at = np.random.default_rng(seed).permutation(sum(need) + 1), np.full((len(lens), columns), -1, np.int32), 0
    for r, x in enumerate(need):
        tables[r, :x] = ids[at:at + x]
        at += x
    pg.tables = ints(tables)
    return pg


@pytest.mark.parametrize("n,b,head_gain", [(600, 1, None), (530, 70, None), (64, 16, 32.0)])
def test_many_requests_equal_a_few_at_a_time(n, b, head_gain):
    """One pass over all requests against passes over at most ten, from the same pools: confidences and the K/V that are stored."""
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        if head_gain is not None:
            B.odb_model_set_tensor(model, B.T_GF, 0, np.full(shape["d_model"], int(np.float32(head_gain).view(np.uint32)) >> 16, np.uint16))
        rng = np.random.default_rng(n)
        lens = [int(x) for x in rng.integers(b, b + 80, n)]
        first = [int(rng.integers(0, x - b + 1)) for x in lens]
        tokens = rng.integers(0, shape["vocab"], (n, b))
        pg = random_pages(shape, model, lens, 16, n)
        positions = np.concatenate([f + np.arange(b) for f in first])
        table = pg.tables.cpu().numpy()
        slots = np.concatenate([table[r, (f + np.arange(b)) // 16] * 16 + (f + np.arange(b)) % 16 for r, f in enumerate(first)])

        def step(lo, hi, k, v):
            return B.odb_step_paged(model, ints(tokens[lo:hi]), k, v, pg.tables[lo:hi].contiguous(), ints(first[lo:hi]), ints(lens[lo:hi]), ints(positions[lo * b:hi * b]),
                                    ints(slots[lo * b:hi * b]), pg.table, tau=0.5)
        pools = [[x.clone() for x in (pg.k, pg.v)] for _ in range(2)]
        conf, argmax, unmask = step(0, n, *pools[0])
        parts = [step(lo, min(lo + 10, n), *pools[1]) for lo in range(0, n, 10)]
        want_conf, want_argmax = (torch.cat([p[i] for p in parts]) for i in (0, 1))
        assert (conf.log() - want_conf.log()).abs().max() <= LOG_CONF
        # (a greedy token whose probability is above one half by more than the bar cannot change)
        sure = want_conf > 0.55
        assert (argmax[sure] == want_argmax[sure]).all() and (head_gain is None or sure.any())
        for x, y, before in zip(pools[0], pools[1], (pg.k, pg.v)):
            assert (x - y).abs().max() <= KV_TOL * y.abs().max()
            changed = (x != before).any(-1).any(0).any(1)                # [pages, positions]
            assert changed.flatten().nonzero().flatten().tolist() == sorted(slots.tolist())
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


def test_a_refresh_of_700_positions_equals_the_dense_one_at_the_8b_width():
    shape = dict(W.MODEL_SHAPES["8b"], n_layers=2)
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        wl = W.decode_workload(shape, 300, 400, 32, 1, 5)
        pg = Paged(shape, model, 1, 44, 16, 45)
        conf, argmax, _ = pg.forward(wl.tokens, [0], [700], skip=300)
        dense = B.odb_cache_create(model, 1, 700)
        conf_d, argmax_d = B.odb_prefill(model, dense, ints(wl.tokens), 300)
        assert conf.shape == conf_d.shape and (conf.log() - conf_d.log()).abs().max() <= LOG_CONF
        for layer in range(2):
            for kv in (0, 1):
                want = B.odb_cache_read(dense, layer, kv, 0, 0, 700, shape["n_heads"], shape["head_dim"])
                assert np.abs(pg.keys(0, layer, kv, 700) - want).max() <= KV_TOL * np.abs(want).max()
        B.odb_cache_destroy(dense)
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


def sure_of(logits):
    """Rows whose two largest probabilities are further apart than the bar's margin."""
    p = np.sort(np.exp(logits - logits.max(-1, keepdims=True)), -1)
    return (p[..., -1] - p[..., -2]) / p.sum(-1) > MARGIN


@pytest.mark.parametrize("n,b", [(24, 16), (7, 32), (3, 16)])
def test_decisions_of_steps_equal_the_dense_ones_at_the_8b_width(n, b):
    """n sequences of one length, which the dense cache takes too; a sharper last norm makes the decisions clear."""
    shape = dict(W.MODEL_SHAPES["8b"], n_layers=2)
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        B.odb_model_set_tensor(model, B.T_GF, 0, np.full(shape["d_model"], int(np.float32(12.0).view(np.uint32)) >> 16, np.uint16))
        length, off = 80, 40
        wl = W.decode_workload(shape, 30, length - 30, b, 1, 9, batch=n)
        pg = Paged(shape, model, n, 5, 16, 5 * n + 1)
        pg.forward(wl.tokens, [0] * n, [length] * n, head=False)
        dense = B.odb_cache_create(model, n, length)
        B.odb_prefill(model, dense, ints(wl.tokens), 0)
        drafts = wl.tokens[:, off:off + b]
        z = B.odb_block_step_logits(model, dense, ints(drafts[:, None]), off, shape["vocab"]).double().cpu().numpy()[:, 0]
        conf_d, argmax_d, unmask_d = (x.cpu().numpy()[:, 0] for x in B.odb_block_step(model, dense, ints(drafts[:, None]), off, 0.9))
        conf, argmax, unmask = (x.cpu().numpy() for x in pg.forward(drafts, [off] * n, [length] * n, tau=0.9))
        assert np.abs(np.log(conf) - np.log(conf_d)).max() <= LOG_CONF
        sure = sure_of(z)
        assert sure.any() and (argmax[sure] == argmax_d[sure]).all()
        for r in range(n):
            masked = drafts[r] == shape["mask_id"]
            best = np.sort(conf_d[r][masked])[-2:] if masked.sum() > 1 else np.array([0.0, 1.0])
            # the acceptance is known where no confidence is near the threshold, and, if none passes it, where the most confident leads
            if masked.any() and not (np.abs(conf_d[r] - 0.9) <= 0.9 * LOG_CONF).any() and (best[1] > 0.95 or best[1] - best[0] > 2 * LOG_CONF * best[1]):
                assert (unmask[r] == unmask_d[r]).all(), r
        B.odb_cache_destroy(dense)
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


def oracle_step(cfg, w, cache, tokens, off):
    """The block's logits in 64 bits, its K/V left in `cache` as the pages keep them."""
    b = len(tokens)
    h = w.embed_rows(tokens)
    for layer in range(cfg.n_layers):
        def kv(kn, vn, layer=layer):
            cache.k[layer][off:off + b], cache.v[layer][off:off + b] = kn, vn
            return [(slice(0, b), cache.k[layer], cache.v[layer])]
        h, _, _ = o._layer(cfg, w, layer, h, off + np.arange(b), kv)
    return o._head(cfg, w, h)


@pytest.mark.parametrize("gain", [None, 32.0])
def test_further_steps_see_the_blocks_of_earlier_ones(gain):
    """Three turns on overlapping and other blocks of ragged requests: the oracle keeps a stepped block's K/V as the pages do."""
    shape = W.MODEL_SHAPES["tiny"]
    cfg = o.Config(**shape)
    w = o.Weights(cfg, W.WEIGHT_SEED, W.WEIGHT_STD)
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        if gain is not None:
            w.set_values(o.T_GF, 0, np.full(cfg.d_model, gain, np.float32))
            B.odb_model_set_tensor(model, B.T_GF, 0, w.bits(o.T_GF, 0))
        lens, b, rng = [70, 33, 129], 16, np.random.default_rng(2)
        work = [W.decode_workload(shape, 10, x - 10, b, 1, 70 + x) for x in lens]
        pg, caches = Paged(shape, model, 3, 6, 32, 14), []
        for r, wl in enumerate(work):
            pg.forward(wl.tokens, [0], [lens[r]], which=[r], head=False)
            caches.append(o.prefill(cfg, w, wl.tokens[0], 0)[0])
        for offs in ([40, 17, 113], [48, 1, 77], [40, 9, 64]):
            drafts = rng.integers(0, shape["vocab"] - 1, (3, b))
            drafts[rng.random((3, b)) < 0.5] = shape["mask_id"]
            conf, argmax, unmask = (x.cpu().numpy() for x in pg.forward(drafts, offs, lens, tau=0.9))
            for r in range(3):
                z = oracle_step(cfg, w, caches[r], drafts[r], offs[r])
                conf_o, argmax_o = o.confidence_argmax(z)
                decide(conf[r], argmax[r], conf_o, argmax_o, z)
                unmask_o = o.threshold_unmask(drafts[r], conf_o, 0.9, cfg.mask_id)
                masked = drafts[r] == shape["mask_id"]
                best = np.sort(conf_o[masked])[-2:] if masked.sum() > 1 else np.array([0.0, 1.0])
                if not (np.abs(conf_o - 0.9) <= 0.9 * LOG_CONF).any() and (best[1] > 0.95 or best[1] - best[0] > 2 * LOG_CONF * best[1]):
                    assert (unmask[r] == unmask_o).all()
                for layer in range(cfg.n_layers):
                    for kv, want in ((0, caches[r].k[layer]), (1, caches[r].v[layer])):
                        assert np.abs(pg.keys(r, layer, kv, lens[r]) - want).max() <= KV_TOL * np.abs(want).max()
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


# ---- captured ---------------------------------------------------------------------------------------------------------------

@pytest.mark.filterwarnings("ignore:The CUDA Graph is empty")       # (of the capture that is refused)
@pytest.mark.parametrize("dense", [False, True])
def test_captured_steps_outlive_larger_calls(dense):
    """A graph holds the address of the scratch that its step uses; a larger call takes new scratch, and the graph is replayed again."""
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        lens, b, rng = [70, 33, 129], 16, np.random.default_rng(4)
        pg = random_pages(shape, model, lens, 16, 8)
        table = pg.tables.cpu().numpy()
        first = [40, 17, 100]
        positions = np.concatenate([f + np.arange(b) for f in first])
        slots = np.concatenate([table[r, (f + np.arange(b)) // 16] * 16 + (f + np.arange(b)) % 16 for r, f in enumerate(first)])
        tokens = ints(rng.integers(0, shape["vocab"], (3, b)))
        args = [ints(first), ints(lens), ints(positions), ints(slots)]
        cache = B.odb_cache_create(model, 1, 1200)
        small = W.decode_workload(shape, 20, 44, b, 1, 3)

        def step():
            if dense:
                return B.odb_block_step(model, cache, tokens[None, :1], 24, 0.5)
            return B.odb_step_paged(model, tokens, pg.k, pg.v, pg.tables, *args, pg.table, tau=0.5)
        graph = torch.cuda.CUDAGraph()
        if not dense:
            with pytest.raises(B.OdbError, match="captured"):         # nothing was allocated yet
                with torch.cuda.graph(graph):
                    step()
            graph = torch.cuda.CUDAGraph()
        B.odb_prefill(model, cache, ints(small.tokens), 0)
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            out = step()
        large = W.decode_workload(shape, 500, 700, b, 1, 5)
        for turn in range(4):
            tokens.copy_(ints(rng.integers(0, shape["vocab"], (3, b))))
            if turn in (1, 3):                                        # takes more scratch than everything before
                B.odb_prefill(model, cache, ints(large.tokens[:, :400 * turn]), 0)
                B.odb_prefill(model, cache, ints(small.tokens), 0)
                fill = [torch.full((1 << 24,), float("nan"), device="cuda") for _ in range(4)]       # what was freed would be written over
            graph.replay()
            torch.cuda.synchronize()
            got = [x.clone() for x in out]
            for x, y in zip(got, step()):
                assert torch.equal(x, y), turn
        del fill
        B.odb_model_status(model)
        B.odb_cache_destroy(cache)
    finally:
        B.odb_model_destroy(model)
