"""The model's forward over paged K/V (odb_step_paged): requests of different lengths refreshed and stepped together, against the
oracle request by request and against the dense cache's calls.  Bars are those of the dense calls: logarithms of confidences within
5e-2, K/V within 1e-2 of the layer's largest value, decisions exact where the oracle's margin is above 1e-2."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import odb_oracle as o                                   # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402
from paper_2511_21759_amd import workloads as W                      # noqa: E402

pytestmark = pytest.mark.gpu
LOG_CONF, KV_TOL, MARGIN, TAU_BAND = 5e-2, 1e-2, 1e-2, 1e-3


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Paged:
    """Pages, tables and lengths of some requests over one model."""

    def __init__(self, shape, model, n, columns, page, n_pages):
        self.shape, self.model, self.page, self.n_pages = shape, model, page, n_pages
        size = (shape["n_layers"], n_pages, shape["n_heads"], page, shape["head_dim"])
        self.k, self.v = (torch.full(size, float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
        self.tables, self.held = ints(np.full((n, columns), -1)), ints([0] * n)
        self.free, self.n_free = ints(np.random.default_rng(3).permutation(n_pages)), ints([n_pages])
        self.table = B.odb_rope_table(columns * page, shape["head_dim"], shape["rope_base"])

    def forward(self, tokens, first, wanted, which=None, **kw):
        """tokens [n, b] at positions first[r] .. of the requests `which` (all), which then have wanted[r] positions."""
        n, b = tokens.shape
        which = list(range(self.held.numel())) if which is None else which
        at = torch.tensor(which, device="cuda")
        tables, held = self.tables[at].contiguous(), self.held[at].contiguous()
        length, cu, slots, positions, state = B.odb_page_tables(held, ints(wanted), tables, self.free, self.n_free, self.page, self.n_pages,
                                                                row_first=ints(first), row_count=ints([b] * n), rows_cap=n * b)
        self.tables[at], self.held[at], self.n_free = tables, length, state[:1].clone()
        assert state[3].item() == 0
        return B.odb_step_paged(self.model, ints(tokens), self.k, self.v, tables, ints(first), length, positions, slots, self.table, **kw)

    def keys(self, r, layer, kv, length):
        """K (channels in the model's order) or V of a request, [length, heads, dim] float32."""
        pool = (self.k if kv == 0 else self.v)[layer]
        ids = self.tables[r, :-(-length // self.page)].long()
        x = pool[ids].permute(0, 2, 1, 3).reshape(-1, pool.shape[1], pool.shape[3])[:length].float().cpu().numpy()
        return x if kv else np.concatenate([x[..., 0::2], x[..., 1::2]], -1)


def decide(conf, argmax, conf_o, argmax_o, z_o):
    p = np.exp(z_o - z_o.max(-1, keepdims=True))
    p = np.sort(p / p.sum(-1, keepdims=True), -1)
    sure = p[..., -1] - p[..., -2] > MARGIN
    assert np.abs(np.log(conf) - np.log(conf_o)).max() <= LOG_CONF
    assert (argmax[sure] == argmax_o[sure]).all()


@pytest.mark.parametrize("gain", [None, 32.0])
def test_ragged_refresh_and_steps_equal_the_oracle(gain):
    shape = W.MODEL_SHAPES["tiny"]
    cfg = o.Config(**shape)
    w = o.Weights(cfg, W.WEIGHT_SEED, W.WEIGHT_STD)
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        if gain is not None:
            w.set_values(o.T_GF, 0, np.full(cfg.d_model, gain, np.float32))
            B.odb_model_set_tensor(model, B.T_GF, 0, w.bits(o.T_GF, 0))
        lens, prompts, blocks, b = [70, 33, 129], [40, 17, 100], [40, 17, 113], 16
        work = [W.decode_workload(shape, p, n - p, b, 1, 50 + i) for i, (p, n) in enumerate(zip(prompts, lens))]
        pg = Paged(shape, model, 3, 6, 32, 14)
        caches = []
        for r, wl in enumerate(work):                                # refreshes of one request each, all its positions
            conf, argmax, unmask = pg.forward(wl.tokens, [0], [lens[r]], which=[r], skip=prompts[r])
            cache, conf_o, argmax_o = o.prefill(cfg, w, wl.tokens[0], prompts[r])
            caches.append(cache)
            assert unmask is None and conf.shape == (1, lens[r] - prompts[r])
            assert np.abs(np.log(conf[0].cpu().numpy()) - np.log(conf_o)).max() <= LOG_CONF
        # the same K/V as the dense cache's
        for r, wl in enumerate(work):
            dense = B.odb_cache_create(model, 1, lens[r])
            conf_d, argmax_d = B.odb_prefill(model, dense, ints(wl.tokens), prompts[r])
            for layer in range(cfg.n_layers):
                for kv in (0, 1):
                    want = B.odb_cache_read(dense, layer, kv, 0, 0, lens[r], cfg.n_heads, cfg.head_dim)
                    assert np.abs(pg.keys(r, layer, kv, lens[r]) - want).max() <= KV_TOL * np.abs(want).max()
            B.odb_cache_destroy(dense)
        for turn in range(2):                                        # steps of all three, each at its own block; the second on other blocks
            offs = blocks if turn == 0 else [54, 1, 77]
            drafts = np.stack([wl.tokens[0, off:off + b] for wl, off in zip(work, offs)])
            conf, argmax, unmask = (t.cpu().numpy() for t in pg.forward(drafts, offs, lens, tau=0.9, max_len=129 if turn else 0))
            for r in range(3):
                # (a block's K/V in the pages are those of its last step: the oracle's cache gets them for the second turn's attention)
                if turn == 0:
                    c_o, a_o, u_o, z_o = o.block_step(cfg, w, caches[r], drafts[r][None], offs[r], 0.9, return_logits=True)
                    decide(conf[r], argmax[r], c_o[0], a_o[0], z_o[0])
                    near = np.abs(c_o[0] - 0.9) <= TAU_BAND
                    masked = drafts[r] == shape["mask_id"]
                    best = np.sort(c_o[0][masked])[-2:] if masked.sum() > 1 else np.array([0.0, 1.0])
                    if not near.any() and best[1] - best[0] > MARGIN:
                        assert (unmask[r] == u_o[0]).all()
                assert ((unmask[r] != 0) <= (drafts[r] == shape["mask_id"])).all()
                assert unmask[r].sum() >= min(1, (drafts[r] == shape["mask_id"]).sum())
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


@pytest.mark.parametrize("n,b", [(2, 32), (3, 7), (1, 1), (12, 16)])
def test_steps_equal_the_dense_ones_at_the_8b_width(n, b):
    shape = dict(W.MODEL_SHAPES["8b"], n_layers=2)
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        rng = np.random.default_rng(n * 100 + b)
        lens = [int(x) for x in rng.integers(b + 5, 200, n)]
        work = [W.decode_workload(shape, 4, length - 4, b, 1, 90 + r) for r, length in enumerate(lens)]
        offs = [int(rng.integers(0, length - b + 1)) for length in lens]
        pg = Paged(shape, model, n, 14, 16, n * 13 + 2)
        want = []
        for r, wl in enumerate(work):
            pg.forward(wl.tokens, [0], [lens[r]], which=[r], head=False)
            dense = B.odb_cache_create(model, 1, lens[r])
            B.odb_prefill(model, dense, ints(wl.tokens), 0)
            want.append([t.cpu().numpy()[0, 0] for t in B.odb_block_step(model, dense, ints(wl.tokens[:, None, offs[r]:offs[r] + b]), offs[r], 0.9)])
            B.odb_cache_destroy(dense)
        drafts = np.stack([wl.tokens[0, off:off + b] for wl, off in zip(work, offs)])
        conf, argmax, unmask = (t.cpu().numpy() for t in pg.forward(drafts, offs, lens, tau=0.9))
        for r in range(n):
            assert np.abs(np.log(conf[r]) - np.log(want[r][0])).max() <= LOG_CONF
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


def test_refusals_and_a_batch_with_padding():
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        wl = W.decode_workload(shape, 20, 44, 16, 1, 7)
        pg = Paged(shape, model, 2, 4, 16, 9)
        conf, argmax, _ = pg.forward(wl.tokens, [0], [64], which=[0], skip=20)
        # request 1 is empty: its rows are padding
        tokens = np.stack([wl.tokens[0, 20:36], np.zeros(16, np.int32)])
        alone = [t.clone() for t in pg.forward(tokens[:1], [20], [64], which=[0], tau=0.9)]
        tables, positions, slots = pg.tables, ints(np.r_[np.arange(20, 36), [-1] * 16]), ints([0] * 32)
        slots[:16] = (pg.tables[0, (positions[:16] // 16).long()] * 16 + positions[:16] % 16).int()
        slots[16:] = -1
        before = pg.k.clone()
        both = B.odb_step_paged(model, ints(tokens), pg.k, pg.v, tables, ints([20, 0]), ints([64, 0]), positions, slots, pg.table, tau=0.9)
        for x, y in zip(both, alone):
            assert torch.equal(x[:1], y)
        assert torch.equal(before.nan_to_num(7.0), pg.k.nan_to_num(7.0))
        args = dict(tokens=ints(tokens), k_pages=pg.k, v_pages=pg.v, tables=tables, first_pos=ints([20, 0]), kv_len=ints([64, 0]), positions=positions,
                    slots=slots, table=pg.table)
        for bad in (dict(k_pages=pg.k.bfloat16(), v_pages=pg.v.bfloat16()), dict(skip=3, tau=0.5), dict(max_len=-1),
                    dict(k_pages=pg.k[:, :, :2], v_pages=pg.v[:, :, :2])):
            with pytest.raises(B.OdbError):
                B.odb_step_paged(model, **dict(args, **bad))
        for bad in (dict(tokens=ints(tokens[:1])), dict(k_pages=pg.k[0], v_pages=pg.v[0]), dict(table=pg.table[:, :8]), dict(slots=slots[:16])):
            with pytest.raises(TypeError):
                B.odb_step_paged(model, **dict(args, **bad))
        with pytest.raises(ValueError):
            B.odb_step_paged(model, **dict(args, skip=16))
        assert B.lib().odb_step_paged(None, None, None, None) == -1
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)
