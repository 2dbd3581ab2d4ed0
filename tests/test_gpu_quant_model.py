"""The model's forward over pages of 8-bit codes (odb_step_paged_quant).  What it attends to are the values that the pages then hold, so it has to
equal odb_step_paged over pages of 16 bits that hold the same values and are not written; what it stores is checked against the keys and
values that odb_step_paged stores.  The bar is that of the dense calls: logarithms of confidences within 5e-2."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import quant_plain as quant                                          # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402
from paper_2511_21759_amd import workloads as W                      # noqa: E402

pytestmark = pytest.mark.gpu
LOG_CONF = 5e-2
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Pages:
    """Pools in 8 bits, and in 16, of some requests over one model, with the same tables."""

    def __init__(self, shape, model, kind, group, lens, page):
        self.shape, self.model, self.kind, self.group, self.page, self.lens = shape, model, kind, group, page, lens
        n_layers, heads, dim = shape["n_layers"], shape["n_heads"], shape["head_dim"]
        need = [-(-length // page) for length in lens]
        self.n_pages, ids, at = sum(need) + 2, np.random.default_rng(2).permutation(sum(need) + 2), 0
        self.tables = np.full((len(lens), max(need) + 1), -1, np.int32)
        for r, count in enumerate(need):
            self.tables[r, :count], at = ids[at:at + count], at + count
        size = (n_layers, self.n_pages, heads, page, dim)
        self.codes = [torch.full(size, 0x7f, dtype=torch.int8, device="cuda").view(CODES[kind]) for _ in range(2)]
        self.scales = [torch.full((*size[:3], page // group), float("nan"), device="cuda") for _ in range(2)]
        self.k16, self.v16 = (torch.zeros(size, dtype=torch.float16, device="cuda") for _ in range(2))
        self.table = B.odb_rope_table(1024, dim, shape["rope_base"])

    def positions(self, first, b):
        return [f + i for f in first for i in range(b)]

    def slots(self, first, b, which):
        return [self.tables[r, p // self.page] * self.page + p % self.page for r, f in zip(which, first) for p in range(f, f + b)]

    def step(self, tokens, first, which, **kw):
        lens = [self.lens[r] for r in which]
        return B.odb_step_paged_quant(self.model, ints(tokens), *self.codes, *self.scales, ints(self.tables[which]), ints(first), ints(lens),
                                      ints(self.positions(first, tokens.shape[1])), self.table, **kw)

    def step16(self, tokens, first, which, store=True, **kw):
        lens, b = [self.lens[r] for r in which], tokens.shape[1]
        slots = self.slots(first, b, which) if store else [-1] * (len(which) * b)
        return B.odb_step_paged(self.model, ints(tokens), self.k16, self.v16, ints(self.tables[which]), ints(first), ints(lens),
                                ints(self.positions(first, b)), ints(slots), self.table, **kw)

    def take_values(self):
        """The 16-bit pools get what the codes are."""
        slots = torch.arange(self.n_pages * self.page, dtype=torch.int32, device="cuda")
        for layer in range(self.shape["n_layers"]):
            k, v = B.odb_paged_read_quant(*(t[layer] for t in self.codes), *(t[layer] for t in self.scales), slots)
            for pool, x in ((self.k16, k), (self.v16, v)):
                pool[layer] = x.view(self.n_pages, self.page, *x.shape[1:]).transpose(1, 2).nan_to_num(0.0)


@pytest.mark.parametrize("kind,group,page", [("int8", 32, 32), ("e4m3", 16, 16), ("int8", 1, 16), ("e4m3", 64, 64)])
def test_refreshes_and_steps(kind, group, page):
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        lens, blocks, b = [70, 33, 129], [40, 17, 113], 16
        work = [W.decode_workload(shape, 10, n - 10, b, 1, 50 + i) for i, n in enumerate(lens)]
        pg = Pages(shape, model, kind, group, lens, page)
        for r, wl in enumerate(work):
            before = [t[0].cpu().clone() for t in pg.codes + pg.scales]
            conf, argmax, unmask = pg.step(wl.tokens, [0], [r], skip=4)
            assert unmask is None and conf.shape == (1, lens[r] - 4)
            # layer 0: the same keys and values as the 16-bit pages', which have rounded them by 2^-11 (2^-25 where they are tiny)
            pg.step16(wl.tokens, [0], [r], head=False)
            rows, live = [lens[r]], torch.ones(lens[r], dtype=torch.bool)
            at = torch.tensor(pg.slots([0], lens[r], [r]), dtype=torch.long)
            for i, pool in ((0, pg.k16), (1, pg.v16)):
                x = pool[0].cpu()[at // page, :, at % page].double()
                quant.check_store(kind, group, (before[i], before[2 + i]), (pg.codes[i][0].cpu(), pg.scales[i][0].cpu()), x, x.abs() * 2.0 ** -11 + 2.0 ** -25,
                                  rows, [0], rows, pg.tables[r:r + 1], live, "kv"[i])
            pg.take_values()
            conf16, argmax16, _ = pg.step16(wl.tokens, [0], [r], store=False, skip=4)
            assert (conf.log() - conf16.log()).abs().max() <= LOG_CONF
        drafts = np.stack([wl.tokens[0, off:off + b] for wl, off in zip(work, blocks)])
        conf, argmax, unmask = pg.step(drafts, blocks, [0, 1, 2], tau=0.9, max_len=129)
        pg.take_values()
        conf16, argmax16, unmask16 = pg.step16(drafts, blocks, [0, 1, 2], store=False, tau=0.9)
        assert (conf.log() - conf16.log()).abs().max() <= LOG_CONF
        assert unmask.shape == (3, b) and ((unmask != 0) <= (ints(drafts) == shape["mask_id"])).all()
        again = pg.step(drafts, blocks, [0, 1, 2], tau=0.9, max_len=129)              # the same values are stored again
        assert torch.equal(conf, again[0]) and torch.equal(argmax, again[1])
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


@pytest.mark.parametrize("n,b", [(2, 32), (3, 7), (1, 1), (12, 16)])
def test_steps_at_the_8b_width(n, b):
    shape = dict(W.MODEL_SHAPES["8b"], n_layers=2)
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        rng = np.random.default_rng(n * 100 + b)
        lens = [int(x) for x in rng.integers(b + 5, 200, n)]
        work = [W.decode_workload(shape, 4, length - 4, b, 1, 90 + r) for r, length in enumerate(lens)]
        offs = [int(rng.integers(0, length - b + 1)) for length in lens]
        pg = Pages(shape, model, "int8", 16, lens, 16)
        for r, wl in enumerate(work):
            pg.step(wl.tokens, [0], [r], head=False)
        drafts = np.stack([wl.tokens[0, off:off + b] for wl, off in zip(work, offs)])
        conf, argmax, unmask = pg.step(drafts, offs, list(range(n)), tau=0.9)
        pg.take_values()
        conf16, argmax16, unmask16 = pg.step16(drafts, offs, list(range(n)), store=False, tau=0.9)
        assert (conf.log() - conf16.log()).abs().max() <= LOG_CONF
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)


def test_refusals_and_a_batch_with_padding():
    shape = W.MODEL_SHAPES["tiny"]
    model = B.odb_model_create(shape)
    try:
        B.odb_model_init_random(model, W.WEIGHT_SEED, W.WEIGHT_STD)
        wl = W.decode_workload(shape, 20, 44, 16, 1, 7)
        pg = Pages(shape, model, "int8", 16, [64, 40], 16)
        pg.step(wl.tokens, [0], [0], head=False)
        tokens = np.stack([wl.tokens[0, 20:36], np.zeros(16, np.int32)])
        alone = [t.clone() for t in pg.step(tokens[:1], [20], [0], tau=0.9)]
        before = [t.view(torch.int8 if t.dtype != torch.float32 else torch.float32).clone() for t in pg.codes + pg.scales]
        args = dict(tokens=ints(tokens), k_pages=pg.codes[0], v_pages=pg.codes[1], k_scale=pg.scales[0], v_scale=pg.scales[1], tables=ints(pg.tables),
                    first_pos=ints([20, 0]), kv_len=ints([64, 0]), positions=ints(np.r_[np.arange(20, 36), [-1] * 16]), table=pg.table)
        both = B.odb_step_paged_quant(model, **args, tau=0.9)                     # request 1 is empty: its rows are padding
        for x, y in zip(both, alone):
            assert torch.equal(x[:1], y)
        for x, y in zip(before, pg.codes + pg.scales):
            assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))
        half = dict(k_pages=pg.codes[0][:, :, :2], v_pages=pg.codes[1][:, :, :2], k_scale=pg.scales[0][:, :, :2], v_scale=pg.scales[1][:, :, :2])
        odd = [torch.zeros(t.shape[0], t.shape[1] * t.shape[2] * t.shape[3] + 1, device="cuda")[:, :-1].unflatten(1, t.shape[1:]) for t in pg.scales]
        for bad in (half, dict(skip=3, tau=0.5), dict(max_len=-1), dict(k_scale=odd[0], v_scale=odd[1]),
                    dict(k_pages=pg.codes[0][:1], v_pages=pg.codes[1][:1], k_scale=pg.scales[0][:1], v_scale=pg.scales[1][:1])):
            with pytest.raises(B.OdbError):
                B.odb_step_paged_quant(model, **dict(args, **bad))
        for bad in (dict(tokens=ints(tokens[:1])), dict(k_pages=pg.codes[0][0], v_pages=pg.codes[1][0]), dict(table=pg.table[:, :8]),
                    dict(k_scale=pg.scales[0][0], v_scale=pg.scales[1][0]), dict(k_pages=pg.codes[0].float(), v_pages=pg.codes[1].float())):
            with pytest.raises(TypeError):
                B.odb_step_paged_quant(model, **dict(args, **bad))
        with pytest.raises(ValueError):
            B.odb_step_paged_quant(model, **dict(args, skip=16))
        assert B.lib().odb_step_paged_quant(None, None, None, 0, None) == -1
        B.odb_model_status(model)
    finally:
        B.odb_model_destroy(model)
