"""The packed calls of 8-bit pages from two threads at once, each with a stream and pages of its own: they run without the interpreter's lock."""
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2511_21759_amd import binding as B                        # noqa: E402
from test_gpu_quant_calls import ints, long_call                     # noqa: E402

pytestmark = pytest.mark.gpu


def chain(a, qkv, table, positions):
    """Store, attend, read back, and a call that is refused."""
    pools = [a[x].clone() for x in ("k_pages", "v_pages", "k_scale", "v_scale")]
    heads, kv = a["q"].shape[1], pools[0].shape[1]
    q = B.odb_qk_norm_rope_quant(qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], *pools, table, positions, a["tables"], a["kv_len"], cu_rows=a["cu_rows"])
    out = B.odb_paged_attention_quant(q, *pools, a["tables"], a["kv_len"], causal=True, cu_rows=a["cu_rows"], max_rows=a["max_rows"])
    try:
        B.odb_paged_attention_quant(q, *pools, a["tables"], a["kv_len"], causal=True, cu_rows=a["cu_rows"], window=-a["max_rows"])
        said = None
    except B.OdbError as e:
        said = str(e)
    return [q, out, *pools, *B.odb_paged_read_quant(*pools, ints(np.arange(70)))], said


@pytest.mark.parametrize("rows,lens", [([1, 1], [4000, 3000]), ([300, 200], [4100, 700])])
def test_two_threads(rows, lens):
    sets = []
    for i in range(2):
        at = [m + i for m in rows]
        a = long_call(41 + i, at, lens, *((8, 2) if rows[0] == 1 else (16, 16)))
        a["cu_rows"] = ints(np.r_[0, np.cumsum(at)])
        qkv = torch.randn(sum(at), a["q"].shape[1] + 2 * a["k_pages"].shape[1], 128, device="cuda").half()
        positions = torch.cat([torch.arange(n - m, n, dtype=torch.int32) for m, n in zip(at, lens)]).cuda()
        sets.append((a, qkv, B.odb_rope_table(5000, 128, 10000.0), positions))
    alone = [chain(*s) for s in sets]
    torch.cuda.synchronize()
    got, wrong = [[], []], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i].append(chain(*sets[i]))
        except Exception as e:                                       # noqa: BLE001
            wrong.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
    for i in range(2):
        assert len(got[i]) == 20 and "window=-%d" % sets[i][0]["max_rows"] in alone[i][1]
        for outs, said in got[i]:
            assert said == alone[i][1]                               # (each thread's own message)
            for x, y in zip(outs, alone[i][0]):
                assert torch.equal(x, y)
