"""The packed calls of 8-bit pages (_marshal) on the host: tensors of the CPU, and entry points of the test's own."""
import sys

import pytest

torch = pytest.importorskip("torch")

import paper_2511_21759_amd as package                               # noqa: E402
from paper_2511_21759_amd import binding as B                        # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    try:
        from paper_2511_21759_amd import _marshal                    # noqa: F401
        B.lib()
    except (ImportError, B.OdbError):
        from paper_2511_21759_amd.build import build_library
        build_library()


def test_a_missing_module_stops_the_packed_calls_alone_and_every_time(monkeypatch):
    """... with an error that says what to build; the library opens without it."""
    monkeypatch.delattr(package, "_marshal", raising=False)
    monkeypatch.setitem(sys.modules, package.__name__ + "._marshal", None)          # (an import of it fails)
    monkeypatch.setattr(B, "_lib", None)
    B._load_torch()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for _ in range(2):
        assert B.lib().odb_paged_attention_quant_workspace(None, None) == -1
        with pytest.raises(B.OdbError, match="_marshal.*build"):
            B._here(0)
        assert B._here(1) is None                                    # another device is left to the binding's own path


def test_the_packed_calls_belong_to_the_library_that_is_open(monkeypatch):
    B._load_torch()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_stream", lambda: 5)
    monkeypatch.setattr(B, "_raw_stream", None)
    assert B._here(0) == 5
    first = B._calls
    assert B._here(0) == 5 and B._calls is first and first[0] is B.lib()
    monkeypatch.setattr(B, "_lib", None)                             # (as a new build does)
    assert B._here(0) == 5 and B._calls[0] is B.lib() and B._calls[0] is not first[0]


# ---- the calls themselves: entry points of the test's own take the place of the library's --------------------------------

STUB = r"""
#include <unistd.h>
static volatile int flag, entered;
static int wait(void) {                      /* until another thread has set the flag, 20 s at most */
    entered = 1;
    for (int i = 0; i < 20000 && !flag; i++) usleep(1000);
    return flag ? 0 : -1;
}
int store(const void *r, const void *p, void *s) { return wait(); }
int attend(const void *r, const void *p, void *s) { return wait(); }
int read_back(const void *p, const void *at, int n, int type, void *k, void *v, long long kr, long long vr, void *s) { return wait(); }
long long room(const void *r, const void *p) { return 0; }
void set(int x) { flag = x; entered = 0; }
int inside(void) { return entered; }
"""


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    import ctypes
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    at = tmp_path_factory.mktemp("stub")
    (at / "stub.c").write_text(STUB)
    subprocess.run([cc, "-O1", "-shared", "-fPIC", str(at / "stub.c"), "-o", str(at / "stub.so")], check=True)
    return ctypes.CDLL(str(at / "stub.so"))


class Call:
    """Arguments of the three calls, three rows of two requests on the CPU (device -1)."""

    def __init__(self, stub):
        import ctypes
        at = lambda f: ctypes.cast(f, ctypes.c_void_p).value         # noqa: E731
        i32 = torch.int32
        self.pools = [torch.zeros(5, 2, 32, 64, dtype=torch.int8) for _ in range(2)] + [torch.zeros(5, 2, 2) for _ in range(2)]
        self.q = torch.zeros(3, 4, 64, dtype=torch.float16)
        self.requests = [torch.zeros(2, 4, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(3, dtype=i32), None]
        self.rope = [torch.zeros(9, 32, 2), torch.zeros(3, dtype=i32)]
        self.at = {name: at(getattr(stub, name)) for name in ("store", "attend", "read_back", "room")}

    def store(self, interleaved=False):
        from paper_2511_21759_amd import _marshal
        return _marshal.store(self.at["store"], 0, -1, self.q, self.q[:, :2], self.q[:, 2:], *self.pools, *self.rope, *self.requests, None, None, 1e-6, interleaved, False,
                              None, None)

    def attend(self, causal=True):
        from paper_2511_21759_amd import _marshal
        return _marshal.attention(self.at["attend"], self.at["room"], 0, -1, self.q, *self.pools, *self.requests, 0.125, causal, 0, 0, 0, 0, None, None)

    def read(self):
        from paper_2511_21759_amd import _marshal
        return _marshal.read(self.at["read_back"], 0, -1, *self.pools, torch.zeros(3, dtype=torch.int32), 0)


@pytest.mark.parametrize("name", ["store", "attend", "read"])
def test_other_threads_run_while_an_entry_point_waits(stub, name):
    """A launch can wait for room in a queue: a second thread of Python has to go on meanwhile (it is what ends the wait here)."""
    import threading
    import time
    stub.set(0)

    def second():
        while not stub.inside():
            time.sleep(0.001)
        stub.set(1)
    thread = threading.Thread(target=second)
    thread.start()
    got = getattr(Call(stub), name)()
    thread.join()
    assert not isinstance(got, int), "the entry point waited in vain"
    shapes = [tuple(t.shape) for t in (got if isinstance(got, tuple) else (got,))]
    assert shapes == {"store": [(3, 4, 64)], "attend": [(3, 4, 64)], "read": [(3, 2, 64)] * 2}[name]


def test_what_has_no_truth_value_is_left_to_the_bindings_own_path(stub):
    """... which names the error: no call is made, and no exception is left behind."""
    call, none = Call(stub), torch.zeros(2)
    for name in ("store", "attend"):
        stub.set(1)
        assert getattr(call, name)(none) is None and not stub.inside()
        assert getattr(call, name)(torch.ones(1)) is not None and stub.inside()


@pytest.mark.gpu
def test_what_has_no_truth_value_is_refused():
    i32, none = torch.int32, torch.zeros(2)
    pools = [torch.zeros(5, 2, 32, 64, dtype=torch.int8, device="cuda") for _ in range(2)] + [torch.zeros(5, 2, 2, device="cuda") for _ in range(2)]
    q = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda")
    requests = torch.zeros(2, 4, dtype=i32, device="cuda"), torch.ones(2, dtype=i32, device="cuda")
    with pytest.raises(RuntimeError, match="ambiguous"):
        B.odb_paged_attention_quant(q, *pools, *requests, causal=none)
    with pytest.raises(RuntimeError, match="ambiguous"):
        B.odb_qk_norm_rope_quant(q, q[:, :2], q[:, 2:], *pools, B.odb_rope_table(64, 64, 10000.0), torch.zeros(2, dtype=i32, device="cuda"), *requests, interleaved=none)
