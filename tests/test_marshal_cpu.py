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
