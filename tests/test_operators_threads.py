"""One context, several threads (CPU: a library that notes who is in it).  A
context takes one call at a time and holds one error message, and automatic
differentiation calls from threads of its own."""

import threading
import time

import pytest

torch = pytest.importorskip("torch")

from paper_2606_07019_amd import operators   # noqa: E402
from paper_2606_07019_amd import pccl as P   # noqa: E402


class Library:
    """Calls that take a while, fail for some shapes, and leave their message in the context."""

    def __init__(self):
        self.inside, self.most, self.message = 0, 0, b""

    def enter(self):
        self.inside += 1
        self.most = max(self.most, self.inside)
        time.sleep(0.002)

    def pccl_mx_quantize(self, h, x, dtype, rows, cols, *rest):
        self.enter()
        status = 1 if rows % 2 else 0
        self.message = b"%d rows" % rows if status else b""
        time.sleep(0.002)
        self.inside -= 1
        return status

    def pccl_last_error(self, h):
        time.sleep(0.002)
        return self.message


@pytest.fixture
def ops(monkeypatch):
    lib = Library()

    class Guard:
        def __init__(self, device):
            pass

        def __enter__(self):
            pass

        def __exit__(self, *exc):
            pass

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(P, "load_library", lambda: lib)
    monkeypatch.setattr(P, "pccl_create", lambda device, seed: 7)
    monkeypatch.setattr(P, "pccl_destroy", lambda h: None)

    def ask(h, *sizes):
        lib.enter()
        lib.inside -= 1
        return 0

    monkeypatch.setattr(P, "pccl_mx_matmul_workspace", ask)
    monkeypatch.setattr(operators.Operators, "_stream", lambda self: None)
    o = operators.Operators(0)
    o.device = torch.device("cpu")
    o.lib = lib
    yield o
    o.close()


def test_calls_of_several_threads_take_turns_and_keep_their_messages(ops):
    wrong = []

    def work(rows):
        for i in range(6):
            try:
                ops.quantize(torch.ones(rows, 4))
                said = None
            except P.PcclError as e:
                said = str(e)
            if said != (f"PCCL_EINVAL: {rows} rows" if rows % 2 else None):
                wrong.append((rows, said))
            ops._space(P.pccl_mx_matmul_workspace, rows, i, 4)

    threads = [threading.Thread(target=work, args=(rows,)) for rows in range(1, 9)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert ops.lib.most == 1 and not wrong


def test_a_closed_context_is_not_used(ops):
    ops.close()
    ops.lib.pccl_mx_quantize = lambda h, *rest: (_ for _ in ()).throw(AssertionError(h)) if h is not None else 1
    ops.lib.pccl_last_error = lambda h: b"null context"
    with pytest.raises(P.PcclError, match="null context"):
        ops.quantize(torch.ones(2, 4))
