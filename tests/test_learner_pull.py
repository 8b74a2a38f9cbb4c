"""What learner.pull_mx4 asks of the server, with a server that only records it: no GPU needed."""
import pytest
import torch

from paper_1509_04210_b200 import binding as rb
from paper_1509_04210_b200 import learner


class Codes:
    """In the place of an MX4 matrix."""

    def __init__(self, rows, cols, device):
        self.rows, self.cols, self.device = rows, cols, device
        self.codes_ptr, self.scales_ptr = 4096, 8192


class Server:
    def __init__(self, device):
        self.device, self.calls = device, []

    def pull_mx4_on(self, *args):
        self.calls.append(args)
        return 17


@pytest.fixture
def parts(monkeypatch):
    """Devices 0 (current) and 3, each with a current stream of its own."""
    made = []

    def empty(kind, rows, cols, device):
        assert kind == 0
        made.append(Codes(rows, cols, device))
        return made[-1]

    monkeypatch.setattr(learner, "MX4", Codes)
    monkeypatch.setattr(learner._n, "empty", empty)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(learner._n, "current_stream", lambda device: 1000 + device)
    return made


@pytest.mark.parametrize("transpose", [False, True])
def test_the_buffer_lies_on_the_servers_device_and_the_work_between_that_of_torchs_stream(parts, transpose):
    ps = Server(3)
    q, ts = learner.pull_mx4(ps, 7, 5, 40, transpose=transpose)
    assert ts == 17 and parts == [q]
    assert (q.rows, q.cols, q.device) == ((40, 5, 3) if transpose else (5, 40, 3))
    assert ps.calls == [(7, 5, 40, transpose, 4096, 8192, 1003)]


def test_a_buffer_on_another_device_is_refused(parts):
    ps = Server(3)
    for bad in (Codes(5, 40, 0), Codes(40, 5, 3), object()):
        with pytest.raises(ValueError):
            learner.pull_mx4(ps, 7, 5, 40, out=bad)
    assert ps.calls == []
    good = Codes(5, 40, 3)
    assert learner.pull_mx4(ps, 7, 5, 40, out=good) == (good, 17) and parts == []


def test_the_entry_points_refuse_what_is_no_handle():
    L = rb.lib()
    assert L.rudra_ps_device(None) == rb.E_INVAL
    assert L.rudra_ps_pull_mx4_on(None, 0, 1, 1, 0, 4096, 4096, None) == rb.E_INVAL and "handle" in rb.last_error()
