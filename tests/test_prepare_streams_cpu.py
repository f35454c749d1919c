"""prepare.fp8_weight on another stream than the current one: which stream waits, and whose memory the
allocator is told of.  Stand-ins for the streams and the library's calls; nothing touches a GPU."""
import pytest

import paper_2509_18344_amd as ss  # noqa: F401
from paper_2509_18344_amd import _binding, prepare

torch = pytest.importorskip("torch")
N, K = 32, 640


class Stream:
    log = None

    def __init__(self, name, handle):
        self.name, self.cuda_stream = name, handle

    def wait_stream(self, other):
        self.log.append(("wait", self.name, other.name))


class External(Stream):
    def __init__(self, handle, device=None):
        # torch takes the handle 0 for none at all and hands out a stream of its pool
        super().__init__("of %d" % handle, handle or 999)


@pytest.fixture
def made(monkeypatch):
    """What fp8_weight does, in order: waits, calls with their stream and addresses, records."""
    log = []
    monkeypatch.setattr(Stream, "log", log)
    monkeypatch.setattr(torch.cuda, "ExternalStream", External)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream("current", 111))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Stream("default", 0))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: log.append(("record", s.name, t.data_ptr())))
    monkeypatch.setattr(_binding, "subspec_fp8_rows", lambda w, n, k, codes, scales, stream=None: log.append(
        ("rows", stream, w.data_ptr(), codes.data_ptr(), scales.data_ptr())))
    monkeypatch.setattr(_binding, "subspec_fp8_pack", lambda codes, n, k, tiles, stream=None: log.append(
        ("pack", stream, codes.data_ptr(), tiles.data_ptr())))
    return log


def _calls(log, w, p, stream):
    rows, pack = [e for e in log if e[0] in ("rows", "pack")]
    assert rows[:2] == ("rows", stream) and pack[:2] == ("pack", stream) and pack[2] == rows[3]
    used = {*rows[2:], *pack[2:]}
    assert used == {w.data_ptr(), rows[3], p["w_scales"].data_ptr(), p["w"].data_ptr()}
    return used


@pytest.mark.parametrize("given,name", [(Stream("side", 555), "side"), (0, "default")])
def test_a_stream_of_torchs_waits_and_holds_every_tensor(made, given, name):
    w = torch.zeros((N, K), dtype=torch.bfloat16)
    p = prepare.fp8_weight(w, given)
    used = _calls(made, w, p, given)
    assert [e for e in made if e[0] == "wait"] == [("wait", name, "current")] and made[0][0] == "wait"
    assert {e[1:] for e in made if e[0] == "record"} == {(name, a) for a in used}


@pytest.mark.parametrize("given", [777, External(777)])
def test_the_current_stream_waits_for_a_stream_that_may_end_before_the_tensors(made, given):
    w = torch.zeros((N, K), dtype=torch.bfloat16)
    p = prepare.fp8_weight(w, given)
    _calls(made, w, p, given)
    assert made[0] == ("wait", "of 777", "current") and made[-1] == ("wait", "current", "of 777") and len(made) == 4


def test_on_the_current_stream_nothing_waits(made):
    w = torch.zeros((N, K), dtype=torch.bfloat16)
    p = prepare.fp8_weight(w)
    _calls(made, w, p, None)
    assert len(made) == 2


@pytest.mark.parametrize("given", [Stream("side", 555), 777])
def test_a_refusal_between_the_two_calls_leaves_the_first_ones_memory_safe(made, monkeypatch, given):
    def refuse(*args):
        raise _binding.SubspecError("subspec_fp8_pack", -2, "N")

    monkeypatch.setattr(_binding, "subspec_fp8_pack", refuse)
    w = torch.zeros((N, K), dtype=torch.bfloat16)
    with pytest.raises(_binding.SubspecError):
        prepare.fp8_weight(w, given)
    rows = next(e for e in made if e[0] == "rows")
    if given == 777:
        assert made[-1] == ("wait", "current", "of 777")
    else:
        assert set(rows[2:]) <= {e[2] for e in made if e[0] == "record"}
