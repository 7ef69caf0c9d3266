"""Which stream owns the memory that MxLinear and quantise_layer allocate (no GPU: the library's calls are recorded)."""
import contextlib
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2607_23099_amd import build, damoe, moe, synth


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(damoe.LIB_PATH):
        build.build_damoe()


class Side:
    """Stands for a stream other than the current one."""


@pytest.fixture
def record(monkeypatch):
    """What was allocated under which stream, which calls were made on which, and what was waited for."""
    r = {"current": None, "made": {}, "calls": [], "waited": 0}

    @contextlib.contextmanager
    def stream(s):
        before, r["current"] = r["current"], s
        yield
        r["current"] = before

    real = torch.empty

    def empty(*args, **kw):
        t = real(*args, **kw)
        r["made"][t.data_ptr()] = r["current"]
        return t

    class Current:
        def synchronize(self):
            r["waited"] += 1

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Current())
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
    monkeypatch.setattr(damoe, "mxfp4_linear",
                        lambda x, T, K, w, N, y, ws, add=None, stream=None: r["calls"].append((y, stream)))
    monkeypatch.setattr(damoe, "mxfp4_quantise", lambda x, rows, cols, codes, scales=None, layout=2, ldx=None, stream=None:
                        r["calls"].append((codes, stream)))
    monkeypatch.setattr(damoe, "mxfp4_bytes", lambda rows, cols, layout=2: rows * cols)
    monkeypatch.setattr(damoe, "mxfp4_linear_workspace_size", lambda T, N, K: 256)
    return r


@pytest.mark.parametrize("stream", [None, Side(), 0x1234], ids=["current", "stream", "handle"])
def test_results_belong_to_the_stream_of_the_call(record, stream):
    lin = moe.MxLinear(torch.zeros(64, 32), 8)
    del record["calls"][:]
    for x, add in [(torch.zeros(8, 32), None), (torch.zeros(3, 32), torch.zeros(3, 64))]:
        y = lin(x, add=add, stream=stream)
        made, used = record["calls"][-1]
        assert made is y and used is stream and record["made"][y.data_ptr()] is stream
    y = torch.zeros(8, 64)
    assert lin(torch.zeros(8, 32), y, stream=stream) is y


@pytest.mark.parametrize("stream", [None, Side(), 0x1234], ids=["current", "stream", "handle"])
def test_packed_weights_belong_to_the_stream_of_the_call(record, stream):
    sh = synth.Shape("streams", E=2, k=1, H=128, I=128, shape_id=9, wdtype="mxfp4")
    w = {n: torch.zeros((sh.E,) + tuple(synth.weight_dims(sh, n)[1:])) for n in ("w1", "w3", "w2")}
    dl = moe.quantise_layer(sh, **w, stream=stream)
    assert len(record["calls"]) == 3
    for made, used in record["calls"]:
        assert used is stream and record["made"][made.data_ptr()] is stream
    assert {t.data_ptr() for t in dl.w.values()} == {t.data_ptr() for t, _ in record["calls"]}


def test_weights_are_ready_for_every_stream(record):
    """A first call may come on any stream: the constructor ends when the tiles are there."""
    moe.MxLinear(torch.zeros(64, 32), 8)
    assert len(record["calls"]) == 1 and record["waited"] == 1


def test_inputs_that_ask_for_a_gradient(record):
    """It would be lost without a word."""
    lin = moe.MxLinear(torch.zeros(64, 32, requires_grad=True), 8)  # a trained layer's weights are no input
    x, add = torch.zeros(8, 32), torch.zeros(8, 64)
    for kw in (dict(x=x.clone().requires_grad_()), dict(x=x, add=add.clone().requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            lin(**kw)
        with torch.no_grad():
            assert not lin(**kw).requires_grad
        lin(**{n: t.detach() for n, t in kw.items()})


def _path(T_max=8, E=64):
    path = moe.Path.__new__(moe.Path)
    path.dl = type("Layer", (), {"shape": synth.Shape("streams", E=E, k=4, H=128, I=128, shape_id=9)})
    path.T_max, path.loss_S, path.logits = T_max, 0, torch.zeros(T_max, E)
    return path


def test_loss_buffers_are_ready_for_every_stream(record):
    """Clearing them late would wipe the results of a first call on another stream."""
    path = _path()
    path.prepare_loss(S=3)
    assert record["waited"] == 1 and path.loss_S == 3
    assert path.loss_counts.shape == (3, 64) and path.loss_tokens.shape == (5,)


@pytest.mark.parametrize("S", [0, -1, (1 << 20) + 1])
def test_loss_of_a_number_of_sequences_that_the_library_does_not_take(record, S):
    path = _path()
    with pytest.raises(ValueError, match="sequences"):
        path.prepare_loss(S)
    assert path.loss_S == 0
