"""Host-only: which workspace a call of RolloutStage gets.  What a recorded call is given must not be what other calls on the stream use or replace: its graph keeps the
address and is replayed at any time, on any stream."""
import pytest
import torch

from paper_2603_06619_amd import binding, rollout


@pytest.fixture
def streams(monkeypatch):
    """The current stream and whether it is being recorded, as the test sets them."""
    now = dict(stream=1, recording=False)
    monkeypatch.setattr(binding, "_stream", lambda: now["stream"])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: now["recording"])
    return now


def test_one_per_stream_that_grows(streams):
    stage = rollout.RolloutStage("cpu")
    a = stage._buf("x", 1000)
    assert stage._buf("x", 1000) is a and stage._buf("x", 10) is a and stage._buf("y", 10) is not a and stage._buf("x", 0) is None
    streams["stream"] = 2
    b = stage._buf("x", 500)
    assert b is not a and b.numel() >= 500
    streams["stream"] = 1
    c = stage._buf("x", 3000)
    assert c.numel() >= 3000 and stage._buf("x", 1000) is c


def test_a_recorded_call_has_its_own(streams):
    stage = rollout.RolloutStage("cpu")
    kept = stage._buf("x", 1000)
    streams["recording"] = True
    first, second = stage._buf("x", 1000), stage._buf("x", 800)
    assert len({t.data_ptr() for t in (kept, first, second)}) == 3 and first.numel() >= 1000 and second.numel() >= 800
    assert stage._buf("z", 100) is not None and stage._buf("x", 0) is None
    streams["recording"] = False
    assert stage._buf("x", 1000) is kept                           # calls beside the replays go on with theirs
    new = stage._buf("z", 100)
    assert stage._buf("z", 100) is new and stage._buf("x", 5000) is not kept
    held = [t for t in stage._ws.values() if t is first or t is second]
    assert not held


def test_a_recorded_loss_call_has_its_own(streams):
    from paper_2603_06619_amd.stage import LossStage
    stage = LossStage.__new__(LossStage)                            # without the pinned words, which need a GPU
    stage.device, stage._ws = torch.device("cpu"), {}
    kept = stage._buf("loss", 1000)
    assert stage._buf("loss", 700) is kept
    streams["recording"] = True
    first, second = stage._buf("loss", 1000), stage._buf("loss", 2000)
    assert len({t.data_ptr() for t in (kept, first, second)}) == 3 and first.numel() >= 1000 and second.numel() >= 2000
    streams["recording"] = False
    assert stage._buf("loss", 1000) is kept
