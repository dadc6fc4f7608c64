"""What the feed-forward operators' Python side does by itself; no GPU needed."""
import threading
import time

import pytest
import torch

from paper_2607_11136_b200 import feedforward as ff


def test_check_without_an_index_looks_at_the_current_device(monkeypatch):
    """"cuda" names the current device, as everywhere in torch, not device 0."""
    waited = []
    monkeypatch.setattr(ff, "_current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: waited.append(device))
    word = torch.tensor([0], dtype=torch.int32)
    monkeypatch.setattr(ff, "_status", {3: (word, 0)})
    ff.check()
    ff.check("cuda")
    ff.check(torch.device("cuda"))
    ff.check("cuda:0")
    ff.check(0)
    ff.check(3)
    assert waited == [3, 3, 3, 0, 0, 3]
    word[0] = 0x54310002
    ff.check("cuda:0")
    with pytest.raises(Exception, match="adapter"):
        ff.check("cuda")
    assert word.item() == 0


class _OnDevice0(torch.Tensor):
    def get_device(self):
        return 0


@pytest.fixture
def no_device(monkeypatch):
    """What making a status word calls of torch, on the CPU and slowly; the words that were made."""
    made, zeros = [], torch.zeros

    def slow_zeros(*size, **kw):
        time.sleep(0.05)
        kw.pop("device")
        made.append(zeros(*size, **kw))
        return made[-1]

    monkeypatch.setattr(ff, "_status", {})
    monkeypatch.setattr(torch, "zeros", slow_zeros)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: type("Stream", (), {"synchronize": lambda self: None})())
    return made


def test_threads_get_the_same_status_word(no_device):
    """One word a device: of two, one would be freed while kernels hold its address."""
    t = torch.empty(1).as_subclass(_OnDevice0)
    got = []
    threads = [threading.Thread(target=lambda: got.append(ff._status_of(t))) for _ in range(8)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert len(no_device) == 1 and got == [no_device[0].data_ptr()] * 8


def test_a_status_word_is_zero_before_its_address_is_given_out(no_device, monkeypatch):
    """Kernels on other streams than the one that fills it would write into memory that is filled later."""
    seen = []
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda device=None: type("Stream", (), {"synchronize": lambda self: seen.append((device, len(no_device), dict(ff._status)))})())
    ff._status_of(torch.empty(1).as_subclass(_OnDevice0))
    assert seen == [(0, 1, {})]


def test_a_status_word_made_in_inference_mode_can_be_cleared_outside(no_device, monkeypatch):
    with torch.inference_mode():
        ff._status_of(torch.empty(1).as_subclass(_OnDevice0))
    no_device[0][0] = 0x54310002
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    with pytest.raises(Exception, match="adapter"):
        ff.check(0)
    ff.check(0)


def test_the_torch_module_is_rebuilt_for_another_torch(monkeypatch, tmp_path):
    """Sources that did not change are no reason to keep a module that was built against another torch or Python."""
    from paper_2607_11136_b200 import build as b
    commands = []
    monkeypatch.setattr(b, "OBJ", str(tmp_path))
    monkeypatch.setattr(b, "TORCH_OPS", str(tmp_path / "_torch_ops.so"))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libxema.so"))
    monkeypatch.setattr(b, "SOURCES", [])
    monkeypatch.setattr(b, "_torch_ops_command", lambda source: ["torch-ops", source])

    def run(cmd, **kw):
        commands.append(cmd[0])
        open(b.TORCH_OPS if cmd[0] == "torch-ops" else b.LIB, "w").close()
        return type("Result", (), {"returncode": 0, "stdout": "", "stderr": ""})()

    monkeypatch.setattr(b.subprocess, "run", run)
    b.build()
    assert commands.count("torch-ops") == 1
    b.build()
    assert commands.count("torch-ops") == 1
    version = b.metadata.version
    monkeypatch.setattr(b.metadata, "version", lambda name: version(name) + ".other")
    b.build()
    b.build()
    assert commands.count("torch-ops") == 2
    monkeypatch.setattr(b.sys, "version", "another Python")
    b.build()
    assert commands.count("torch-ops") == 3
