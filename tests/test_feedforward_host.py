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
