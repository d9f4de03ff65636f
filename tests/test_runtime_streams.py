"""The stream that calls are enqueued on, with and without torch's quick way to its handle."""
import importlib.util

import torch

from paper_2605_22566_b200 import runtime


def test_the_current_stream_without_the_quick_way(monkeypatch):
    """(A copy of the module, loaded where torch has no such call.)"""
    asked = []

    class Stream:
        cuda_stream = 4711
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: asked.append(index) or Stream())
    spec = importlib.util.spec_from_file_location("paper_2605_22566_b200.runtime_copy", runtime.__file__)
    copy = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(copy)
    assert copy._raw_stream(3) == 4711 and asked == [3]
    pa = object.__new__(copy.PathAttention)
    pa.g, pa._guards, pa.pool = None, [], type("Pool", (), {"device": torch.device("cuda", 2)})
    assert pa.stream == 4711 and asked == [3, 2]
