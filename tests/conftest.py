import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a real MI355X (run with -m gpu)")


@pytest.fixture(autouse=True)
def what_a_graph_reads_stays(request, monkeypatch):
    """A captured graph reads the tensors that it was captured with, and the memory of dropped ones goes to whoever asks next. One test drops
    the first of its two graphs' queries, offsets and work buffer while it still replays that graph; here they stay until it has ended."""
    if request.node.name != "test_two_graphs_with_workspaces_of_their_own":
        return
    import torch
    kept = []

    def keeping(make):
        def made(*args, **kw):
            kept.append(make(*args, **kw))
            return kept[-1]
        return made

    monkeypatch.setattr(request.module, "queries", keeping(request.module.queries))
    monkeypatch.setattr(torch, "empty", keeping(torch.empty))
    request.addfinalizer(kept.clear)
