"""What set_tokens of the stack of gated blocks refuses (no GPU: the buffers are on the host)."""
import contextlib

import pytest
import torch

from paper_1807_11205_amd import gated_mlp


@pytest.fixture
def net(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    m = gated_mlp.GatedMLP.__new__(gated_mlp.GatedMLP)
    m.rows, m.vocab, m.device = 6, 24, torch.device("cpu")
    m.ids, m.labels = torch.full((6,), 99, dtype=torch.int32), torch.full((6,), 99, dtype=torch.int32)
    return m


@pytest.mark.parametrize("ids,labels", [(torch.zeros(()), torch.zeros(6)), (torch.tensor(3), torch.arange(6)), (torch.tensor([3]), torch.arange(6)), (torch.arange(6), torch.tensor([3])),
                                        (torch.arange(5), torch.arange(5)), (torch.arange(6).view(6, 1), torch.arange(6)), (torch.arange(6).float(), torch.arange(6)),
                                        (torch.arange(6).half(), torch.arange(6))])
def test_refused_and_nothing_written(net, ids, labels):
    with pytest.raises(ValueError):
        net.set_tokens(ids, labels)
    assert bool((net.ids == 99).all()) and bool((net.labels == 99).all())


@pytest.mark.parametrize("dtype", [torch.int64, torch.int32, torch.int16, torch.uint8])
def test_taken(net, dtype):
    net.set_tokens(torch.arange(6, dtype=dtype), torch.arange(6, dtype=dtype).flip(0))
    assert net.ids.tolist() == [0, 1, 2, 3, 4, 5] and net.labels.tolist() == [5, 4, 3, 2, 1, 0]
