"""Tokens and classes as a tokenizer's int64: numbers that int32 does not hold are masked places and classes that there are none of, as any others outside the vocabulary."""
import pytest
import torch

pytestmark = pytest.mark.gpu
FAR = [2 ** 32 + 3, -2 ** 32 + 3, 2 ** 31, -2 ** 31 - 1, 2 ** 63 - 1, -2 ** 63, 2 ** 33, 2 ** 32 - 1]


def make(**kw):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    return GatedMLP(2 * len(FAR), 64, 64, 16, 1, **kw)


def mixed(near):
    """Every second place far away, and the same with -1 there."""
    far, masked = torch.tensor(FAR), torch.full((len(FAR),), -1)
    return [torch.stack([near, f], 1).view(-1) for f in (far, masked)]


@pytest.mark.parametrize("device", ["cpu", "cuda:0"])
def test_a_step(device):
    nets = make(vocab=24), make(vocab=24)
    near = torch.arange(len(FAR))
    for m, ids, labels in zip(nets, mixed(near), mixed(near + 4)):
        m.set_tokens(ids.to(device), labels.to(device))
        m.step()
    torch.cuda.synchronize()
    a, b = nets
    assert torch.equal(a.r[0], b.r[0]) and bool((a.r[0][1::2] == 0).all()) and bool((a.r[0][::2] != 0).any(1).all())
    assert torch.equal(a.logits, b.logits) and torch.equal(a.dlogits, b.dlogits) and torch.equal(a.master, b.master)
    for m in nets:          # a class that there is none of: no loss, and no gradient
        assert bool(torch.isnan(m.loss[1::2]).all()) and bool(torch.isfinite(m.loss[::2]).all()) and bool((m.dlogits[1::2] == 0).all())


def test_classes_of_rows():
    a, b = make(), make()
    x = torch.randn(2 * len(FAR), 64, generator=torch.Generator().manual_seed(1))
    for m, labels in zip((a, b), mixed(torch.arange(len(FAR)))):
        m.set_batch(x, labels)
        m.step()
    torch.cuda.synchronize()
    assert bool(torch.isnan(a.loss[1::2]).all()) and torch.equal(a.dlogits, b.dlogits) and torch.equal(a.master, b.master)


@pytest.mark.parametrize("i8", [False, True])
def test_answers(i8):
    m = make(vocab=24)
    m.prepare_answers_i8()
    far, masked = (t.cuda() for t in mixed(torch.arange(len(FAR))))
    assert torch.equal(m.answer(far, i8=i8), m.answer(masked, i8=i8))
    assert torch.equal(m.answer(far, i8=i8), m.answer(masked.to(torch.int32), i8=i8))
