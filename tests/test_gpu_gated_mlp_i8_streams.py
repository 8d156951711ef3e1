"""Answers in 8-bit integers while the codes are written on another stream, with other work in front of either."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
CYCLES = 50_000_000         # some tens of milliseconds


def make():
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    return GatedMLP(96, 128, 352, 40, 2, vocab=56)


def tokens():
    return torch.from_numpy(np.random.default_rng(1).integers(0, 56, 70).astype(np.int32)).cuda()


@pytest.mark.parametrize("how", ["current", "other"])
def test_answers_wait_for_codes_that_are_being_written(how):
    a, b, codes, other = make(), make(), torch.cuda.Stream(), torch.cuda.Stream()
    ids = tokens()
    a.prepare_answers_i8()
    want = a.answer(ids, i8=True)
    torch.cuda.synchronize()
    with torch.cuda.stream(codes):
        torch.cuda._sleep(CYCLES)
    b.prepare_answers_i8(stream=codes)
    got = b.answer(ids, other if how == "other" else None, i8=True)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(got, want) and bool(want.any())


def test_codes_wait_for_answers_in_flight():
    m, codes, other = make(), torch.cuda.Stream(), torch.cuda.Stream()
    ids = tokens()
    m.prepare_answers_i8()
    want = [m.answer(ids, i8=True)]
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        torch.cuda._sleep(CYCLES)
    got = [m.answer(ids, other, i8=True)]
    with torch.cuda.stream(codes):
        m._param(m.w16, "w_up_0").mul_(-3)      # an answer with codes reads it no more
    m.prepare_answers_i8(stream=codes.cuda_stream)
    got.append(m.answer(ids, other, i8=True))
    torch.cuda.synchronize()
    want.append(m.answer(ids, i8=True))
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and not torch.equal(*want)


def test_answers_in_a_graph():
    m, ids = make(), tokens()
    m.prepare_answers_i8(stream=torch.cuda.Stream())
    m.answer(ids, i8=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.answer(ids, i8=True)
    for k in range(4):
        m._param(m.w16, "w_down_1").mul_(-1.5)
        m.prepare_answers_i8()
        want = m.answer(ids, i8=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
