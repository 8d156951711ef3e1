"""The stack of gated blocks with tokens in front, orthogonalised updates and 8-bit answers (paper_1807_11205_amd/gated_mlp.py): the operators run together, each against its
definition on what it saw, and the whole against the network in 64 bits with the bounds of test_gpu_gated_mlp.py (about ten roundings to FP16 between a weight and
its gradient in each block)."""
import types

import numpy as np
import pytest
import torch

from oracle import blocks, tokens
from test_gpu_gated_mlp import in_64_bits, rel

pytestmark = pytest.mark.gpu
C32 = tuple(float(np.float32(c)) for c in (3.4445, -4.7750, 2.0315))
S = 256.0


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


def make(tied=False, optimizer="lars", rows=96, seed=1, **kw):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    m = GatedMLP(rows, 128, 352, 40, 2, seed=seed, vocab=40 if tied else 56, embed_scale=3.0, tied=tied, optimizer=optimizer, initial_loss_scale=S, **kw)
    g = np.random.default_rng(17)
    ids, labels = np.minimum(g.exponential(9, rows), m.vocab - 1).astype(np.int32), g.integers(0, 40, rows)
    ids[5] = -1
    m.set_tokens(torch.from_numpy(ids), torch.from_numpy(labels).int())
    return m, ids, labels


def host(t):
    return t.detach().double().cpu().numpy()


def plain(m):
    """The network with its classifier under the name that in_64_bits knows."""
    shapes = {("w_fc" if n == m.fc else n): s for n, s in m.shapes.items() if n in (m.fc,) or n != "embed"}
    return types.SimpleNamespace(shapes=shapes, blocks=m.blocks, scale=m.scale, master=m.master, w16=m.w16, _param=lambda buf, n: m._param(buf, m.fc if n == "w_fc" else n))


@pytest.mark.parametrize("tied", [False, True])
def test_forward_and_backward(jz, tied):
    m, ids, labels = make(tied)
    m.forward()
    m.backward()
    torch.cuda.synchronize()
    x = tokens.embed_fwd(ids, host(m._param(m.w16, "embed")), 3.0)
    assert np.array_equal(host(m.r[0]), x.astype(np.float32))           # one rounding of FP32
    z, loss, grads = in_64_bits(plain(m), x, labels)
    assert rel(host(m.logits), z) <= 2e-3 and abs(m.mean_loss() - loss.mean()) <= 2e-3 * loss.mean()
    for n, g in grads.items():
        if not (tied and n == "w_fc"):
            assert rel(host(m._param(m.grad, m.fc if n == "w_fc" else n)).reshape(g.shape) / S, g) <= 5e-3, n
    # the table's, from the gradient that arrived at the rows; a tied one holds the classifier's too
    before = S * grads["w_fc"] if tied else None
    ref, _ = tokens.embed_bwd(ids, host(m.dr), m.vocab, 3.0, before)
    assert rel(host(m._param(m.grad, "embed")), ref) <= 5e-3


@pytest.mark.parametrize("tied", [False, True])
def test_the_muon_update(jz, tied):
    m, ids, labels = make(tied, "muon", max_norm=0.05, muon=dict(lr=0.03, weight_decay=0.01))
    m.forward()
    m.backward()
    m.momentum.copy_(torch.randn(m.momentum.shape, generator=torch.Generator().manual_seed(3)) * 1e-4)
    torch.cuda.synchronize()
    w0, v0 = m.master.clone(), m.momentum.clone()
    m.update()
    torch.cuda.synchronize()
    assert int(m.found_inf) == int(m.clip_found_inf) == 0 and jz.loss_scale_state(m.ls_state) == (S, 1)
    for n, shape in m.shapes.items():
        if not n.startswith(("w_gate_", "w_up_", "w_down_")):
            assert not torch.equal(m._param(m.master, n), m._param(w0, n)), n
            continue
        hp = dict(lr=float(np.float32(0.03)), momentum=float(np.float32(0.95)), weight_decay=float(np.float32(0.01)), nesterov=True,
                  update_scale=float(np.float32(max(1.0, shape[0] / shape[1]) ** 0.5)))
        w, v, o, _ = tokens.muon(host(m._param(w0, n)), host(m._param(v0, n)), host(m._param(m.grad, n)) / S, hp, C32, 5, float(np.float32(1e-7)))
        assert rel(host(m._param(m.momentum, n)), v) <= 2.0 ** -22
        # the iteration's result is within 2^-12 of itself at these sizes (test_gpu_ortho.py), and its roundings to FP32 are far below
        assert np.linalg.norm(host(m._param(m.master, n)) - w) <= 2.0 ** -12 * hp["lr"] * hp["update_scale"] * np.linalg.norm(o) + 2.0 ** -22 * np.linalg.norm(w), n
    assert torch.equal(m.w16, m.master.half())


@pytest.mark.parametrize("where", ["w_up_1", "w_down_0", "w_pre_1", "embed"])
def test_an_overflow_anywhere_skips_everything(jz, where):
    m, _, _ = make(False, "muon")
    m.step()
    m.forward()
    m.backward()
    m._param(m.grad, where).view(-1)[77] = float("nan")
    w0, v0, h0 = m.master.clone(), m.momentum.clone(), m.w16.clone()
    m.update()
    torch.cuda.synchronize()
    assert int(m.clip_found_inf) == int(m.found_inf) == 1
    assert torch.equal(m.master, w0) and torch.equal(m.momentum, v0) and torch.equal(m.w16, h0)
    assert jz.loss_scale_state(m.ls_state)[0] == S / 2
    m.step()
    torch.cuda.synchronize()
    assert int(m.found_inf) == 0 and not torch.equal(m._param(m.master, "w_up_1"), m._param(w0, "w_up_1")) and not torch.equal(m._param(m.master, "w_pre_1"), m._param(w0, "w_pre_1"))


@pytest.mark.parametrize("optimizer", ["lars", "muon"])
def test_the_step_in_a_graph(jz, optimizer):
    a, _, _ = make(True, optimizer, seed=5)
    b, _, _ = make(True, optimizer, seed=5)
    a.step()
    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(4):
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.master, b.master) and torch.equal(a.grad, b.grad) and torch.equal(a.momentum, b.momentum) and torch.equal(a.logits, b.logits)


def half(v):
    return v.astype(np.float16).astype(np.float64)


@pytest.mark.parametrize("rows", [1, 3, 64, 96])
def test_answers_in_8_bits(jz, rows):
    """Against the same network in 64 bits with codes: what is rounded to FP16 between the products is rounded there too."""
    from paper_1807_11205_amd.gated_mlp import EPS
    m, ids, _ = make()
    with pytest.raises(ValueError):
        m.answer(torch.from_numpy(ids).cuda(), i8=True)
    m.prepare_answers_i8()
    side = torch.cuda.Stream()
    t = torch.from_numpy(ids[:rows]).cuda()
    got = m.answer(t, i8=True)
    again = m.answer(t, stream=side, i8=True)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, again)
    w = lambda n: host(m._param(m.master, n))
    code = {n: tokens.quantize(host(m._param(m.w16, n))) for n in m.i8}
    for n, (q, s) in m.i8.items():
        assert np.array_equal(q.cpu().numpy()[:, :m.shapes[n][1]], code[n][0]) and np.array_equal(s.cpu().numpy(), code[n][1])
    r = tokens.embed_fwd(ids[:rows], host(m._param(m.w16, "embed")), 3.0)
    k = dict(eps=EPS, res_scale=1.0, branch_scale=m.scale)
    n = blocks.norm_residual_fwd(r, None, None, None, w("w_pre_0"), **k)["n"]
    for i in range(m.blocks):
        y, _ = tokens.ffn_i8(*tokens.quantize(half(n)), *(code["%s_%d" % (a, i)] for a in ("w_gate", "w_up", "w_down")), "silu")
        f = blocks.norm_residual_fwd(r, half(y), w("w_post_%d" % i), w("gate_%d" % i), w("w_pre_%d" % (i + 1)), **k)
        r, n = f["r_out"], f["n"]
    z = tokens.linear_i8(*tokens.quantize(half(n)), *code["w_fc"])
    assert rel(host(got), z) <= 2e-3
    # and the matrices' own rounding to codes: 127 steps to a row's largest, so a product's two operands are off by 1 / 254 sqrt(3) of 3 to 4 times their root mean square
    assert rel(host(got), host(m.answer(t))) <= 0.1


def test_what_is_refused(jz):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    for bad in (dict(vocab=24, tied=True), dict(tied=True), dict(vocab=-1), dict(optimizer="sgd")):
        with pytest.raises(ValueError):
            GatedMLP(8, 64, 64, 16, 1, **bad)
    with pytest.raises(ValueError):
        GatedMLP(8, 64, 64, 16, 1).set_tokens(torch.zeros(8, dtype=torch.int32), torch.zeros(8, dtype=torch.int32))


def test_tokens_and_rows_are_not_mixed_up(jz):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    m = GatedMLP(8, 64, 64, 16, 1, vocab=24)
    with pytest.raises(ValueError):
        m.set_batch(torch.zeros(8, 64), torch.zeros(8, dtype=torch.int32))
    with pytest.raises(ValueError):
        m.answer(torch.zeros(8, 64, device=m.device))
    with pytest.raises(ValueError):
        m.answer(torch.zeros(8, device=m.device))
    with pytest.raises(ValueError):
        m.answer(torch.zeros(8, dtype=torch.int32, device=m.device), i8=True)
    m.prepare_answers_i8()
    ids = torch.tensor([3, 0, 23, 24, -1, 3], device=m.device)
    for i8 in (False, True):
        assert torch.equal(m.answer(ids, i8=i8), m.answer(ids.to(torch.int32), i8=i8))


def test_without_blocks(jz):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    m = GatedMLP(16, 64, 64, 16, 0, vocab=16, tied=True, optimizer="muon")
    m.set_tokens(torch.arange(16, dtype=torch.int32), torch.arange(16, dtype=torch.int32))
    before = m.master.clone()
    m.step()
    assert np.isfinite(m.mean_loss()) and int(m.found_inf) == 0 and not torch.equal(m.master, before)
