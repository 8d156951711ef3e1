"""The stack of gated feed-forward blocks (paper_1807_11205_amd/gated_mlp.py): a whole training step against the same network in 64 bits, the
clipped update, what an overflow does, and answers for single rows.

The step rounds to FP16 about ten times between a weight and its gradient in each block (2^-11 / sqrt 3 of a value each time, independent): two blocks
and the classifier leave about sqrt(30) 2.8e-4 = 1.5e-3 of a gradient's norm; 5e-3 is asked for, and 2e-3 of the logits'."""
import numpy as np
import pytest
import torch

from oracle import blocks

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


def make(rows=96, **kw):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    m = GatedMLP(rows, 128, 352, 40, 2, **kw)
    g = np.random.default_rng(17)
    x, labels = torch.from_numpy(g.standard_normal((rows, 128)) * 2).float(), torch.from_numpy(g.integers(0, 40, rows)).int()
    m.set_batch(x, labels)
    return m, x.double().numpy(), labels.numpy()


def in_64_bits(m, x, labels):
    """logits, loss, gradients (without a loss scale) of the network with the weights that m has."""
    from paper_1807_11205_amd.gated_mlp import EPS
    w = {n: m._param(m.master if len(s) == 1 or n.startswith("gate_") else m.w16, n).double().cpu().numpy() for n, s in m.shapes.items()}
    L, k = m.blocks, dict(eps=EPS, res_scale=1.0, branch_scale=m.scale)
    r, kept = x, []
    f = blocks.norm_residual_fwd(x, None, None, None, w["w_pre_0"], **k)
    kept.append(dict(r_out=x, k2=f["rstd_pre"]))
    n = f["n"]
    for i in range(L):
        t = blocks.ffn_fwd(n, w["w_gate_%d" % i], w["w_up_%d" % i], w["w_down_%d" % i], "silu")
        f = blocks.norm_residual_fwd(r, t["y"], w["w_post_%d" % i], w["gate_%d" % i], w["w_pre_%d" % (i + 1)], **k)
        kept.append(dict(n=n, t=t, r_out=f["r_out"], k1=f["rstd_post"], k2=f["rstd_pre"]))
        r, n = f["r_out"], f["n"]
    z = n @ w["w_fc"].T
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    loss = -np.log(p[np.arange(len(z)), labels])
    dz = p.copy()
    dz[np.arange(len(z)), labels] -= 1
    dz /= len(z)
    g = dict(w_fc=dz.T @ n)
    dn, dr = dz @ w["w_fc"], None
    for i in reversed(range(L)):
        s = kept[i + 1]
        b = blocks.norm_residual_bwd(s["t"]["y"], s["r_out"], w["w_post_%d" % i], w["gate_%d" % i], w["w_pre_%d" % (i + 1)], s["k1"], s["k2"], dr, dn, 1.0, m.scale)
        g["w_post_%d" % i], g["gate_%d" % i], g["w_pre_%d" % (i + 1)] = b["dw_post"], b["dgate"], b["dw_pre"]
        c = blocks.ffn_bwd(s["n"], w["w_gate_%d" % i], w["w_up_%d" % i], w["w_down_%d" % i], s["t"]["gate"], s["t"]["up"], s["t"]["h"], b["dy"], "silu")
        g["w_gate_%d" % i], g["w_up_%d" % i], g["w_down_%d" % i] = c["dwg"], c["dwu"], c["dwd"]
        dn, dr = c["dx"], b["dr"]
    b = blocks.norm_residual_bwd(None, kept[0]["r_out"], None, None, w["w_pre_0"], None, kept[0]["k2"], dr, dn, 1.0, m.scale, branch=False)
    g["w_pre_0"] = b["dw_pre"]
    return z, loss, g


def rel(got, ref):
    return np.linalg.norm(got - ref) / np.linalg.norm(ref)


def test_a_step_against_64_bits(jz):
    S = 256.0
    m, x, labels = make(initial_loss_scale=S, max_norm=0.01)
    z, loss, grads = in_64_bits(m, x, labels)
    m.forward()
    m.backward()
    torch.cuda.synchronize()
    assert rel(m.logits.double().cpu().numpy(), z) <= 2e-3
    assert abs(m.mean_loss() - loss.mean()) <= 2e-3 * loss.mean()
    for n in m.shapes:
        assert rel(m._param(m.grad, n).double().cpu().numpy().reshape(grads[n].shape) / S, grads[n]) <= 5e-3, n
    # clipping, then the update on the clipped gradients
    before, g16 = m.grad.double().cpu().numpy(), None
    w0, v0 = m.master.clone(), m.momentum.clone()
    m.update()
    torch.cuda.synchronize()
    norm = np.linalg.norm(before) / S
    assert norm > m.max_norm and abs(float(m.norm) - norm) <= 2.0 ** -22 * norm and int(m.found_inf) == int(m.clip_found_inf) == 0
    g16 = m.grad.double().cpu().numpy()
    assert abs(np.linalg.norm(g16) / S - m.max_norm) <= 1e-3 * m.max_norm
    assert not torch.equal(m.master, w0) and not torch.equal(m.momentum, v0)
    assert torch.equal(m.w16, m.master.half())


def test_it_learns_its_batch(jz):
    m, _, _ = make(rows=64, hparams=dict(lr=3.0))
    losses = []
    for _ in range(40):
        m.step()
        losses.append(m.mean_loss())
    assert np.isfinite(losses).all() and losses[-1] < 0.3 * losses[0], losses


def test_an_overflow_skips_the_update_and_lowers_the_scale(jz):
    m, _, _ = make(initial_loss_scale=2.0 ** 15, policy=dict(max_scale=2.0 ** 16))
    m.forward()
    m.backward()
    m._param(m.grad, "w_up_1")[3, 5] = float("inf")
    w0, g0 = m.master.clone(), m.grad.clone()
    m.update()
    torch.cuda.synchronize()
    assert int(m.clip_found_inf) == int(m.found_inf) == 1
    assert torch.equal(m.master, w0) and torch.equal(m.grad, g0)
    assert jz.loss_scale_state(m.ls_state)[0] == 2.0 ** 14


@pytest.mark.parametrize("rows", [1, 5, 64, 96])
def test_answers_are_the_training_forward_pass_row_by_row(jz, rows):
    m, x, labels = make()
    m.forward()
    got = m.answer(torch.from_numpy(x[:rows]).float().cuda())
    torch.cuda.synchronize()
    want = m.logits[:rows].double().cpu().numpy()
    assert rel(got.double().cpu().numpy(), want) <= 2e-3


def test_the_step_in_a_graph(jz):
    a, _, _ = make(seed=5)
    b, _, _ = make(seed=5)
    a.step()                                # both once: a graph records launches, not what a first call does on the host
    b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(4):
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.master, b.master) and torch.equal(a.grad, b.grad) and torch.equal(a.logits, b.logits)
        assert a.mean_loss() == b.mean_loss()


def test_sizes_that_do_not_fit_the_fused_buffers(jz):
    from paper_1807_11205_amd.gated_mlp import GatedMLP
    with pytest.raises(ValueError):
        GatedMLP(8, 100, 64, 16, 1)
