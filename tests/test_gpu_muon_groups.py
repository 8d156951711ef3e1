"""The orthogonalised updates of the stack of gated blocks are one step with LARS' over both groups of matrices: a momentum that is not finite, or will not be, stops all of it."""
import pytest
import torch

from test_gpu_token_mlp import S, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


@pytest.mark.parametrize("where", ["w_gate_0", "w_up_1", "w_down_0", "w_down_1"])
@pytest.mark.parametrize("value,momentum", [(float("inf"), 0.95), (float("nan"), 0.95), (3e38, 1.5)])
def test_a_momentum_that_overflows_skips_everything(jz, where, value, momentum):
    m, _, _ = make(False, "muon", muon=dict(momentum=momentum))
    m.step()
    m.forward()
    m.backward()
    at = m._param(m.momentum, where).view(-1)
    kept = float(at[77])
    at[77] = value
    w0, v0, h0 = m.master.clone(), m.momentum.clone(), m.w16.clone()
    m.update()
    torch.cuda.synchronize()
    assert int(m.found_inf) == 1 and int(m.clip_found_inf) == 0
    assert torch.equal(m.master, w0) and torch.equal(m.momentum.view(torch.int32), v0.view(torch.int32)) and torch.equal(m.w16, h0)
    assert jz.loss_scale_state(m.ls_state)[0] == S / 2
    at[77] = kept
    m.step()
    torch.cuda.synchronize()
    assert int(m.found_inf) == 0
    for n in ("w_gate_0", "w_up_1", "w_down_1", "w_pre_1", "embed"):
        assert not torch.equal(m._param(m.master, n), m._param(w0, n)), n


@pytest.mark.parametrize("B,R,C", [(3, 40, 90), (2, 2100, 2050), (300, 33, 20)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_the_flag_ahead_of_an_update(jz, B, R, C, dtype):
    """The flag that the update sets, and nothing else is written."""
    g = torch.Generator(device="cuda").manual_seed(R)
    d, hp = jz.ortho_desc(B, R, C, jz.dtype_of(dtype)), jz.muon_hparams(momentum=1.25, loss_scale=2.0)
    grad, v = torch.randn((B, R, C), generator=g, device="cuda").to(dtype), torch.randn((B, R, C), generator=g, device="cuda")
    ws = torch.full((jz.jz_muon_mp_update_workspace_bytes(d),), 0x7f, dtype=torch.uint8, device="cuda")
    flag, skip = torch.full((1,), 77, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jz.jz_muon_mp_overflow(d, hp, v, grad, flag, ws, skip=skip)
    inf = float("inf")
    # what is put at one place of the gradient and of the momentum: nothing, what is not finite, and what the momentum's factor takes beyond FP32
    for in_grad, in_v, skipped in [(None, None, 0), (inf, None, 0), (None, None, 1), (float("nan"), None, 0), (None, -inf, 0), (None, 2.9e38, 0), (None, 2.0e38, 0), (None, None, 0)]:
        at = (B - 1, R // 2, C - 1)
        kept = grad[at].clone(), v[at].clone()
        if in_grad is not None:
            grad[at] = in_grad
        if in_v is not None:
            v[at] = in_v
        skip.fill_(skipped)
        before = grad.clone(), v.clone()
        flags = []
        for how in ("call", "address", "graph"):
            flag.fill_(77)
            if how == "graph":
                graph.replay()
            else:
                jz.jz_muon_mp_overflow(d, hp, v, grad, flag if how == "call" else flag.data_ptr(), ws, skip=skip if how == "call" else skip.data_ptr())
            flags.append(int(flag))
        bits = lambda t: t.view(torch.int32 if t.element_size() == 4 else torch.int16)
        assert torch.equal(bits(grad), bits(before[0])) and torch.equal(bits(v), bits(before[1]))
        # 2.0e38: 1.25 of it is a number, and 1.25 of that one more
        want = int(skipped or in_grad is not None or in_v in (-inf, 2.9e38))
        assert flags == [want] * 3, (in_grad, in_v, skipped)
        w, w16 = torch.zeros((B, R, C), device="cuda"), torch.zeros((B, R, C), dtype=dtype, device="cuda")
        moved = v.clone()
        jz.jz_muon_mp_update(d, hp, w, moved, grad, w16, flag, ws, skip=skip.data_ptr())
        assert int(flag) == want
        grad[at], v[at] = kept


def test_the_flag_without_matrices(jz):
    d = jz.ortho_desc(0, 8, 8)
    flag, skip, ws = torch.full((1,), 5, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"), torch.empty(16, dtype=torch.uint8, device="cuda")
    f, e = torch.empty((0, 8, 8), device="cuda"), torch.empty((0, 8, 8), dtype=torch.float16, device="cuda")
    jz.jz_muon_mp_overflow(d, jz.muon_hparams(), f, e, flag, ws)
    assert int(flag) == 0
    jz.jz_muon_mp_overflow(d, jz.muon_hparams(), f, e, flag, ws, skip=skip)
    assert int(flag) == 1
