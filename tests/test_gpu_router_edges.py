"""The router's gradient where logits or the weights' gradients are not finite."""
import pytest
import torch

import paper_2411_08446_amd as lsh

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _forward(logits, k, flags):
    T = logits.shape[0]
    ids = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), 7.0, device="cuda")
    lsh.lshmoe_gate_topk(logits, ids, w, flags=flags)
    return ids, w


def _backward(logits, ids, w, g, E, flags):
    out = torch.full((ids.shape[0], E), 7.0, device="cuda")
    lsh.lshmoe_gate_topk_backward(logits, ids, w, g, out, flags=flags)
    return out.cpu()


# one and more pieces of logits to a lane, rows that end inside the last lane's pieces and rows that do not
@pytest.mark.parametrize("E", [2, 3, 4, 5, 6, 8, 17, 60, 64, 100, 128, 160, 256, 333, 512, 1000, 1024])
def test_nan_among_the_logits_reaches_the_gradient(E):
    """With the softmax over all experts every weight of such a token is NaN, and so is every entry of its gradient; only a token
    without any expert left gets zeros.  Tokens beside it are not touched."""
    k = min(3, E)
    gen = torch.Generator().manual_seed(E)
    logits = torch.randn(8, E, generator=gen)
    logits[0] = NAN
    logits[1], logits[1, E // 2] = -INF, NAN
    logits[2, E - 1] = NAN
    logits[3], logits[3, 0] = -INF, NAN
    logits[4, 1] = INF
    logits[5] = -INF
    flags = lsh.LSHMOE_FLAG_GATE_FULL_SOFTMAX
    lt = logits.cuda()
    ids, w = _forward(lt, k, flags)
    got = _backward(lt, ids, w, torch.randn(8, k, generator=gen).cuda(), E, flags)
    w = w.cpu()
    for t in range(5):
        assert torch.isnan(w[t]).all() and torch.isnan(got[t]).all(), "token %d" % t
    assert (w[5] == 0.0).all() and (got[5] == 0.0).all()
    assert torch.isfinite(got[6:]).all()
    # over the chosen experts: NaN for those, zeros for the others
    ids, w = _forward(lt, k, 0)
    got = _backward(None, ids, w, torch.randn(8, k, generator=gen).cuda(), E, 0)
    ids = ids.cpu().long()
    for t in (0, 2, 3):
        chosen = torch.zeros(E, dtype=torch.bool)
        chosen[ids[t]] = True
        assert torch.isnan(got[t][chosen]).all() and (got[t][~chosen] == 0.0).all(), "token %d" % t
    assert (got[5] == 0.0).all() and torch.isfinite(got[6:]).all()


@pytest.mark.parametrize("full", [False, True])
@pytest.mark.parametrize("E", [3, 8, 60, 256, 1000])
def test_a_token_without_experts_gets_zeros_whatever_its_gradient_is(E, full):
    """Its weights are 0, and the rows behind them may hold anything: infinities and NaN of their gradients end there."""
    k = min(4, E)
    gen = torch.Generator().manual_seed(E)
    logits = torch.randn(5, E, generator=gen)
    logits[1:4] = -INF
    g = torch.randn(5, k, generator=gen)
    g[1], g[2, 0], g[3, k - 1] = NAN, INF, -INF
    flags = lsh.LSHMOE_FLAG_GATE_FULL_SOFTMAX if full else 0
    lt = logits.cuda()
    ids, w = _forward(lt, k, flags)
    got = _backward(lt if full else None, ids, w, g.cuda(), E, flags)
    assert (w.cpu()[1:4] == 0.0).all() and (got[1:4] == 0.0).all()
    assert torch.isfinite(got[0]).all() and torch.isfinite(got[4]).all() and (got[0] != 0.0).any()


def test_a_gradient_that_is_not_finite_reaches_the_token_whose_weights_are_not_zero():
    logits = torch.tensor([[1.0, -INF, 0.0, -INF, 2.0]] * 2)
    g = torch.tensor([[1.0, NAN, 0.5], [1.0, 2.0, INF]])
    for flags in (0, lsh.LSHMOE_FLAG_GATE_FULL_SOFTMAX):
        lt = logits.cuda()
        ids, w = _forward(lt, 3, flags)
        got = _backward(lt, ids, w, g.cuda(), 5, flags)
        assert ids.tolist() == [[4, 0, 2]] * 2
        assert torch.isnan(got[0, [4, 0, 2]]).all() and not torch.isfinite(got[1, [4, 0, 2]]).any()
