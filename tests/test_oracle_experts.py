"""The oracle of the router, the experts' products and the 4-bit rows against hand-worked values and differences, and the
refusals of their entry points (no GPU)."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import oracle
import paper_2411_08446_amd as lsh


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lsh.LIB_PATH):
        from paper_2411_08446_amd import build
        build.build(verbose=False)
    return lsh.load_library()


def test_choice_by_hand():
    inf = np.inf
    logits = np.array([[1.0, 3.0, 3.0, 2.0], [-inf, 0.0, -inf, -inf], [-inf] * 4, [0.0, -0.0, 5.0, 5.0]])
    ids, w = oracle.gate_topk_ref(logits, 2, False)
    assert ids.tolist() == [[1, 2], [1, 0], [0, 1], [2, 3]]
    np.testing.assert_allclose(w, [[0.5, 0.5], [1.0, 0.0], [0.0, 0.0], [0.5, 0.5]])
    _, w = oracle.gate_topk_ref(logits, 1, True)
    z = 2 + math.exp(-2) + math.exp(-1)
    np.testing.assert_allclose(w[:, 0], [1 / z, 1.0, 0.0, 1 / (2 + 2 * math.exp(-5))])


def _differences(f, x, h=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        out[i] = (f(up) - f(down)) / (2 * h)
    return out


@pytest.mark.parametrize("full", [False, True])
def test_logit_gradient_against_differences(full):
    rng = np.random.default_rng(3)
    logits, g = rng.standard_normal((5, 6)), rng.standard_normal((5, 3))
    ids, _ = oracle.gate_topk_ref(logits, 3, full)
    want = _differences(lambda l: float((oracle.gate_topk_ref(l, 3, full)[1] * g).sum()), logits)
    np.testing.assert_allclose(oracle.gate_topk_backward_ref(logits, ids, g, full), want, atol=1e-8)


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
def test_product_gradients_against_differences(act):
    """Two layers, the first with the activation: its pre-activation gradient is what the second one's input call gives."""
    rng = np.random.default_rng(4)
    offsets = [0, 3, 3, 7]
    x, w1, w2 = rng.standard_normal((7, 4)), rng.standard_normal((3, 5, 4)), rng.standard_normal((3, 2, 5))
    b1, b2, g = rng.standard_normal((3, 5)), rng.standard_normal((3, 2)), rng.standard_normal((7, 2))

    def loss(x, w1, b1, w2, b2):
        h = oracle.expert_forward_ref(x, w1, b1, offsets, act)[1]
        return float((oracle.expert_forward_ref(h, w2, b2, offsets, "none")[1] * g).sum())

    pre, h, _ = oracle.expert_forward_ref(x, w1, b1, offsets, act)
    gp = oracle.expert_backward_input_ref(g, w2, offsets, act, pre)[0]
    gw2, gb2, _, _ = oracle.expert_backward_weight_ref(g, h, offsets, 3)
    gx = oracle.expert_backward_input_ref(gp, w1, offsets, "none", None)[0]
    gw1, gb1, _, _ = oracle.expert_backward_weight_ref(gp, x, offsets, 3)
    for got, args in ((gx, 0), (gw1, 1), (gb1, 2), (gw2, 3), (gb2, 4)):
        vals = [x, w1, b1, w2, b2]

        def f(v, args=args, vals=vals):
            return loss(*(vals[:args] + [v] + vals[args + 1:]))
        np.testing.assert_allclose(got, _differences(f, vals[args]), atol=1e-7)


def test_blocks_by_hand():
    x = np.zeros((1, 64))
    x[0, :9] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, -3.5, 5.0, -0.3]       # scale 2^0: ties go to the even code
    x[0, 32:35] = [7.9, -1.0, 3.0]                                       # 7.9 saturates at 6
    codes, scales = oracle.mx4_quantize_ref(x)
    assert scales.tolist() == [[127, 127]]
    assert oracle.mx4_values_ref(codes, scales)[0, :9].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, -4.0, 4.0, -0.5]
    assert oracle.mx4_values_ref(codes, scales)[0, 32:35].tolist() == [6.0, -1.0, 3.0]
    assert codes[0, 0] == 0x07 and codes[0, 4] == 0x09
    x[0, 40] = np.inf
    x[0, :32] = 0.0
    x[0, 3] = 2.0 ** -130
    codes, scales = oracle.mx4_quantize_ref(x)
    assert scales.tolist() == [[0, 255]]
    got = oracle.mx4_values_ref(codes, scales)
    assert np.isnan(got[0, 32:]).all() and got[0, 3] == 0.0
    x[0, 3] = 2.0 ** -126
    assert oracle.mx4_values_ref(*oracle.mx4_quantize_ref(x))[0, 3] == 2.0 ** -126


def test_refusals(lib):
    p, odd = 0x1000, 0x1008       # never dereferenced: every call below is refused before any GPU call
    NULL, SHAPE, UNSUP, WS = lsh.LSHMOE_ERR_NULL, lsh.LSHMOE_ERR_SHAPE, lsh.LSHMOE_ERR_UNSUPPORTED, lsh.LSHMOE_ERR_WORKSPACE
    topk = lib.lshmoe_gate_topk
    assert topk(None, 16, 8, 2, 0, p, p, None) == NULL and topk(p, 16, 8, 2, 0, None, p, None) == NULL
    assert topk(p, 16, 8, 2, 0, p, None, None) == NULL
    assert topk(p, 0, 8, 2, 0, p, p, None) == SHAPE and topk(p, 16, 8, 0, 0, p, p, None) == SHAPE
    assert topk(p, 16, 8, 9, 0, p, p, None) == SHAPE and topk(p, 16, 0, 1, 0, p, p, None) == SHAPE
    assert topk(p, 16, 1025, 2, 0, p, p, None) == UNSUP and topk(p, 16, 128, 65, 0, p, p, None) == UNSUP
    assert topk(p, 1 << 30, 8, 2, 0, p, p, None) == UNSUP and topk(p, 16, 8, 2, 1, p, p, None) == UNSUP
    assert topk(odd, 16, 8, 2, 0, p, p, None) == UNSUP and b"aligned" in lib.lshmoe_last_error()
    back = lib.lshmoe_gate_topk_backward
    for i in range(1, 4):
        args = [p, p, p, p]
        args[i] = None
        assert back(*args, 16, 8, 2, 0, p, None) == NULL
    assert back(p, p, p, p, 16, 8, 2, 0, None, None) == NULL
    assert back(None, p, p, p, 16, 8, 2, lsh.LSHMOE_FLAG_GATE_FULL_SOFTMAX, p, None) == NULL
    assert back(p, p, p, p, 16, 8, 2, 4, p, None) == UNSUP and back(p, p, p, p, 16, 8, 9, 0, p, None) == SHAPE

    fwd = lib.lshmoe_expert_forward
    assert fwd(None, p, None, p, 16, 64, 64, 4, 1, 0, None, p, None) == NULL
    assert fwd(p, p, None, None, 16, 64, 64, 4, 1, 0, None, p, None) == NULL
    assert fwd(p, p, None, p, 16, 64, 64, 4, 1, 0, None, None, None) == NULL
    sizes = [((0, 64, 64, 4, 1), SHAPE), ((16, 0, 64, 4, 1), SHAPE), ((16, 64, -8, 4, 1), SHAPE), ((16, 64, 64, 0, 1), SHAPE),
             ((16, 60, 64, 4, 1), UNSUP), ((16, 64, 60, 4, 1), UNSUP), ((16, 62, 64, 4, 0), UNSUP), ((16, 64, 64, 4, 2), UNSUP),
             ((1 << 30, 8, 8, 4, 1), UNSUP), ((1 << 29, 1024, 8, 4, 1), UNSUP), ((16, 64, 64, 4097, 1), UNSUP),
             ((16, 1 << 22, 8, 1, 1), UNSUP), ((16, 32768, 32768, 1, 1), UNSUP)]
    size = ctypes.c_size_t(0)
    for s, want in sizes:
        assert fwd(p, p, None, p, *s, 0, None, p, None) == want, s
        assert lib.lshmoe_expert_backward_input(p, p, p, *s, 0, None, p, None) == want, s
        assert lib.lshmoe_expert_backward_weight(p, p, p, *s, p, None, p, 1 << 40, None) == want, s
        assert lib.lshmoe_expert_workspace_bytes(*s, ctypes.byref(size)) == want, s
    assert fwd(p, p, None, p, 16, 64, 64, 4, 1, 3, None, p, None) == UNSUP
    for i in (0, 1, 2, 3, 10, 11):
        args = [p, p, p, p, 16, 64, 64, 4, 1, 0, p, p, None]
        args[i] = odd
        assert fwd(*args) == UNSUP and b"aligned" in lib.lshmoe_last_error()
    assert lib.lshmoe_expert_backward_input(p, p, p, 16, 64, 64, 4, 1, 1, None, p, None) == NULL      # slope without pre
    assert lib.lshmoe_expert_backward_input(p, None, p, 16, 64, 64, 4, 1, 0, None, p, None) == NULL
    assert lib.lshmoe_expert_workspace_bytes(16, 64, 64, 4, 1, None) == NULL
    assert lib.lshmoe_expert_backward_weight(p, p, p, 16, 64, 64, 4, 1, None, p, p, 1 << 40, None) == NULL
    for s in ((65536, 256, 512, 1, 1), (8192, 1024, 64, 2, 0), (131072, 1024, 4096, 64, 1)):
        need = lsh.lshmoe_expert_workspace_bytes(*s)
        if need > 0:
            call = lib.lshmoe_expert_backward_weight
            assert call(p, p, p, *s, p, None, None, 1 << 40, None) == WS
            assert call(p, p, p, *s, p, None, 0x1010, 1 << 40, None) == WS
            assert call(p, p, p, *s, p, None, p, need - 1, None) == WS

    for q in (lib.lshmoe_mx4_quantize, None):
        def call(a, rows, d, dt, b, c):
            if q is not None:
                return q(a, rows, d, dt, b, c, None)
            return lib.lshmoe_mx4_dequantize(b, c, rows, d, dt, a, None)
        assert call(None, 16, 64, 1, p, p) == NULL and call(p, 16, 64, 1, None, p) == NULL and call(p, 16, 64, 1, p, None) == NULL
        assert call(p, 0, 64, 1, p, p) == SHAPE and call(p, 16, 0, 1, p, p) == SHAPE
        assert call(p, 16, 48, 1, p, p) == UNSUP and call(p, 16, 64, 5, p, p) == UNSUP and call(p, 1 << 30, 32, 1, p, p) == UNSUP
        assert call(p, 16, 64, 1, odd, p) == UNSUP and call(p, 16, 64, 1, p, odd) == UNSUP
    mx = lib.lshmoe_expert_forward_mx4
    for i in (0, 1, 2, 3, 5, 12):
        args = [p, p, p, p, None, p, 16, 64, 64, 4, 1, 0, p, None]
        args[i] = None
        assert mx(*args) == NULL, i
        args[i] = odd
        assert mx(*args) == UNSUP, i
    assert mx(p, p, p, p, None, p, 16, 48, 64, 4, 1, 0, p, None) == UNSUP
    assert mx(p, p, p, p, None, p, 16, 64, 64, 4, 1, 7, p, None) == UNSUP


def test_binding_refuses_mismatched_tensors():
    """Shapes, types and places are looked at before anything is launched."""
    f, b, i, u = (lambda *s: torch.zeros(*s), lambda *s: torch.zeros(*s, dtype=torch.bfloat16),
                  lambda *s: torch.zeros(*s, dtype=torch.int32), lambda *s: torch.zeros(*s, dtype=torch.uint8))
    with pytest.raises(ValueError):
        lsh.lshmoe_gate_topk(f(4, 8), i(4, 2), f(4, 3))
    with pytest.raises(ValueError):
        lsh.lshmoe_gate_topk(f(4, 8), i(4, 2), f(4, 2))                       # on the host
    with pytest.raises(ValueError):
        lsh.lshmoe_gate_topk_backward(f(4, 7), i(4, 2), f(4, 2), f(4, 2), f(4, 8))
    with pytest.raises(ValueError):
        lsh.lshmoe_expert_forward(b(4, 8), b(2, 16, 16), None, i(3), b(4, 16))
    with pytest.raises(ValueError):
        lsh.lshmoe_expert_forward(b(4, 8), b(2, 16, 8), b(2, 8), i(3), b(4, 16))
    with pytest.raises(ValueError):
        lsh.lshmoe_expert_forward(b(4, 8), b(2, 16, 8), None, i(2), b(4, 16))
    with pytest.raises(ValueError):
        lsh.lshmoe_expert_backward_input(b(4, 16), b(2, 16, 8), i(3), b(4, 16))
    with pytest.raises(ValueError):
        lsh.lshmoe_expert_backward_weight(b(4, 16), b(5, 8), i(3), b(2, 16, 8), None, u(0))
    with pytest.raises(ValueError):
        lsh.lshmoe_mx4_quantize(b(4, 64), u(4, 32), u(4, 3))
    with pytest.raises(ValueError):
        lsh.lshmoe_mx4_dequantize(u(4, 32), u(4, 1), b(4, 64))
    with pytest.raises(ValueError):
        lsh.lshmoe_expert_forward_mx4(u(4, 32), u(4, 2), u(2, 16, 32), u(2, 16, 1), None, i(3), b(4, 16))


def test_a_workspace_shorter_than_its_alignment_has_no_bytes():
    from paper_2411_08446_amd import binding
    ws = torch.zeros(600, dtype=torch.uint8)
    start = (-ws.data_ptr()) % 256 + 1
    assert binding._aligned_ws(ws[start:start + 16])[1] == 0
