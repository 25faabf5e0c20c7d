"""GELU and its slope over all of their range, by their error relative to the value, on each kernel that applies them.

The value comes through the bias of a product of zeros, so that v is exact; the slope through a product that is 1.  With
u = |v|, Q(u) the normal distribution beyond u and phi its density, v Phi(v) is max(v, 0) - u Q(u) and the slope Phi(v) + v phi(v).

Bounds, in units of 2^-24 of Q, for binary32 results: the reciprocal and its argument 3, up to twice that in the polynomial, which is
steepest at 0 (6); the polynomial's terms, sums and coefficients 6; the exponential, its argument's rest and their product 5;
the products behind it 3: 20 together.  bfloat16 results: 2^-11 of Q, and 2^-16 of Q and phi for an exponent that is
rounded once (u^2 / 2 reaches 88, 2^-24 of it, 1.5 times, times ln 2).  Below 2^-126 the exponential may be 0: an
absolute 2^-123, since u phi(u) is up to 6 times that."""
import math

import pytest
import torch

import paper_2411_08446_amd as lsh
from test_gpu_experts import DT, HALF_STEP

pytestmark = pytest.mark.gpu

# rows of each expert: the few-row kernel (bf16 and 4 bits up to 8, binary32 up to 32), small tiles, large tiles
ROWS = {"few": 3, "small": 100, "large": 150}
E = 4


def _sweep(columns, dtype):
    """[E, columns] numbers: -14 .. 14, and magnitudes down to 2^-100 on both sides of 0."""
    n = E * columns
    line = torch.linspace(-14.0, 14.0, n - n // 8, dtype=torch.float64)
    small = torch.exp2(torch.linspace(-100.0, 0.0, n // 16, dtype=torch.float64))
    v = torch.cat([line, small, -small, torch.zeros(n - line.numel() - 2 * small.numel(), dtype=torch.float64)])
    return v[torch.randperm(n, generator=torch.Generator().manual_seed(columns))].view(E, columns).to(DT[dtype])


def _parts(v):
    u = v.double().abs()
    beyond = 0.5 * torch.special.erfc(u / math.sqrt(2.0))
    return u, beyond, torch.exp(-0.5 * u * u) / math.sqrt(2.0 * math.pi)


def _columns(rows):
    return 16384 if rows == "large" else 2048


def _offsets(rows):
    return torch.arange(0, E * ROWS[rows] + 1, ROWS[rows], dtype=torch.int32, device="cuda")


def _assert_within(got, want, bound, what):
    got = got.double().cpu().view(E, -1, want.shape[1])
    excess = (got - want[:, None, :]).abs() / bound[:, None, :]
    assert not torch.isnan(excess).any(), what
    worst = int(excess.argmax()) % want.shape[1]
    assert float(excess.max()) <= 1.0, "%s: %.3g of the bound, value %s" % (what, float(excess.max()), want[:, worst].tolist())


def _check_value(out, v, dtype):
    u, beyond, _ = _parts(v)
    want = torch.clamp(v.double(), min=0.0) - u * beyond
    before = (20 * 2.0 ** -24 if dtype == "f32" else 2.0 ** -11) * u * beyond
    _assert_within(out, want, before + HALF_STEP[dtype] * (want.abs() + before) + 2.0 ** -123, "GELU")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", list(ROWS))
def test_value(rows, dtype):
    d_in, columns, n = 16, _columns(rows), E * ROWS[rows]
    v = _sweep(columns, dtype)
    x = torch.zeros(n, d_in, dtype=DT[dtype], device="cuda")
    w = torch.zeros(E, columns, d_in, dtype=DT[dtype], device="cuda")
    out = torch.full((n, columns), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_forward(x, w, v.cuda(), _offsets(rows), out, act=lsh.LSHMOE_ACT_GELU)
    _check_value(out, v, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", list(ROWS))
def test_value_of_4_bit_products(rows, dtype):
    d_in, columns, n = 128, _columns(rows), E * ROWS[rows]
    v = _sweep(columns, dtype)
    u8 = dict(dtype=torch.uint8, device="cuda")
    out = torch.full((n, columns), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_forward_mx4(torch.zeros(n, d_in // 2, **u8), torch.zeros(n, d_in // 32, **u8), torch.zeros(E, columns, d_in // 2, **u8),
                                  torch.zeros(E, columns, d_in // 32, **u8), v.cuda(), _offsets(rows), out, act=lsh.LSHMOE_ACT_GELU)
    _check_value(out, v, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", list(ROWS))
def test_slope(rows, dtype):
    d_out, columns, n = 16, _columns(rows), E * ROWS[rows]
    v = _sweep(columns, dtype)
    g = torch.zeros(n, d_out, dtype=DT[dtype], device="cuda")
    w = torch.zeros(E, d_out, columns, dtype=DT[dtype], device="cuda")
    g[:, 5] = 1.0
    w[:, 5, :] = 1.0
    pre = v.cuda().repeat_interleave(ROWS[rows], dim=0)
    got = torch.full((n, columns), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_backward_input(g, w, _offsets(rows), got, act=lsh.LSHMOE_ACT_GELU, pre=pre)
    u, beyond, density = _parts(v)
    below = beyond - u * density                       # the slope at -u
    want = torch.where(v < 0, below, 1.0 - below)
    if dtype == "f32":
        before = 20 * 2.0 ** -24 * (beyond + u * density) + 2 * 2.0 ** -24 * want.abs()
    else:
        before = 2.0 ** -11 * beyond + 2.0 ** -16 * (beyond + u * density)
    _assert_within(got, want, before + HALF_STEP[dtype] * (want.abs() + before) + 2.0 ** -123, "slope")
