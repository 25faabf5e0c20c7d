"""The experts' products on tiles, several to a workgroup: 4-bit rows on 256 x 256 tiles with every form of their chunks, every
activation and result type; input gradients through an activation, kept values, and more tiles than a workgroup's table holds of
each product.  test_gpu_experts_large.py has the rest.

A call takes these tiles when it has more than 128 rows of buffer per expert on average and at least 256 tiles; more than 256 tiles are
several to a workgroup, more than 64 * 256 also run past a workgroup's table of tiles.  References are binary64 products on the GPU;
bounds as in test_gpu_experts.py, with GELU and its slope as in test_gpu_gelu.py."""
import math

import pytest
import torch

import paper_2411_08446_amd as lsh
from test_gpu_experts import ACT, DT, HALF_STEP, _offsets

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _large_tiles(rows, E, columns):
    return (rows // 256 + min(E, rows)) * -(-columns // 256)


def _quantized(t):
    """Codes, scales and the values that they stand for of the rows of t (its last dimension is a row's)."""
    rows, d = t.numel() // t.shape[-1], t.shape[-1]
    codes = torch.empty(rows, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, d // 32, dtype=torch.uint8, device="cuda")
    values = torch.empty(rows, d, device="cuda")
    lsh.lshmoe_mx4_quantize(t.reshape(rows, d).contiguous(), codes, scales)
    lsh.lshmoe_mx4_dequantize(codes, scales, values)
    return codes.view(*t.shape[:-1], d // 2), scales.view(*t.shape[:-1], d // 32), values.view(t.shape)


def _activated(v, act):
    if act == "relu":
        return torch.clamp(v, min=0.0)
    if act == "gelu":
        return v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
    return v


def _check_rows(out, x, w, bias, act, dtype, what):
    """out against act(x w^T + bias) of binary64 x [n, K], w [p, K], bias [p]."""
    if out.shape[0] == 0:
        return
    K = x.shape[1]
    v, size = torch.mm(x, w.t().contiguous()), torch.mm(x.abs(), w.abs().t().contiguous())
    if bias is not None:
        v, size = v + bias, size + bias.abs()
    want, before = _activated(v, act), (K + 4) * 2.0 ** -24 * size
    if act == "gelu":
        tail = 0.5 * torch.special.erfc(v.abs() / math.sqrt(2.0))
        before = 1.13 * before + v.abs() * (20 * 2.0 ** -24 * tail if dtype == "f32" else 2.0 ** -21)
    bound = before + HALF_STEP[dtype] * (want.abs() + before) + 1e-300
    assert not torch.isnan(out).any(), what
    worst = float(((out.double() - want).abs() / bound).max())
    assert worst <= 1.0, "%s: %.3g of the bound" % (what, worst)


# rows of each expert, rows behind, d_in (a half chunk, whole and half ones, one whole, whole ones), d_out
MX4 = [
    ([3001, 0, 2500, 1, 2700], 40, 128, 2200),
    ([3001, 0, 2500, 1, 2700], 40, 384, 2200),
    ([2049, 2047, 0, 4099], 0, 256, 2056),
    ([3001, 0, 2500, 1, 2700], 40, 1024, 2200),
    ([4500, 700], 5, 1152, 4104),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("counts,spare,d_in,d_out", MX4)
def test_4_bit_products(counts, spare, d_in, d_out, act, dtype):
    E, filled = len(counts), sum(counts)
    rows, off = filled + spare, _offsets(counts)
    assert rows > 128 * E and _large_tiles(rows, E, d_out) > 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d_in)
    x = torch.randn(rows, d_in, device="cuda", generator=gen)
    # blocks of different scales
    w = torch.randn(E, d_out, d_in, device="cuda", generator=gen)
    w *= torch.exp2(torch.randint(-3, 4, (E, d_out, d_in // 32), device="cuda", generator=gen).float()).repeat_interleave(32, dim=2)
    x[filled:] = NAN
    bias = torch.randn(E, d_out, device="cuda", generator=gen).to(DT[dtype])
    xc, xs, xv = _quantized(x)
    wc, ws, wv = _quantized(w)
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    out = torch.full((rows, d_out), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_forward_mx4(xc, xs, wc, ws, bias, offsets, out, act=ACT[act])
    assert (out[filled:] == 7.0).all(), "rows behind the last expert's are left alone"
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        _check_rows(out[lo:hi], xv[lo:hi].double(), wv[e].double(), bias[e].double(), act, dtype, "expert %d" % e)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_in", [128, 640])
def test_4_bit_products_of_more_tiles_than_a_workgroups_table(d_in, dtype):
    """More than 64 tiles to a workgroup: samples of the columns over all rows, samples of the rows over all columns."""
    d_out, E = 4096, 5
    counts = [120000, 0, 77777, 1, 71000]
    filled, off = sum(counts), _offsets(counts)
    rows = filled + 33
    assert _large_tiles(filled, 1, d_out) > 64 * 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d_in + 1)
    x = torch.randn(rows, d_in, device="cuda", generator=gen).to(torch.bfloat16)
    w = torch.randn(E, d_out, d_in, device="cuda", generator=gen).to(torch.bfloat16)
    x[filled:] = NAN
    bias = torch.randn(E, d_out, device="cuda", generator=gen).to(DT[dtype])
    xc, xs, xv = _quantized(x)
    wc, ws, wv = _quantized(w)
    out = torch.full((rows, d_out), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_forward_mx4(xc, xs, wc, ws, bias, torch.tensor(off, dtype=torch.int32, device="cuda"), out, act=ACT["relu"])
    assert (out[filled:] == 7.0).all()
    for e in range(E):
        for lo in range(off[e], off[e + 1], 32768):
            hi = min(lo + 32768, off[e + 1])
            for p in range(0, d_out, 256):         # of each tile's columns the first and the last ones, of both halves of waves
                at = [p, p + 1, p + 62, p + 127, p + 128, p + 200, p + 255]
                _check_rows(out[lo:hi, at], xv[lo:hi].double(), wv[e, at].double(), bias[e, at].double(), "relu", dtype,
                            "expert %d, rows from %d, columns from %d" % (e, lo, p))
        for lo in {off[e], max(off[e + 1] - 70, off[e])}:
            hi = min(lo + 70, off[e + 1])
            if lo < hi:
                _check_rows(out[lo:hi], xv[lo:hi].double(), wv[e].double(), bias[e].double(), "relu", dtype, "expert %d, rows from %d" % (e, lo))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_4_bit_products_on_small_tiles_several_to_a_workgroup(dtype):
    """At most 128 rows per expert on average: 128 x 128 tiles, more than the 512 workgroups that run at a time."""
    counts, d_in, d_out = [200, 0, 129, 1, 60, 128, 255, 90, 17, 300] * 5, 384, 1288
    E, filled, off = len(counts), sum(counts), _offsets(counts)
    rows = filled + 3
    assert rows <= 128 * E and sum(-(-n // 128) for n in counts) * -(-d_out // 128) > 512
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.randn(rows, d_in, device="cuda", generator=gen)
    w = torch.randn(E, d_out, d_in, device="cuda", generator=gen)
    x[filled:] = NAN
    bias = torch.randn(E, d_out, device="cuda", generator=gen).to(DT[dtype])
    xc, xs, xv = _quantized(x)
    wc, ws, wv = _quantized(w)
    out = torch.full((rows, d_out), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_forward_mx4(xc, xs, wc, ws, bias, torch.tensor(off, dtype=torch.int32, device="cuda"), out, act=ACT["gelu"])
    assert (out[filled:] == 7.0).all()
    for e in range(E):
        if counts[e]:
            _check_rows(out[off[e]:off[e + 1]], xv[off[e]:off[e + 1]].double(), wv[e].double(), bias[e].double(), "gelu", dtype, "expert %d" % e)


@pytest.mark.parametrize("d_in", [128, 384, 512])
@pytest.mark.parametrize("counts,d_out", [([300, 0, 77], 520), ([4000, 0, 3000], 2600)])
def test_a_4_bit_block_of_nan_on_tiles(counts, d_out, d_in):
    """Scale byte 255 in a block of the rows, at each of its places in a chunk, reaches its row only; in a block of the weights, its
    column of its expert only.  (300, 0, 77 rows: 128 x 128 tiles; 4000, 0, 3000: 256 x 256 ones.)"""
    E, off = len(counts), _offsets(counts)
    rows, blocks = off[-1], d_in // 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d_in + 7)
    xc, xs, _ = _quantized(torch.randn(rows, d_in, device="cuda", generator=gen))
    wc, ws, _ = _quantized(torch.randn(E, d_out, d_in, device="cuda", generator=gen))
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    clean = torch.full((rows, d_out), 7.0, device="cuda")
    lsh.lshmoe_expert_forward_mx4(xc, xs, wc, ws, None, offsets, clean)
    assert torch.isfinite(clean).all()
    bad_rows = {(37 * b + 11) % rows: b for b in range(blocks)}
    bad_rows[rows - 1] = blocks - 1
    bad_columns = {(53 * b + 5) % d_out: b for b in range(blocks)}
    bad_columns[d_out - 1] = blocks - 1
    for r, b in bad_rows.items():
        xs[r, b] = 255
    for c, b in bad_columns.items():
        ws[2, c, b] = 255
    got = torch.full((rows, d_out), 7.0, device="cuda")
    lsh.lshmoe_expert_forward_mx4(xc, xs, wc, ws, None, offsets, got)
    nan = torch.zeros(rows, d_out, dtype=torch.bool, device="cuda")
    nan[list(bad_rows)] = True
    nan[off[2]:, list(bad_columns)] = True
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], clean[~nan])


@pytest.mark.parametrize("act", ["relu", "gelu"])
@pytest.mark.parametrize("counts,spare,d_in,d_out", [
    ([3001, 0, 2500, 1, 2700], 40, 2200, 136),         # columns that end inside a tile; three chunks of k
    ([2049, 2047, 0, 4099], 3, 2048, 64),              # one chunk: a tile's first is its last
    ([9000, 300], 700, 4104, 520),
    ([20000, 3, 15000], 0, 1032, 72),
])
def test_input_gradients_through_an_activation(counts, spare, d_in, d_out, act):
    """The bf16 gradient through the activation of the layer below: the values kept there are read while the next tile's operands
    are on their way."""
    E, filled, off = len(counts), sum(counts), _offsets(counts)
    rows = filled + spare
    assert rows > 128 * E and _large_tiles(rows, E, d_in) > 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d_in)
    g = torch.randn(rows, d_out, device="cuda", generator=gen).to(torch.bfloat16)
    w = torch.randn(E, d_out, d_in, device="cuda", generator=gen).to(torch.bfloat16)
    pre = (2 * torch.randn(rows, d_in, device="cuda", generator=gen)).to(torch.bfloat16)
    g[filled:], pre[filled:] = NAN, NAN
    got = torch.full((rows, d_in), 7.0, dtype=torch.bfloat16, device="cuda")
    lsh.lshmoe_expert_backward_input(g, w, torch.tensor(off, dtype=torch.int32, device="cuda"), got, act=ACT[act], pre=pre)
    assert (got[filled:] == 7.0).all(), "rows behind the last expert's are left alone"
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        if lo == hi:
            continue
        ge, we, v = g[lo:hi].double(), w[e].double(), pre[lo:hi].double()
        plain, size = torch.mm(ge, we), torch.mm(ge.abs(), we.abs())
        off_by = (d_out + 4) * 2.0 ** -24 * size
        if act == "relu":
            slope = (v > 0).double()
            slope_off = torch.zeros_like(slope)
        else:
            beyond = 0.5 * torch.special.erfc(v.abs() / math.sqrt(2.0))
            density = v.abs() * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
            slope = torch.where(v < 0, beyond - density, 1.0 - (beyond - density))
            slope_off = 2.0 ** -11 * beyond + 2.0 ** -16 * (beyond + density) + 2.0 ** -123
        want = plain * slope
        before = off_by * slope.abs() + (plain.abs() + off_by) * (slope_off + 2.0 ** -24 * slope.abs())
        bound = before + HALF_STEP["bf16"] * (want.abs() + before) + 1e-300
        here = got[lo:hi].double()
        assert not torch.isnan(here).any(), "expert %d" % e
        worst = float(((here - want).abs() / bound).max())
        assert worst <= 1.0, "expert %d: %.3g of the bound" % (e, worst)


@pytest.mark.parametrize("act", ["relu", "gelu"])
@pytest.mark.parametrize("dtype,counts,d_in,d_out", [
    ("f32", [3000, 7, 0, 2500], 72, 2052),              # 128 x 128 tiles, more than 512 of them
    ("bf16", [100, 128, 3, 0, 129] * 20, 72, 2056),
])
def test_values_kept_before_the_activation_on_small_tiles(dtype, counts, d_in, d_out, act):
    E, filled, off = len(counts), sum(counts), _offsets(counts)
    rows = filled + 2
    assert (dtype == "f32" or rows <= 128 * E) and sum(-(-n // 128) for n in counts) * -(-d_out // 128) > 512
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d_out)

    def make(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(DT[dtype])
    x, w, bias = make(rows, d_in), make(E, d_out, d_in), make(E, d_out)
    x[filled:] = NAN
    out, pre = (torch.full((rows, d_out), 7.0, dtype=DT[dtype], device="cuda") for _ in range(2))
    lsh.lshmoe_expert_forward(x, w, bias, torch.tensor(off, dtype=torch.int32, device="cuda"), out, act=ACT[act], pre=pre)
    assert (out[filled:] == 7.0).all() and (pre[filled:] == 7.0).all()
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        args = x[lo:hi].double(), w[e].double(), bias[e].double()
        _check_rows(pre[lo:hi], *args, "none", dtype, "pre of expert %d" % e)
        _check_rows(out[lo:hi], *args, act, dtype, "out of expert %d" % e)


def _check_product(got, a, b, dtype, what):
    """got against a @ b of binary64."""
    want, off_by = torch.mm(a, b), (a.shape[1] + 4) * 2.0 ** -24 * torch.mm(a.abs(), b.abs())
    bound = off_by + HALF_STEP[dtype] * (want.abs() + off_by) + 1e-300
    assert not torch.isnan(got).any(), what
    worst = float(((got.double() - want).abs() / bound).max())
    assert worst <= 1.0, "%s: %.3g of the bound" % (what, worst)


@pytest.mark.parametrize("dtype,counts", [("bf16", [150000, 0, 61000, 1, 60001]), ("f32", [80000, 0, 29000, 1, 28001])])
def test_input_gradients_of_more_tiles_than_a_workgroups_table(dtype, counts):
    d_in, d_out, act = 4096, 72, "relu"
    filled, off = sum(counts), _offsets(counts)
    tile, workgroups = (256, 256) if dtype == "bf16" else (128, 512)
    assert filled // tile * (d_in // tile) > 64 * workgroups
    gen = torch.Generator(device="cuda")
    gen.manual_seed(9)

    def make(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(DT[dtype])
    g, w, pre = make(filled, d_out), make(len(counts), d_out, d_in), make(filled, d_in)
    got = torch.full((filled, d_in), 7.0, dtype=DT[dtype], device="cuda")
    lsh.lshmoe_expert_backward_input(g, w, torch.tensor(off, dtype=torch.int32, device="cuda"), got, act=ACT[act], pre=pre)
    assert ((got == 0) | (pre > 0)).all()
    for e in range(len(counts)):
        for lo in range(off[e], off[e + 1], 32768):
            hi = min(lo + 32768, off[e + 1])
            for p in range(0, d_in, tile):
                at = [p, p + 33, p + 63, p + tile // 2, p + tile - 1]
                kept = pre[lo:hi, at] > 0
                a, b = g[lo:hi].double(), w[e][:, at].double()
                want, off_by = torch.mm(a, b), (d_out + 4) * 2.0 ** -24 * torch.mm(a.abs(), b.abs())
                bound = off_by + HALF_STEP[dtype] * (want.abs() + off_by) + 1e-300
                excess = torch.where(kept, (got[lo:hi, at].double() - want).abs() / bound, torch.zeros_like(want))
                assert not torch.isnan(excess).any() and float(excess.max()) <= 1.0, "expert %d, rows from %d, columns from %d" % (e, lo, p)


@pytest.mark.parametrize("dtype,d_in,d_out,E", [("bf16", 4096, 4096, 70), ("bf16", 264, 136, 4096), ("f32", 4096, 4096, 34), ("f32", 260, 132, 4096)])
def test_weight_gradients_of_more_tiles_than_a_workgroups_table(dtype, d_in, d_out, E):
    """Many tiles of weights, and many experts of few; one expert is long (cut into parts where there are few tiles to it)."""
    gen = torch.Generator().manual_seed(E)
    counts = torch.randint(0, 12, (E,), generator=gen).tolist()
    counts[E // 3], counts[E - 1] = 3000, 1
    off = _offsets(counts)
    rows, code = off[-1], lsh.LSHMOE_F32 if dtype == "f32" else lsh.LSHMOE_BF16
    tile, workgroups = (256, 256) if dtype == "bf16" else (128, 512)
    tiles = E * -(-d_in // tile) * -(-d_out // tile)
    assert tiles > 64 * workgroups or d_in < 4096
    cuda = torch.Generator(device="cuda")
    cuda.manual_seed(E)
    g = torch.randn(rows, d_out, device="cuda", generator=cuda).to(DT[dtype])
    x = torch.randn(rows, d_in, device="cuda", generator=cuda).to(DT[dtype])
    gw = torch.full((E, d_out, d_in), 7.0, dtype=DT[dtype], device="cuda")
    gb = torch.full((E, d_out), 7.0, dtype=DT[dtype], device="cuda")
    ws = torch.full((lsh.lshmoe_expert_workspace_bytes(rows, d_in, d_out, E, code) + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    lsh.lshmoe_expert_backward_weight(g, x, torch.tensor(off, dtype=torch.int32, device="cuda"), gw, gb, ws)
    for e in sorted({0, 1, 2, 31, 32, 33, E // 3 - 1, E // 3, E // 3 + 1, E // 2, E - 2, E - 1} | set(range(0, E, max(1, E // 40)))):
        lo, hi = off[e], off[e + 1]
        if lo == hi:
            assert (gw[e] == 0.0).all() and (gb[e] == 0.0).all(), "expert %d has no rows" % e
            continue
        gt = g[lo:hi].double().t().contiguous()
        _check_product(gw[e], gt, x[lo:hi].double(), dtype, "grad_w of expert %d" % e)
        _check_product(gb[e][:, None], gt, torch.ones(hi - lo, 1, dtype=torch.float64, device="cuda"), dtype, "grad_bias of expert %d" % e)
