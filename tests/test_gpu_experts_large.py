"""The experts' products where their kernels change their ways: many tiles to a workgroup, experts cut into parts, more than 64
experts, offsets beyond 32 bits, and each kernel's first and last sizes.  The reference is a binary64 product on the GPU, of samples
where the whole would be large; bounds as in test_gpu_experts.py."""
import numpy as np
import pytest
import torch

import paper_2411_08446_amd as lsh
from test_gpu_experts import ACT, DT, HALF_STEP, _code, _offsets, _workspace

pytestmark = pytest.mark.gpu


def _check(got, a, b, K, dtype, what, add=None):
    """got against a @ b (+ add) of K terms in binary64."""
    want, size = torch.mm(a, b), torch.mm(a.abs(), b.abs())
    if add is not None:
        want, size = want + add, size + add.abs()
    bound = (K + 4) * 2.0 ** -24 * size
    bound = bound + HALF_STEP[dtype] * (want.abs() + bound) + 1e-300
    got = got.double()
    assert not torch.isnan(got).any(), what
    worst = float(((got - want).abs() / bound).max()) if got.numel() else 0.0
    assert worst <= 1.0, "%s: %.3g of the bound" % (what, worst)


def _make(counts, spare, d_in, d_out, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, E = sum(counts) + spare, len(counts)

    def t(*shape):
        return torch.randn(*shape, device="cuda", generator=gen).to(DT[dtype])
    x, g, w, b = t(rows, d_in), t(rows, d_out), t(E, d_out, d_in), t(E, d_out)
    x[sum(counts):] = float("nan")
    g[sum(counts):] = float("nan")
    return rows, E, x, g, w, b, torch.tensor(_offsets(counts), dtype=torch.int32, device="cuda")


def _blank(*shape, dtype):
    return torch.full(shape, 7.0, dtype=DT[dtype], device="cuda")


def _all_three(counts, spare, d_in, d_out, dtype, seed, experts=None):
    rows, E, x, g, w, b, off = _make(counts, spare, d_in, d_out, dtype, seed)
    out, gx = _blank(rows, d_out, dtype=dtype), _blank(rows, d_in, dtype=dtype)
    gw, gb = _blank(E, d_out, d_in, dtype=dtype), _blank(E, d_out, dtype=dtype)
    lsh.lshmoe_expert_forward(x, w, b, off, out)
    lsh.lshmoe_expert_backward_input(g, w, off, gx)
    lsh.lshmoe_expert_backward_weight(g, x, off, gw, gb, _workspace(rows, d_in, d_out, E, dtype))
    o = _offsets(counts)
    assert (out[o[-1]:] == 7.0).all() and (gx[o[-1]:] == 7.0).all()
    for e in range(E) if experts is None else experts:
        lo, hi = o[e], o[e + 1]
        xe, ge, we = x[lo:hi].double(), g[lo:hi].double(), w[e].double()
        _check(out[lo:hi], xe, we.t().contiguous(), d_in, dtype, "out of expert %d" % e, b[e].double())
        _check(gx[lo:hi], ge, we, d_out, dtype, "grad_x of expert %d" % e)
        _check(gw[e], ge.t().contiguous(), xe, hi - lo, dtype, "grad_w of expert %d" % e)
        _check(gb[e][:, None], ge.t().contiguous(), torch.ones(hi - lo, 1, dtype=torch.float64, device="cuda"), hi - lo, dtype,
               "grad_bias of expert %d" % e)
    return gw, gb


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts,spare,d_in,d_out", [
    # parts of experts: one that has nearly everything, one row of an expert, none, sizes about a part's
    ([9000, 0, 1, 700], 100, 264, 136),
    ([511, 512, 513, 536, 537, 538, 1025, 1100], 0, 128, 256),
    ([5000], 3, 72, 520),
    ([0, 0, 6000, 0], 0, 512, 512),
    ([300] * 3 + [20000] + [10] * 4, 0, 256, 256),
])
def test_experts_in_parts(counts, spare, d_in, d_out, dtype):
    _all_three(counts, spare, d_in, d_out, dtype, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("experts,each", [(65, 140), (130, 131), (200, 3), (1000, 5)])
def test_more_experts_than_lanes(experts, each, dtype):
    rng = np.random.default_rng(experts)
    counts = rng.integers(0, 2 * each, experts).tolist()
    _all_three(counts, 5, 136, 264, dtype, 2, experts=list(range(0, experts, 7)) + [63, 64, experts - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("each", [7, 8, 9, 31, 32, 33, 127, 128, 129])
def test_both_sides_of_the_rules(each, dtype):
    """Rows per expert at which another kernel takes over, on few and on many columns."""
    for d_in, d_out, E in ((64, 72, 6), (136, 2056, 3)):
        _all_three([each] * E, 0, d_in, d_out, dtype, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d_in", [8, 72, 136, 200])
def test_many_tiles_to_a_workgroup(d_in, dtype):
    """More than 64 tiles to a workgroup: with one, two, three and four chunks of k to a tile."""
    d_out = 4096
    big = dtype == "bf16"
    tiles, block = 256 * 66, 256
    if not big:
        tiles, block = 512 * 66, 128
    rows = tiles // (d_out // block) * block
    counts = [rows // 2 + 3, 0, rows - rows // 2 - 40, 1]
    rows, E, x, g, w, b, off = _make(counts, 30, d_in, d_out, dtype, 5)
    out = _blank(rows, d_out, dtype=dtype)
    lsh.lshmoe_expert_forward(x, w, b, off, out)
    o = _offsets(counts)
    assert (out[o[-1]:] == 7.0).all()
    for e in range(E):
        for lo in range(o[e], o[e + 1], 16384):
            hi = min(lo + 16384, o[e + 1])
            _check(out[lo:hi], x[lo:hi].double(), w[e].double().t().contiguous(), d_in, dtype, "rows from %d" % lo, b[e].double())


@pytest.mark.parametrize("act", ["relu", "gelu"])
def test_values_kept_before_the_activation_over_many_tiles(act):
    """Two results a tile, more tiles than workgroups: every store has landed where it should."""
    counts, d_in, d_out = [20000, 3, 15000], 136, 2056
    rows, E, x, g, w, b, off = _make(counts, 0, d_in, d_out, "bf16", 6)
    out, pre = _blank(rows, d_out, dtype="bf16"), _blank(rows, d_out, dtype="bf16")
    lsh.lshmoe_expert_forward(x, w, b, off, out, act=ACT[act], pre=pre)
    o = _offsets(counts)
    for e in range(E):
        _check(pre[o[e]:o[e + 1]], x[o[e]:o[e + 1]].double(), w[e].double().t().contiguous(), d_in, "bf16", "pre", b[e].double())
    # out and pre are rounded from one binary32 value: out lies between the activation of pre's neighbours, whose distance is a
    # bf16 step (2^-7 of the value), times the steepest slope, plus out's own half step
    v = pre.double()
    want = torch.clamp(v, min=0.0) if act == "relu" else v * torch.special.ndtr(v)
    bound = 1.13 * 2.0 ** -8 * v.abs() + 2.0 ** -8 * (want.abs() + 1.13 * 2.0 ** -8 * v.abs()) + v.abs() * 2.0 ** -21
    assert bool(((out.double() - want).abs() <= bound).all())


def test_rows_beyond_32_bits():
    """Rows, results and their gradients of more than 4 GiB, one expert's rows of more than 2: the last rows of each expert."""
    counts, d_in, d_out = [300001, 0, 320000], 4096, 264
    rows, E, x, g, w, b, off = _make(counts, 7, d_in, d_out, "bf16", 7)
    out, gx = _blank(rows, d_out, dtype="bf16"), _blank(rows, d_in, dtype="bf16")
    gw, gb = _blank(E, d_out, d_in, dtype="bf16"), _blank(E, d_out, dtype="bf16")
    lsh.lshmoe_expert_forward(x, w, b, off, out)
    lsh.lshmoe_expert_backward_input(g, w, off, gx)
    lsh.lshmoe_expert_backward_weight(g, x, off, gw, gb, _workspace(rows, d_in, d_out, E, "bf16"))
    o = _offsets(counts)
    assert (out[o[-1]:] == 7.0).all() and (gx[o[-1]:] == 7.0).all()
    for e in (0, 2):
        for lo, hi in ((o[e], o[e] + 300), (o[e + 1] - 300, o[e + 1])):
            _check(out[lo:hi], x[lo:hi].double(), w[e].double().t().contiguous(), d_in, "bf16", "out", b[e].double())
            _check(gx[lo:hi], g[lo:hi].double(), w[e].double(), d_out, "bf16", "grad_x")
        part = x[o[e]:o[e + 1], :64].double()
        _check(gw[e][:, :64], g[o[e]:o[e + 1]].double().t().contiguous(), part, counts[e], "bf16", "grad_w")
    assert (gw[1] == 0.0).all() and (gb[1] == 0.0).all()


def test_sums_over_more_than_a_gibibyte_of_rows():
    """One expert, uncut, whose rows' offsets pass 2^30 within a tile's sum: the descriptors move on."""
    counts, d_in, d_out = [150000], 4096, 4096
    rows, E, x, g, w, b, off = _make(counts, 0, d_in, d_out, "bf16", 8)
    gw = _blank(E, d_out, d_in, dtype="bf16")
    lsh.lshmoe_expert_backward_weight(g, x, off, gw, None, _workspace(rows, d_in, d_out, E, "bf16"))
    for p, q in ((0, 0), (4032, 4032), (2000, 1000)):
        _check(gw[0][q:q + 64, p:p + 64], g[:, q:q + 64].double().t().contiguous(), x[:, p:p + 64].double(), rows, "bf16", "grad_w")


def test_weights_of_more_than_a_gibibyte():
    counts, d_in, d_out = [300], 32768, 24576
    rows, E, x, g, w, b, off = _make(counts, 0, d_in, d_out, "bf16", 9)
    gx, out = _blank(rows, d_in, dtype="bf16"), _blank(rows, d_out, dtype="bf16")
    lsh.lshmoe_expert_backward_input(g, w, off, gx)
    lsh.lshmoe_expert_forward(x, w, b, off, out)
    for p in (0, 32704):
        _check(gx[:, p:p + 64], g.double(), w[0][:, p:p + 64].double(), d_out, "bf16", "grad_x")
    for p in (0, 24512):
        _check(out[:, p:p + 64], x.double(), w[0][p:p + 64].double().t().contiguous(), d_in, "bf16", "out", b[0][p:p + 64].double())


def test_two_parts_at_once_on_two_streams():
    """Cut experts' partial sums lie in the caller's workspace: two calls that overlap, a workspace each, ten times."""
    counts, d_in, d_out = [9000, 10, 3000], 264, 136
    rows, E, x, g, w, b, off = _make(counts, 0, d_in, d_out, "bf16", 10)
    ws = [_workspace(rows, d_in, d_out, E, "bf16") for _ in range(2)]
    alone = (_blank(E, d_out, d_in, dtype="bf16"), _blank(E, d_out, dtype="bf16"))
    lsh.lshmoe_expert_backward_weight(g, x, off, *alone, ws[0])
    outs = [(_blank(E, d_out, d_in, dtype="bf16"), _blank(E, d_out, dtype="bf16")) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, t, o in zip(streams, ws, outs):
            lsh.lshmoe_expert_backward_weight(g, x, off, *o, t, stream=s)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o[0], alone[0]) and torch.equal(o[1], alone[1])


def test_the_workspace_ends_where_it_says():
    """Bytes behind the workspace's size stay as they were, at sizes that use nearly all of it."""
    for counts, d_in, d_out, dtype in (([4000, 300], 520, 264, "bf16"), ([131072], 256, 256, "bf16"), ([2000, 1100], 136, 72, "f32")):
        rows, E, x, g, w, b, off = _make(counts, 0, d_in, d_out, dtype, 11)
        need = lsh.lshmoe_expert_workspace_bytes(rows, d_in, d_out, E, _code(dtype))
        ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        assert ws.data_ptr() % 256 == 0
        gw, gb = _blank(E, d_out, d_in, dtype=dtype), _blank(E, d_out, dtype=dtype)
        lsh.lshmoe_expert_backward_weight(g, x, off, gw, gb, ws[:need])
        assert bool((ws[need:] == 0xA5).all())


@pytest.mark.parametrize("d_in,d_out,dtype", [(4096, 4096, "bf16"), (4104, 4120, "bf16"), (4096, 8200, "f32")])
def test_weights_of_many_tiles_need_no_workspace(d_in, d_out, dtype):
    """As many tiles of an expert as workgroups: no expert is cut, whatever its rows."""
    counts = [1500, 0, 20]
    assert lsh.lshmoe_expert_workspace_bytes(sum(counts), d_in, d_out, len(counts), _code(dtype)) == 0
    assert lsh.lshmoe_expert_workspace_bytes(1 << 20, d_in, d_out, len(counts), _code(dtype)) == 0
    rows, E, x, g, w, b, off = _make(counts, 5, d_in, d_out, dtype, 15)
    gw = _blank(E, d_out, d_in, dtype=dtype)
    lsh.lshmoe_expert_backward_weight(g, x, off, gw, None, torch.empty(0, dtype=torch.uint8, device="cuda"))
    o = _offsets(counts)
    for e in range(E):
        lo, hi = o[e], o[e + 1]
        _check(gw[e], g[lo:hi].double().t().contiguous(), x[lo:hi].double(), hi - lo, dtype, "grad_w of expert %d" % e)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_longest_rows(dtype):
    """Rows of 16 bytes less than 8 MiB, more than 2 GiB of them to an expert, as d_in of the forward product and the weight gradient
    and as d_out of the input gradient; on tiles and (the second call, with few rows) without."""
    piece = 8 if dtype == "bf16" else 4
    d = (8 << 20) * piece // 16 - piece
    for counts in ([300, 7], [5, 2]):
        rows, E, long, short, w, b, off = _make(counts, 2, d, piece, dtype, 16)      # long [rows, d], short [rows, piece], w [E, piece, d]
        o = _offsets(counts)
        out, gw, gx = _blank(rows, piece, dtype=dtype), _blank(E, piece, d, dtype=dtype), _blank(rows, piece, dtype=dtype)
        wt = w.transpose(1, 2).contiguous()                                         # [E, d, piece]: from `piece` to d columns
        lsh.lshmoe_expert_forward(long, w, b, off, out)
        lsh.lshmoe_expert_backward_input(long, wt, off, gx)
        lsh.lshmoe_expert_backward_weight(short, long, off, gw, None, _workspace(rows, d, piece, E, dtype))
        assert (out[o[-1]:] == 7.0).all() and (gx[o[-1]:] == 7.0).all()
        for e in range(E):
            lo, hi = o[e], o[e + 1]
            xe, we = long[lo:hi].double(), wt[e].double()
            _check(out[lo:hi], xe, we, d, dtype, "out of expert %d" % e, b[e].double())
            _check(gx[lo:hi], xe, we, d, dtype, "grad_x of expert %d" % e)
            _check(gw[e], short[lo:hi].double().t().contiguous(), xe, hi - lo, dtype, "grad_w of expert %d" % e)
            del xe, we


def test_as_many_experts_as_there_may_be():
    """4096 experts of 0 to 40 rows, most of the sizes at once."""
    gen = torch.Generator().manual_seed(17)
    counts = torch.randint(0, 41, (4096,), generator=gen).tolist()
    _all_three(counts, 3, 64, 40, "bf16", 18, experts=[0, 1, 63, 64, 65, 2047, 2048, 4094, 4095])


@pytest.mark.parametrize("d_in", [128, 160, 256, 384, 1024])
def test_mx4_over_tiles_and_beside_them(d_in):
    """Whole and half chunks of 4-bit numbers, and rows that the tiles do not take (160)."""
    counts, d_out = [700, 0, 1500, 3], 520
    rows, E, x, g, w, b, off = _make(counts, 9, d_in, d_out, "bf16", 12)
    u8 = dict(dtype=torch.uint8, device="cuda")
    xc, xs, wc, wsc = (torch.empty(rows, d_in // 2, **u8), torch.empty(rows, d_in // 32, **u8),
                       torch.empty(E, d_out, d_in // 2, **u8), torch.empty(E, d_out, d_in // 32, **u8))
    lsh.lshmoe_mx4_quantize(x, xc, xs)
    lsh.lshmoe_mx4_quantize(w.view(E * d_out, d_in), wc.view(E * d_out, -1), wsc.view(E * d_out, -1))
    x4, w4 = torch.empty(rows, d_in, device="cuda"), torch.empty(E * d_out, d_in, device="cuda")
    lsh.lshmoe_mx4_dequantize(xc, xs, x4)
    lsh.lshmoe_mx4_dequantize(wc.view(E * d_out, -1), wsc.view(E * d_out, -1), w4)
    w4 = w4.view(E, d_out, d_in)
    o = _offsets(counts)
    for dtype in ("bf16", "f32"):
        out = _blank(rows, d_out, dtype=dtype)
        bias = b.to(DT[dtype])
        lsh.lshmoe_expert_forward_mx4(xc, xs, wc, wsc, bias, off, out)
        assert (out[o[-1]:] == 7.0).all()
        for e in range(E):
            _check(out[o[e]:o[e + 1]], x4[o[e]:o[e + 1]].double(), w4[e].double().t().contiguous(), d_in, dtype, "expert %d" % e,
                   bias[e].double())
