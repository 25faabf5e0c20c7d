"""The router and the 4-bit rows where arrays pass 2^32 elements or bytes: samples at both ends and around the border."""
import pytest
import torch

import paper_2411_08446_amd as lsh

pytestmark = pytest.mark.gpu


def _samples(rows, each, unit):
    """Rows at both ends and on both sides of where offsets of `unit` per row pass 2^31 and 2^32."""
    at = {0, rows - 1} | {b // unit + i for b in (1 << 31, 1 << 32) for i in (-1, 0, 1)}
    at |= set(torch.randint(rows, (each,), generator=torch.Generator().manual_seed(unit)).tolist())
    return torch.tensor(sorted(r for r in at if 0 <= r < rows), device="cuda")


@pytest.mark.parametrize("E", [512, 513])
def test_router(E):
    T, k = (1 << 32) // E + 70001, 3
    logits = torch.empty(T, E, device="cuda")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(E)
    for lo in range(0, T, 1 << 20):
        logits[lo:lo + (1 << 20)].normal_(generator=gen)
    ids, w = torch.full((T, k), -7, dtype=torch.int32, device="cuda"), torch.full((T, k), float("nan"), device="cuda")
    flags = lsh.LSHMOE_FLAG_GATE_FULL_SOFTMAX
    lsh.lshmoe_gate_topk(logits, ids, w, flags=flags)
    assert bool((ids >= 0).all()) and not bool(torch.isnan(w).any())
    at = _samples(T, 3000, E)
    l = logits[at].double()
    p = torch.softmax(l, dim=1)
    assert torch.equal(ids[at].long(), torch.topk(l, k, dim=1).indices)         # random binary32 numbers: hardly two alike in a row
    want = p.gather(1, ids[at].long())
    # exponentials of differences below 16 (their rounding and 2 units), a sum of E terms, a division
    rel = (2 * 16 + E + 12) * 2.0 ** -24
    assert bool(((w[at].double() - want).abs() <= rel * want).all())
    g = torch.randn(T, k, device="cuda", generator=gen)
    out = torch.full((T, E), float("nan"), device="cuda")
    lsh.lshmoe_gate_topk_backward(logits, ids, w, g, out, flags=flags)
    assert not bool(torch.isnan(out[-100000:]).any())
    full = torch.zeros_like(l).scatter_(1, ids[at].long(), g[at].double())
    want = p * (full - (p * full).sum(dim=1, keepdim=True))
    size = 2 * g[at].double().abs().amax(dim=1, keepdim=True)
    assert bool(((out[at].double() - want).abs() <= p * size * (2 * rel + (k + 4) * 2.0 ** -24)).all())


def _plain(x):
    """Scales and values of rows in blocks of 32, by distance to each of the eight magnitudes (ties to the even code)."""
    b = x.double().reshape(x.shape[0], -1, 32)
    s = (torch.frexp(b.abs().amax(dim=2, keepdim=True)).exponent - 3).clamp(min=-127)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    odd = torch.arange(8, device=x.device) % 2
    away = (torch.ldexp(b, -s).abs()[..., None] - grid).abs()
    pick = (away + odd * 2.0 ** -40).argmin(dim=-1)           # numbers of 8 or 24 bits differ by more where they differ
    return (s[:, :, 0] + 127).to(torch.uint8), torch.ldexp(torch.copysign(grid[pick], b), s).reshape(x.shape)


@pytest.mark.parametrize("d_in,d_out", [(4096, 40), (4128, 40)])
def test_4_bit_rows_and_their_product(d_in, d_out):
    """Rows of 17 GiB, their codes of more than 4; d_in = 4128 is no whole 128 numbers."""
    E = 3
    rows = (1 << 33) // d_in + 5003
    counts = [rows // 2 - 17, 0, rows - rows // 2]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(d_in)
    x = torch.empty(rows, d_in, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, rows, 1 << 17):
        x[lo:lo + (1 << 17)].normal_(generator=gen)
    u8 = dict(dtype=torch.uint8, device="cuda")
    codes, scales = torch.full((rows, d_in // 2), 0xEE, **u8), torch.full((rows, d_in // 32), 0xEE, **u8)
    lsh.lshmoe_mx4_quantize(x, codes, scales)
    at = _samples(rows, 500, d_in // 2)
    s, values = _plain(x[at])
    assert torch.equal(scales[at], s)
    back = torch.full((rows, d_in), 7.0, dtype=torch.bfloat16, device="cuda")
    lsh.lshmoe_mx4_dequantize(codes, scales, back)
    for rows_at in (at, _samples(rows, 500, d_in)):
        assert torch.equal(back[rows_at].double(), _plain(x[rows_at])[1])
    del back
    w = torch.randn(E, d_out, d_in, device="cuda", generator=gen)
    wc, ws, wv = torch.empty(E, d_out, d_in // 2, **u8), torch.empty(E, d_out, d_in // 32, **u8), torch.empty(E, d_out, d_in, device="cuda")
    lsh.lshmoe_mx4_quantize(w.view(E * d_out, d_in), wc.view(E * d_out, -1), ws.view(E * d_out, -1))
    lsh.lshmoe_mx4_dequantize(wc.view(E * d_out, -1), ws.view(E * d_out, -1), wv.view(E * d_out, -1))
    out = torch.full((rows, d_out), 7.0, device="cuda")
    off = [0, counts[0], counts[0], counts[0] + counts[2]]
    assert off[-1] == rows - 17
    lsh.lshmoe_expert_forward_mx4(codes, scales, wc, ws, None, torch.tensor(off, dtype=torch.int32, device="cuda"), out)
    assert (out[off[-1]:] == 7.0).all() and not torch.isnan(out).any()
    edges = torch.tensor([off[1] - 1, off[1], off[-1] - 1], device="cuda")
    for r in (at[at < off[-1]], edges):
        _, v = _plain(x[r])
        for e, mine in ((0, r < off[1]), (2, r >= off[1])):
            a, b = v[mine], wv[e].double().t().contiguous()
            if a.shape[0] == 0:
                continue
            want, size = torch.mm(a, b), torch.mm(a.abs(), b.abs())
            bound = ((d_in + 4) * 2.0 ** -24 * size) + 2.0 ** -24 * want.abs()
            assert bool(((out[r[mine]].double() - want).abs() <= bound).all()), "expert %d" % e
