"""A layer as it is served: gate, choice, compression, the experts in 4 bits on the centroids it leaves, restoration.  Each operator
against the oracle on what the one before it left, then the whole in a replayed graph against eager calls."""
import numpy as np
import pytest
import torch

import oracle
import paper_2411_08446_amd as lsh
from test_gpu_experts import DT, HALF_STEP, _assert_within, _gate_bounds, _rounded, _wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,h", [(5, 128, 96), (300, 256, 384), (2500, 160, 512)])
def test_layer_in_4_bits(T, d, h, dtype):
    """d = 256 goes over tiles, 160 and 96 are no whole 128 numbers; 5 tokens are a decoding batch."""
    k, E, L, r, dt = 2, 6, 2, 8, DT[dtype]
    N = T * k
    gen = torch.Generator().manual_seed(T)
    centers = torch.randn(40, d, generator=gen)

    def tokens():
        return (centers[torch.randint(40, (T,), generator=gen)] + 0.05 * torch.randn(T, d, generator=gen)).to(dt).cuda()
    x = tokens()
    rot, gate_w = torch.randn(L, r, d, generator=gen).to(dt).cuda(), (torch.randn(E, d, generator=gen) / 16).to(dt).cuda()
    b1, b2 = torch.randn(E, h, generator=gen).to(dt).cuda(), torch.randn(E, d, generator=gen).to(dt).cuda()
    u8 = dict(dtype=torch.uint8, device="cuda")

    def room(*shape):
        return torch.full((*shape[:-1], shape[-1] // 2), 0xEE, **u8), torch.full((*shape[:-1], shape[-1] // 32), 0xEE, **u8)

    def weights(out, into):                      # quantised once, in front of the layer
        w = (torch.randn(E, out, into, generator=gen) / into ** 0.5).to(dt).cuda()
        codes, scales = room(E, out, into)
        lsh.lshmoe_mx4_quantize(w.view(E * out, into), codes.view(E * out, -1), scales.view(E * out, -1))
        return codes, scales
    w1, w2 = weights(h, d), weights(d, h)
    bucket = torch.empty(T, dtype=torch.int64, device="cuda")
    logits = torch.empty(T, E, device="cuda")
    expert, weight = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    o = lsh.CompressOutputs.allocate(T, d, k, E, L, r, dt)
    o.centroids.fill_(float("nan"))              # the rows that the compression leaves are quantised with the others
    c4, h4 = room(N, d), room(N, h)
    hid, eo, y = (torch.full((N, n), 7.0, dtype=dt, device="cuda") for n in (h, d, d))
    y = y[:T]

    fused_gate = d * x.element_size() % 512 == 0      # what lshmoe_hash_gate takes; otherwise the projection is the caller's

    def project():
        if not fused_gate:
            logits.copy_(x.float() @ gate_w.float().t())

    def step():
        if fused_gate:
            lsh.lshmoe_hash_gate(x, rot, gate_w, bucket, logits)
        else:
            lsh.lshmoe_hash(x, rot, bucket)
        lsh.lshmoe_gate_topk(logits, expert, weight)
        lsh.lshmoe_compress(x, expert, bucket, E, L, r, o)
        lsh.lshmoe_mx4_quantize(o.centroids, *c4)
        lsh.lshmoe_expert_forward_mx4(*c4, *w1, b1, o.expert_offsets, hid, act=lsh.LSHMOE_ACT_GELU)
        lsh.lshmoe_mx4_quantize(hid, *h4)
        lsh.lshmoe_expert_forward_mx4(*h4, *w2, b2, o.expert_offsets, eo)
        lsh.lshmoe_decompress_combine(x, o.centroids, eo, o.seg_of, o.seg_offsets, weight, y)

    project()
    step()
    torch.cuda.synchronize()
    S, off = int(o.num_segments.item()), o.expert_offsets.tolist()
    assert 0 < S <= N and off[-1] == S
    ids, want = oracle.gate_topk_ref(_wide(logits), k, False)
    assert np.array_equal(expert.cpu().numpy(), ids)
    _assert_within(weight, want, _gate_bounds(_wide(logits), ids, want, False) * want, "weights")
    for codes, scales, rows, (wc, ws), bias, act, out, what in ((*c4, o.centroids, w1, b1, "gelu", hid, "hidden"),
                                                               (*h4, hid, w2, b2, "none", eo, "expert output")):
        ref_codes, ref_scales = oracle.mx4_quantize_ref(_wide(rows[:S]))
        assert np.array_equal(codes[:S].cpu().numpy(), ref_codes) and np.array_equal(scales[:S].cpu().numpy(), ref_scales), what
        pre, want, size = oracle.expert_forward_ref(oracle.mx4_values_ref(ref_codes, ref_scales),
                                                    oracle.mx4_values_ref(wc.cpu().numpy(), ws.cpu().numpy()), _wide(bias), off, act)
        K, extra = 2 * codes.shape[1], np.abs(pre) * 2.0 ** -21 if act == "gelu" else 0.0
        _assert_within(out[:S], want, _rounded(size, K, dtype, want, 1.13 if act == "gelu" else 1.0, extra), what)
        assert (out[S:] == 7.0).all()
    # the sum over a token's experts of w (its cluster's output + the residual, x less the centroid)
    seg, w = o.seg_of.view(T, k).long().cpu().numpy(), _wide(weight)
    e, c, xs = _wide(eo[:S]), _wide(o.centroids[:S]), _wide(x)
    parts = np.stack([e[seg[:, j]] + (xs - c[seg[:, j]]) for j in range(k)], axis=1)
    size = np.stack([np.abs(e[seg[:, j]]) + np.abs(xs) + np.abs(c[seg[:, j]]) for j in range(k)], axis=1)
    want = (w[:, :, None] * parts).sum(axis=1)
    off_by = (w[:, :, None] * size).sum(axis=1)
    # k terms of two subtractions and a product each, summed in binary32 and rounded once
    off_by *= (4 * k + 4) * 2.0 ** -24
    _assert_within(y, want, off_by + HALF_STEP[dtype] * (np.abs(want) + off_by), "layer")

    outs = (weight, hid, eo, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.copy_(tokens())
        project()
        for t in outs:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.fill_(7.0)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b), "a replay gives what the eager step gives, bit for bit"
