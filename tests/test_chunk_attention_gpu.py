"""A chunk's attention over pot and chunk (ipot_chunk_attention) against its definition in 64 bits, and its refusals.

Tolerances, per output element, with A = sum_j p_j |v_j|, X = max_j sum_c |q_c k_jc| / sqrt(d), N keys:
  logits    fp32 sums of d products, scaled:  dx <= (d + 4) 2^-23 X  (a tensor core may cut a product's sum instead of rounding it)
  weights   e^x from an fp32 logit in binary orders and an exponential good to 2^-21: dp <= p (2 dx + 2^-21), in numerator and denominator
  sums      fp32, N terms of one sign: N 2^-24
  f32       |err| <= A (4 dx + 2^-20 + 2 N 2^-24) + 2^-24 |out|
  bf16      the same + 2^-8 A (a weight rounded to bf16) + 2^-8 |out| (the result rounded)
  lse       |err| <= 2 dx + 2^-20 + N 2^-24 + 2^-22 |lse|"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2410_01518_b200 import inputs, ipot
from parity import make_pot

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(g, shape, dtype, layout, scale=1.0):
    L, B, H, n, d = shape
    if layout == "packed":    # rows of a token side by side
        return (scale * torch.randn((L, B, n, H, d), generator=g, device="cuda")).to(dtype).transpose(2, 3)
    if layout == "fused":     # queries, keys and values of a token in one array, with room between
        return (scale * torch.randn((L, B, n, H, 2 * d + 16), generator=g, device="cuda")).to(dtype)[..., 8:8 + d].transpose(2, 3)
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def reference(q, k, v, K, V, t):
    """One query head's first t rows: (out, A, X, lse) in 64 bits.  q, k, v [n][d], K, V [len][d]."""
    d, N = q.shape[1], K.shape[0]
    keys, values, q = torch.cat([K, k[:t]]).double(), torch.cat([V, v[:t]]).double(), q[:t].double()
    x = q @ keys.T / math.sqrt(d)
    seen = torch.arange(N + t, device=q.device)[None] <= N + torch.arange(t, device=q.device)[:, None]
    x = x.masked_fill(~seen, -math.inf)
    p = torch.softmax(x, dim=1)
    X = ((q.abs() @ keys.abs().T / math.sqrt(d)) * seen).amax(dim=1)
    return p @ values, p @ values.abs(), X, torch.logsumexp(x, dim=1)


def check(out, lse, ref, d, N, dtype):
    o, A, X, e = ref
    dx = (d + 4) * 2.0 ** -23 * X
    tol = A * (4 * dx + 2.0 ** -20 + 2 * N * 2.0 ** -24)[:, None] + 2.0 ** -24 * o.abs()
    if dtype == "bf16":
        tol = (tol + 2.0 ** -8 * A) * (1 + 2.0 ** -8) + 2.0 ** -8 * o.abs()
    err = (out.double() - o).abs()
    assert bool((err <= tol).all()), f"{(err / tol).max().item():.3g} of the tolerance"
    if lse is not None:
        err = (lse.double() - e).abs()
        assert bool((err <= 2 * dx + 2.0 ** -20 + N * 2.0 ** -24 + 2.0 ** -22 * e.abs()).all()), err.max().item()


class Case:
    """A pot with `len` rows, a chunk, and outputs full of a mark."""

    def __init__(self, dtype, L, B, Hq, Hkv, d, length, n, layout="dense", tokens=None, scale=1.0, seed=0, mode=None, pot_size=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = DT[dtype]
        self.dtype, self.L, self.B, self.Hq, self.Hkv, self.d, self.len, self.n = dtype, L, B, Hq, Hkv, d, length, n
        self.cfg = inputs.small_config(cfg_id=985, pot_size=pot_size or max(length, 2), keep=1, nuc_slots=0, cap_rows=1, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, layers=L, batch=B)
        self.K, self.V = (torch.randn((L, B, Hkv, length, d), generator=g, device="cuda").to(dt) for _ in range(2))
        self.q, self.k, self.v = rows(g, (L, B, Hq, n, d), dt, layout, scale), rows(g, (L, B, Hkv, n, d), dt, layout), rows(g, (L, B, Hkv, n, d), dt, layout)
        self.tokens = tokens
        if tokens is not None:
            for b, t in enumerate(tokens):   # padding may hold anything
                for x in (self.q, self.k, self.v):
                    x[:, b, :, max(t, 0):] = math.nan
        self.out = torch.full((L, B, n, Hq, d), 5.0, dtype=dt, device="cuda").transpose(2, 3) if layout != "dense" else torch.full((L, B, Hq, n, d), 5.0, dtype=dt, device="cuda")
        self.lse = torch.full((L, B, Hq, n), 5.0, device="cuda")
        self.h = make_pot(self.cfg)
        if mode == "deferred":
            ipot.ipot_set_deferred_append(self.h, True)
        if length:
            ipot.ipot_append_chunk(self.h, self.K, self.V, length)

    def run(self, layer=0, layers=None, with_lse=True):
        layers = layers or self.L
        part = slice(layer, layer + layers)
        tok = None if self.tokens is None else torch.tensor(self.tokens, dtype=torch.int32, device="cuda")
        q, k, v, out, lse = (x[part] for x in (self.q, self.k, self.v, self.out, self.lse))
        ipot.ipot_chunk_attention(self.h, layer, layers, self.n, q, k, v, out, lse if with_lse else None, tokens=tok, q_strides=q.stride()[:4], k_strides=k.stride()[:4],
                                  v_strides=v.stride()[:4], out_strides=out.stride()[:4])
        assert ipot.ipot_sync_status(self.h) == 0
        return self

    def verify(self, layers=None, heads=None, with_lse=True):
        for l in layers if layers is not None else range(self.L):
            for b in range(self.B):
                t = self.n if self.tokens is None else min(max(self.tokens[b], 0), self.n)
                for h in heads or range(self.Hq):
                    kv = h // (self.Hq // self.Hkv)
                    o, e = self.out[l, b, h], self.lse[l, b, h]
                    assert bool((o[t:] == 5).all() and (e[t if with_lse else 0:] == 5).all()), "rows behind the last token were written"
                    if t:
                        ref = reference(self.q[l, b, h], self.k[l, b, kv], self.v[l, b, kv], self.K[l, b, kv], self.V[l, b, kv], t)
                        check(o[:t], e[:t] if with_lse else None, ref, self.d, self.len + t, self.dtype)
        return self

    def close(self):
        ipot.ipot_destroy(self.h)


def run_case(*a, **kw):
    c = Case(*a, **kw)
    try:
        c.run().verify()
    finally:
        c.close()


SHAPES = [
    # L, B, Hq, Hkv, d, rows in the pot, new tokens
    (1, 1, 4, 1, 128, 0, 1), (1, 1, 4, 1, 128, 1, 1), (2, 1, 8, 2, 128, 777, 1), (1, 2, 8, 1, 64, 300, 2), (1, 1, 32, 8, 128, 4095, 1),
    (1, 1, 8, 2, 128, 0, 300), (1, 2, 4, 2, 128, 128, 128), (2, 1, 4, 2, 128, 127, 129), (1, 1, 2, 2, 128, 1000, 255), (1, 1, 6, 2, 128, 65, 77),
    (1, 1, 5, 1, 64, 333, 100), (1, 3, 12, 4, 96, 199, 33), (1, 1, 7, 1, 32, 64, 64), (1, 1, 3, 3, 40, 513, 130), (1, 1, 8, 1, 72, 100, 50),
    (1, 1, 4, 2, 256, 400, 129), (1, 1, 2, 1, 192, 30, 65), (1, 1, 16, 1, 136, 257, 19), (1, 1, 16, 1, 128, 129, 40), (1, 1, 48, 1, 64, 200, 9),
    (1, 1, 136, 1, 64, 70, 3), (1, 2, 8, 2, 128, 600, 4), (1, 1, 16, 1, 64, 100, 1), (2, 1, 5, 1, 96, 333, 3), (1, 1, 1, 1, 40, 50, 16), (1, 1, 12, 1, 256, 70, 1), (1, 1, 1, 1, 256, 1500, 1), (1, 1, 8, 8, 64, 2047, 65), (3, 2, 2, 1, 248, 5, 70),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    run_case(dtype, *shape, seed=hash(shape) % 1000)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["packed", "fused"])
@pytest.mark.parametrize("shape", [(2, 2, 8, 2, 128, 200, 150), (1, 3, 6, 2, 96, 70, 1), (1, 2, 4, 4, 40, 129, 37), (1, 1, 8, 2, 256, 100, 70)])
def test_strides(shape, layout, dtype):
    run_case(dtype, *shape, layout=layout)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,tokens", [((2, 4, 8, 2, 128, 200, 150), [150, 1, 0, 97]), ((1, 3, 4, 4, 64, 0, 300), [-7, 300, 129]), ((1, 2, 6, 2, 96, 31, 5), [9, 2]),
                                          ((1, 2, 4, 1, 256, 130, 70), [64, 3]), ((1, 3, 32, 8, 128, 500, 1), [1, 0, 1]), ((1, 2, 4, 2, 128, 64, 700), [641, 128])])
@pytest.mark.parametrize("layout", ["dense", "packed"])
def test_padded_streams(shape, tokens, layout, dtype):
    """Streams of different lengths; q, k and v are NaN behind them, and out and lse stay as they were there."""
    run_case(dtype, *shape, tokens=tokens, layout=layout)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.0, 8.0, 40.0])
@pytest.mark.parametrize("shape", [(1, 1, 4, 1, 128, 700, 200), (1, 1, 8, 1, 64, 1300, 1), (1, 1, 2, 1, 256, 300, 70)])
def test_flat_and_far_logits(shape, scale, dtype):
    """All logits equal; and logits hundreds apart, so that references move and most weights vanish."""
    run_case(dtype, *shape, scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 4, 1, 128, 1100, 140), (1, 1, 4, 1, 64, 900, 1)])
@pytest.mark.parametrize("rising", [False, True])
def test_references_that_rise_or_fall_along_the_keys(shape, rising, dtype):
    c = Case(dtype, *shape)
    try:
        L, B, Hq, Hkv, d, N, n = shape
        up = torch.linspace(0.2, 3.0, N, device="cuda") if rising else torch.linspace(3.0, 0.2, N, device="cuda")
        one = torch.randn(d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
        c.K.copy_((one * up[:, None]).to(DT[dtype]))
        c.q.copy_((one * torch.linspace(-2.0, 2.0, Hq * n, device="cuda").view(Hq, n, 1)).to(DT[dtype]))
        ipot.ipot_reset(c.h)
        ipot.ipot_append_chunk(c.h, c.K, c.V, N)
        c.run().verify()
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_layer_of_many_without_lse_and_with_a_deferred_chunk(dtype):
    c = Case(dtype, 3, 2, 4, 2, 128, 300, 70, mode="deferred", pot_size=400)
    try:
        c.run(layer=1, layers=1, with_lse=False)
        assert bool((c.out[0] == 5).all() and (c.out[2] == 5).all() and (c.lse == 5).all())
        c.verify(layers=[1], with_lse=False)
        c.run(layer=1, layers=2).verify(layers=[1, 2])
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,shape", [("bf16", (1, 1, 32, 8, 128, 2048, 2048)), ("bf16", (1, 4, 32, 8, 128, 6144, 1000)), ("bf16", (1, 1, 64, 8, 128, 16383, 3)),
                                         ("bf16", (4, 2, 8, 2, 64, 5000, 999)), ("f32", (1, 1, 8, 2, 128, 3000, 500)), ("bf16", (1, 1, 8, 2, 256, 4000, 700)),
                                         ("bf16", (32, 1, 32, 8, 128, 4095, 1))])
def test_long(dtype, shape):
    c = Case(dtype, *shape)
    try:
        c.run().verify(layers=[0, shape[0] - 1] if shape[0] > 1 else [0], heads=[0, shape[2] // 2, shape[2] - 1])
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_behind_two_to_the_31_elements(dtype, n):
    """520 units of 32768 slots of 128 channels: the last layer's rows start behind element 2^31 of the pot."""
    c = Case(dtype, 65, 1, 16, 8, 128, 200, n, pot_size=32768)
    try:
        c.run(layer=64, layers=1).verify(layers=[64], heads=[0, 15])
        assert bool((c.out[:64] == 5).all() and (c.lse[:64] == 5).all())
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_call_gives_the_same_bits(dtype):
    for shape in ((1, 1, 8, 2, 128, 4000, 1), (1, 1, 8, 2, 128, 1500, 200)):
        c = Case(dtype, *shape)
        try:
            first = c.run().out.clone()
            for _ in range(5):
                c.out.fill_(0)
                assert torch.equal(c.run().out, first)
        finally:
            c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 150), ("f32", 40)])
def test_own_stream_and_captured_calls(dtype, n):
    """On a stream of its own, captured twice (two graphs of one pot, replayed in turn) and replayed on other inputs."""
    c = Case(dtype, 1, 2, 8, 2, 128, 1000, n)
    try:
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        ipot.ipot_set_stream(c.h, s.cuda_stream)
        c.run().verify()
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        for gr in graphs:
            with torch.cuda.graph(gr, stream=s):
                ipot.ipot_set_stream(c.h, s.cuda_stream)
                ipot.ipot_chunk_attention(c.h, 0, 1, n, c.q, c.k, c.v, c.out, c.lse)
        g = torch.Generator(device="cuda").manual_seed(77)
        for i in range(4):
            c.q.copy_(torch.randn(c.q.shape, generator=g, device="cuda"))
            c.out.fill_(5)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graphs[i % 2].replay()
            s.synchronize()
            c.verify()
        del graphs, gr
    finally:
        torch.cuda.synchronize()
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_flow_equals_attention_over_rotated_rows(interleaved):
    """tables -> rotated q, k -> chunk attention over the pot's rotated copy -> append of the unrotated rows, chunk after chunk, then a
    cycle and one generated token: as a model's layer uses them together."""
    L, B, Hq, Hkv, d, size, n = 1, 2, 8, 2, 128, 384, 128
    cfg = inputs.small_config(cfg_id=986, pot_size=size, keep=100, nuc_slots=0, cap_rows=4, Hq=Hq, Hkv=Hkv, d=d, dtype="bf16", layers=L, batch=B)
    pairing = ipot.IPOT_ROPE_INTERLEAVED if interleaved else ipot.IPOT_ROPE_HALF
    g = torch.Generator(device="cuda").manual_seed(4)
    bf = torch.bfloat16
    cos, sin = (torch.empty((size + 64, d // 2), dtype=bf, device="cuda") for _ in range(2))
    ipot.ipot_rope_tables(cos, sin, 0, size + 64, d, ipot.IPOT_BF16)
    h = make_pot(cfg)
    Kr, Vr = torch.empty((L, B, Hkv, 0, d), dtype=bf, device="cuda"), torch.empty((L, B, Hkv, 0, d), dtype=bf, device="cuda")
    try:
        ipot.ipot_enable_rope(h, cos, sin, pairing)
        ipot.ipot_enable_blocks(h, 16)

        def step(m):
            nonlocal Kr, Vr
            at = Kr.shape[3]
            q, k, v = (rows(g, (L, B, x, m, d), bf, "packed", 1.5) for x in (Hq, Hkv, Hkv))
            qr, kr = torch.empty_like(q), torch.empty_like(k)
            ipot.ipot_rope_rows(h, L, m, cos, sin, size + 64, d, pairing, ipot.IPOT_BF16, first=at, q=q, q_out=qr, k=k, k_out=kr, q_strides=q.stride()[:4],
                                q_out_strides=qr.stride()[:4], k_strides=k.stride()[:4], k_out_strides=kr.stride()[:4])
            out, lse = torch.empty_like(q), torch.empty((L, B, Hq, m), device="cuda")
            ipot.ipot_chunk_attention(h, 0, L, m, qr, kr, v, out, lse, q_strides=qr.stride()[:4], k_strides=kr.stride()[:4], v_strides=v.stride()[:4],
                                      out_strides=out.stride()[:4])
            kc, vc = k.contiguous(), v.contiguous()
            ipot.ipot_append_chunk(h, kc, vc, m)
            assert ipot.ipot_sync_status(h) == 0
            for b in range(B):
                for hh in range(Hq):
                    kv = hh // (Hq // Hkv)
                    check(out[0, b, hh], lse[0, b, hh], reference(qr[0, b, hh], kr[0, b, kv], v[0, b, kv], Kr[0, b, kv], Vr[0, b, kv], m), d, at + m, "bf16")
            Kr, Vr = torch.cat([Kr, kr], 3), torch.cat([Vr, v], 3)

        for m in (n, n, 127, 1):
            step(m)
        Q = torch.randn((L, B, Hq, 4, d), generator=g, device="cuda").to(bf)
        ipot.ipot_score_and_compress(h, Q, 4, torch.zeros((B, size), device="cuda"))
        assert ipot.ipot_sync_status(h) == 0
        Kr = ipot.device_array(ipot.ipot_view_rope(h), (L, B, Hkv, size, d), "bf16")[:, :, :, :100].clone()
        Vr = ipot.device_array(ipot.ipot_view(h)[1], (L, B, Hkv, size, d), "bf16")[:, :, :, :100].clone()
        step(1)
        step(60)
        # one generated token: over the pot, over all of its blocks, over some of them.  Outputs are fp32: the head's bound for f32, and
        # weights in two bf16 terms (over the pot, 2^-16 A) or three (over blocks, 2^-22 A).
        q = torch.randn((L, B, Hq, d), generator=g, device="cuda").to(bf)
        blocks = torch.zeros((L, B, Hkv, 3), dtype=torch.int32, device="cuda")
        for kind in ("pot", "all", "some"):
            out, lse = torch.zeros((L, B, Hq, d), device="cuda"), torch.zeros((L, B, Hq), device="cuda")
            if kind == "pot":
                ipot.ipot_decode_attention(h, q, out, lse)
            else:
                ipot.ipot_decode_attention_blocks(h, 0, L, q, *((11, out, lse) if kind == "all" else (3, out, lse, blocks)))   # 161 rows
            assert ipot.ipot_sync_status(h) == 0
            for b in range(B):
                for hh in range(Hq):
                    kv = hh // (Hq // Hkv)
                    at = torch.arange(161) if kind != "some" else torch.cat([torch.arange(int(i) * 16, min(161, int(i) * 16 + 16)) for i in blocks[0, b, kv]])
                    K, V, qd = Kr[0, b, kv][at.cuda()].double(), Vr[0, b, kv][at.cuda()].double(), q[0, b, hh].double()
                    x = K @ qd / math.sqrt(d)
                    w, N = torch.softmax(x, 0), len(at)
                    dx, A = (d + 4) * 2.0 ** -23 * float((K.abs() @ qd.abs()).max()) / math.sqrt(d), w @ V.abs()
                    tol = A * (4 * dx + 2.0 ** -20 + 2 * N * 2.0 ** -24 + (2.0 ** -16 if kind == "pot" else 2.0 ** -22)) + 2.0 ** -24 * (w @ V).abs()
                    assert bool(((w @ V - out[0, b, hh]).abs() <= tol).all())
                    want = float(torch.logsumexp(x, 0))
                    assert abs(want - float(lse[0, b, hh])) <= 2 * dx + 2.0 ** -20 + N * 2.0 ** -24 + 2.0 ** -22 * abs(want)
        assert bool((blocks[..., 2] == 10).all())
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
def test_pots_on_streams_of_their_own_at_once():
    """Calls that overlap on the GPU give what they give alone: nothing is shared."""
    cases = [Case("bf16", 1, 1, 8, 2, 128, 3000, 1, seed=1), Case("bf16", 1, 1, 8, 2, 128, 3000, 60, seed=2), Case("bf16", 1, 2, 8, 2, 64, 900, 700, seed=3), Case("f32", 1, 1, 8, 2, 64, 500, 90, seed=4)]
    try:
        want = [c.run().out.clone() for c in cases]
        streams = [torch.cuda.Stream() for _ in cases]
        torch.cuda.synchronize()
        for c, s in zip(cases, streams):
            ipot.ipot_set_stream(c.h, s.cuda_stream)
            c.out.fill_(0)
        torch.cuda.synchronize()
        for _ in range(20):
            for c in cases:
                ipot.ipot_chunk_attention(c.h, 0, 1, c.n, c.q, c.k, c.v, c.out, c.lse)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert ipot.ipot_sync_status(c.h) == 0 and torch.equal(c.out, w)
    finally:
        torch.cuda.synchronize()
        for c in cases:
            c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 5, 140])
def test_inputs_that_repeat_by_a_stride_of_zero(n, dtype):
    """One chunk's keys and values for every stream, one query for every head (an expanded tensor, not a copy)."""
    c = Case(dtype, 1, 3, 8, 2, 64, 150, n)
    try:
        c.k, c.v, c.q = c.k[:, :1].expand(1, 3, 2, n, 64), c.v[:, :1].expand(1, 3, 2, n, 64), c.q[:, :, :1].expand(1, 3, 8, n, 64)
        assert c.k.stride(1) == 0 and c.q.stride(2) == 0
        c.run().verify()
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 150, 2000])
def test_large_values_do_not_overflow_on_the_way(n):
    """Values near the end of bf16's range, logits far above those of the row's first keys: weights and outputs are finite all the same."""
    c = Case("bf16", 1, 2, 8, 4, 128, 1500, n)
    try:
        c.V.mul_(2.0 ** 80)
        c.v.mul_(2.0 ** 80)
        c.K[:, :, :, 700] *= 9
        ipot.ipot_reset(c.h)
        ipot.ipot_append_chunk(c.h, c.K, c.V, 1500)
        c.run().verify(heads=[0, 5])
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 1, 4, 1, 128, 1000, 60), (1, 1, 2, 2, 64, 300, 300), (2, 4, 32, 8, 128, 500, 400), (1, 1, 4, 1, 256, 600, 100)])
@pytest.mark.parametrize("stream", [0, 1])
def test_a_wait_that_runs_out_ends_the_call_and_the_next_is_right(shape, stream):
    c = Case("bf16", *shape)
    try:
        ipot.ipot_set_tuning(c.h, ipot.IPOT_TUNE_WAIT_LIMIT_NS, 2_000_000)
        ipot.ipot_set_tuning(c.h, ipot.IPOT_TUNE_TEST_WITHHOLD_RANK, stream)
        ipot.ipot_chunk_attention(c.h, 0, shape[0], shape[6], c.q, c.k, c.v, c.out, c.lse)
        one_stream = shape[4] > 128 and stream == 1   # (wide heads have one)
        assert ipot.ipot_sync_status(c.h) == (0 if one_stream else ipot.IPOT_E_TIMEOUT)
        ipot.ipot_set_tuning(c.h, ipot.IPOT_TUNE_TEST_WITHHOLD_RANK, -1)
        ipot.ipot_set_tuning(c.h, ipot.IPOT_TUNE_WAIT_LIMIT_NS, 200_000_000)
        c.out.fill_(5)
        ipot.ipot_chunk_attention(c.h, 0, shape[0], shape[6], c.q, c.k, c.v, c.out, c.lse)
        torch.cuda.synchronize()
        c.verify(heads=[0, shape[2] - 1])
    finally:
        c.close()


@pytest.mark.gpu
def test_refusals_leave_everything_alone():
    c = Case("bf16", 2, 1, 4, 2, 64, 10, 8)
    try:
        L, st = ipot.lib(), ipot.ipot_strides_t

        def rc(h=c.h, layer=0, layers=2, n=8, tokens=None, q=c.q.data_ptr(), qs=None, k=c.k.data_ptr(), ks=None, v=c.v.data_ptr(), vs=None, out=c.out.data_ptr(), os=None, lse=None):
            by = [C.byref(st(*x)) if x else None for x in (qs, ks, vs, os)]
            return L.ipot_chunk_attention(h, layer, layers, n, tokens, q, by[0], k, by[1], v, by[2], out, by[3], lse)
        a = c.q.data_ptr()
        for kw in (dict(h=None), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=a + 8), dict(k=a + 2), dict(v=a + 4), dict(out=a + 8), dict(lse=a + 2), dict(tokens=a + 1),
                   dict(layer=-1), dict(layers=0), dict(layer=1), dict(layers=3), dict(layer=2 ** 31 - 1), dict(n=0), dict(n=-1), dict(n=1 << 30), dict(n=(1 << 29) + 1),
                   dict(qs=(2048, 2048, 512, 63)), dict(ks=(-8, 2048, 512, 64)), dict(vs=(2048, 2048, 4, 64)), dict(os=(1 << 41, 2048, 512, 64))):
            assert rc(**kw) == ipot.IPOT_E_INVALID, kw
        torch.cuda.synchronize()
        assert bool((c.out == 5).all()) and ipot.ipot_sync_status(c.h) == 0
        assert rc() == 0
    finally:
        c.close()


def test_refusals_without_a_pot():
    assert ipot.lib().ipot_chunk_attention(None, 0, 1, 1, None, 16, None, 16, None, 16, None, 16, None, None) == ipot.IPOT_E_INVALID
    assert ipot.lib().ipot_rope_rows(None, None, 1, 1, None, 0, 16, None, 16, None, None, None, None, None) == ipot.IPOT_E_INVALID
