"""Bounds of the keys' channels over blocks of slots and generation over the blocks that they select (ipot_enable_blocks,
ipot_view_blocks, ipot_decode_attention_blocks) against their definitions in 64 bits, and refusals.

Bounds and lists are compared for equality (scores are sums in 64 bits on both sides; inputs are random, so that no two scores agree to
64-bit rounding but where a test makes ties, whose scores are exact).  Outputs, as in test_chunk_attention_gpu.py, all in fp32:
|err| <= A (4 dx + 2^-20 + 2 N 2^-24) + 2^-24 |out| with A = sum_j p_j |v_j|, dx = (d + 4) 2^-23 max_j sum_c |q_c k_jc| / sqrt(d), and for bf16 pots
2^-22 A more (weights enter their product with three bf16 terms, 24 bits); lse: 2 dx + 2^-20 + N 2^-24 + 2^-22 |lse|."""
import math

import numpy as np
import pytest
import torch

from paper_2410_01518_b200 import inputs, ipot
from parity import make_pot

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def config(dtype, L, B, Hq, Hkv, d, size, keep=1, cap_rows=1):
    return inputs.small_config(cfg_id=987, pot_size=size, keep=keep, nuc_slots=0, cap_rows=cap_rows, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, layers=L, batch=B)


def pot_rows(h, cfg, n, rope=False):
    """The keys that are attended to, and the values."""
    shape = (cfg.layers, cfg.batch, cfg.Hkv, cfg.pot_size, cfg.d)
    K, V, at = ipot.ipot_view(h)
    assert at == n
    K = ipot.ipot_view_rope(h) if rope else K
    return tuple(ipot.device_array(x, shape, cfg.dtype)[:, :, :, :n].clone() for x in (K, V))


def check_bounds(h, cfg, K, R):
    lo, hi, used = ipot.ipot_view_blocks(h)
    n = K.shape[3]
    assert used == -(-n // R)
    shape = (cfg.layers, cfg.batch, cfg.Hkv, -(-cfg.pot_size // R), cfg.d)
    got = [ipot.device_array(x, shape, cfg.dtype)[:, :, :, :used].float() for x in (lo, hi)]
    for b in range(used):
        part = K[:, :, :, b * R:(b + 1) * R].float()
        assert torch.equal(got[0][:, :, :, b], part.amin(dim=3)) and torch.equal(got[1][:, :, :, b], part.amax(dim=3)), b


def chosen(q, K, R, n_blocks):
    """[G, d], [n, d] -> the ascending list, in numpy's float64, block by block."""
    q, K = q.double().cpu().numpy(), K.double().cpu().numpy()
    total = -(-len(K) // R)
    s = []
    for b in range(total - 1):
        part = K[b * R:(b + 1) * R]
        lo, hi = part.min(axis=0), part.max(axis=0)
        s.append(float(np.maximum(q * lo, q * hi).sum()))
    best = sorted(range(total - 1), key=lambda b: (-s[b], b))[:n_blocks - 1]
    return sorted(best + [total - 1])


def verify(cfg, q, K, V, R, n_blocks, out, lse, blocks, layers=None):
    G, n = cfg.Hq // cfg.Hkv, K.shape[3]
    for l in range(q.shape[0]) if layers is None else layers:
        for b in range(cfg.batch):
            for kv in range(cfg.Hkv):
                heads = slice(kv * G, (kv + 1) * G)
                want = chosen(q[l, b, heads], K[l, b, kv], R, n_blocks)
                assert blocks[l, b, kv].tolist() == want + [-1] * (n_blocks - len(want))
                at = torch.cat([torch.arange(i * R, min(n, (i + 1) * R)) for i in want]).cuda()
                k, v, x = K[l, b, kv][at].double(), V[l, b, kv][at].double(), q[l, b, heads].double()
                z = x @ k.T / math.sqrt(cfg.d)
                p, e = torch.softmax(z, dim=1), torch.logsumexp(z, dim=1)
                o, A, N = p @ v, p @ v.abs(), len(at)
                dx = (cfg.d + 4) * 2.0 ** -23 * (x.abs() @ k.abs().T / math.sqrt(cfg.d)).amax(dim=1)
                tol = A * (4 * dx + 2.0 ** -20 + 2 * N * 2.0 ** -24 + (2.0 ** -22 if cfg.dtype == "bf16" else 0))[:, None] + 2.0 ** -24 * o.abs()
                err = (out[l, b, heads].double() - o).abs()
                assert bool((err <= tol).all()), (err / tol).max().item()
                if lse is not None:
                    err = (lse[l, b, heads].double() - e).abs()
                    assert bool((err <= 2 * dx + 2.0 ** -20 + N * 2.0 ** -24 + 2.0 ** -22 * e.abs()).all()), err.max().item()


def attend(h, cfg, q, n_blocks, layer=0):
    L = q.shape[0]
    out, lse = torch.full(q.shape, 5.0, device="cuda"), torch.full(q.shape[:3], 5.0, device="cuda")
    blocks = torch.full((L, cfg.batch, cfg.Hkv, n_blocks), -9, dtype=torch.int32, device="cuda")
    ipot.ipot_decode_attention_blocks(h, layer, L, q, n_blocks, out, lse, blocks)
    assert ipot.ipot_sync_status(h) == 0
    return out, lse, blocks


SHAPES = [
    # L, B, Hq, Hkv, d, rows, rows of a block, blocks
    (1, 1, 4, 1, 128, 1, 16, 1), (1, 1, 8, 2, 128, 64, 64, 1), (2, 1, 8, 2, 128, 65, 64, 2), (1, 2, 32, 8, 128, 2000, 64, 5), (1, 1, 64, 8, 128, 5000, 32, 40),
    (1, 3, 6, 2, 96, 777, 16, 9), (1, 1, 5, 1, 40, 300, 16, 19), (1, 1, 7, 1, 64, 1023, 128, 3), (1, 1, 2, 2, 256, 500, 32, 4), (1, 1, 16, 1, 192, 260, 16, 6),
    (1, 1, 24, 2, 72, 999, 64, 7), (1, 1, 1, 1, 32, 4096, 16, 100), (4, 2, 8, 4, 128, 1500, 32, 12), (1, 1, 8, 1, 248, 140, 16, 3), (1, 1, 136, 4, 64, 600, 16, 8),
    (3, 1, 12, 4, 136, 400, 128, 2),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, dtype):
    L, B, Hq, Hkv, d, n, R, n_blocks = shape
    cfg = config(dtype, L, B, Hq, Hkv, d, max(n + 37, 2))
    n_blocks = min(n_blocks, -(-cfg.pot_size // R))
    g = torch.Generator(device="cuda").manual_seed(n + R)
    K, V = (torch.randn((L, B, Hkv, n, d), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    q = (1.5 * torch.randn((L, B, Hq, d), generator=g, device="cuda")).to(DT[dtype])
    h = make_pot(cfg)
    try:
        ipot.ipot_enable_blocks(h, R)
        ipot.ipot_append_chunk(h, K, V, n)
        check_bounds(h, cfg, K, R)
        for c in {n_blocks, 1, -(-cfg.pot_size // R)}:   # the last: all there are
            verify(cfg, q, K, V, R, c, *attend(h, cfg, q, c))
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("early", [False, True])   # bounds taken along by the appends, or from the rows that are there
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_layer_behind_two_to_the_31_elements(dtype, early):
    """520 units of 32768 slots of 128 channels: the last layer's rows start behind element 2^31 of the pot."""
    cfg = config(dtype, 65, 1, 16, 8, 128, 32768)
    g = torch.Generator(device="cuda").manual_seed(12)
    K, V = (torch.randn((65, 1, 8, 200, 128), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    q = torch.randn((1, 1, 16, 128), generator=g, device="cuda").to(DT[dtype])
    h = make_pot(cfg)
    try:
        if early:
            ipot.ipot_enable_blocks(h, 16)
        for part in (slice(0, 90), slice(90, 200)):
            ipot.ipot_append_chunk(h, K[:, :, :, part].contiguous(), V[:, :, :, part].contiguous(), part.stop - part.start)
        if not early:
            ipot.ipot_enable_blocks(h, 16)
        out, lse, blocks = attend(h, cfg, q, 5, layer=64)
        verify(cfg, q, K[64:], V[64:], 16, 5, out, lse, blocks)
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,R,n_blocks", [("bf16", 32768, 16, 300), ("bf16", 16384, 64, 32), ("f32", 20000, 16, 64), ("bf16", 32767, 16, 2000), ("bf16", 30000, 128, 17)])
def test_long_pots(dtype, n, R, n_blocks):
    cfg = config(dtype, 1, 1, 16, 4, 128, n)
    g = torch.Generator(device="cuda").manual_seed(9)
    K, V = (torch.randn((1, 1, 4, n, 128), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    q = torch.randn((1, 1, 16, 128), generator=g, device="cuda").to(DT[dtype])
    h = make_pot(cfg)
    try:
        ipot.ipot_append_chunk(h, K, V, n)
        ipot.ipot_enable_blocks(h, R)   # rows that are there are taken in
        verify(cfg, q, K, V, R, n_blocks, *attend(h, cfg, q, n_blocks))
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,R", [(4096, 16), (4096, 64), (700, 32)])
def test_ties_go_to_the_lower_block(dtype, n, R):
    """All keys equal: every score is the same; then two kinds of blocks in turn."""
    cfg = config(dtype, 1, 1, 4, 2, 64, n)
    q = torch.ones((1, 1, 4, 64), device="cuda").to(DT[dtype])
    V = torch.randn((1, 1, 2, n, 64), device="cuda").to(DT[dtype])
    total = -(-n // R)
    h = make_pot(cfg)
    try:
        ipot.ipot_enable_blocks(h, R)
        K = torch.ones((1, 1, 2, n, 64), device="cuda").to(DT[dtype])
        ipot.ipot_append_chunk(h, K, V, n)
        _, _, blocks = attend(h, cfg, q, 6)
        assert (blocks == torch.tensor([0, 1, 2, 3, 4, total - 1], device="cuda")).all()
        K[:, :, :, torch.arange(n, device="cuda") // R % 2 == 1] = 2   # odd blocks score higher
        ipot.ipot_reset(h)
        ipot.ipot_append_chunk(h, K, V, n)
        _, _, blocks = attend(h, cfg, q, 5)
        assert (blocks == torch.tensor([1, 3, 5, 7, total - 1], device="cuda")).all()
        odd = total // 2 - (total % 2 == 0)   # odd blocks that are not the newest one
        _, _, blocks = attend(h, cfg, q, odd + 3)
        assert blocks[0, 0, 0].tolist() == sorted(list(range(1, total - 1, 2)) + [0, 2] + [total - 1])
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("mode", ["plain", "deferred", "rope", "rope deferred"])
def test_bounds_follow_every_call_that_moves_rows(mode, dtype, d):
    """Appends of all sizes from device and host, cycles, resets, single tokens: after every one the bounds are those of the rows."""
    cfg = config(dtype, 2, 2, 8, 2, d, 500, keep=203, cap_rows=3)
    g = torch.Generator(device="cuda").manual_seed(21)
    R, rope = 16, "rope" in mode
    h = make_pot(cfg)
    try:
        if rope:
            cos, sin = (torch.empty((500, d // 2), dtype=DT[dtype], device="cuda") for _ in range(2))
            ipot.ipot_rope_tables(cos, sin, 0, 500, d, ipot.IPOT_F32 if dtype == "f32" else ipot.IPOT_BF16)
            ipot.ipot_enable_rope(h, cos, sin, ipot.IPOT_ROPE_HALF)
        if "deferred" in mode:
            ipot.ipot_set_deferred_append(h, True)
        ipot.ipot_enable_blocks(h, R)
        n, held = 0, []
        for step in (100, 1, 15, "host", 3, 256, "cycle", 1, 296, "cycle", "cycle host rows", "reset", 7, "host", 33, "again"):
            if step == "cycle" or step == "cycle host rows":
                if step == "cycle host rows":
                    K, V = (torch.randn((2, 2, 2, 60, d), generator=g, device="cuda").to(DT[dtype]).cpu().pin_memory() for _ in range(2))
                    held += [K, V]
                    ipot.ipot_append_chunk_host(h, K, V, 60)
                Q = torch.randn((2, 2, 8, 3, d), generator=g, device="cuda").to(DT[dtype])
                held.append(Q)
                ipot.ipot_score_and_compress(h, Q, 3, None)
                n = 203
            elif step == "reset":
                ipot.ipot_reset(h)
                n = 0
                continue
            elif step == "again":
                R = 64
                ipot.ipot_enable_blocks(h, R)
            else:
                m = 50 if step == "host" else step
                K, V = (torch.randn((2, 2, 2, m, d), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
                if step == "host":
                    K, V = K.cpu().pin_memory(), V.cpu().pin_memory()
                held += [K, V]
                (ipot.ipot_append_chunk_host if step == "host" else ipot.ipot_append_chunk)(h, K, V, m)
                n += m
            q = torch.randn((2, 2, 8, d), generator=g, device="cuda").to(DT[dtype])
            got = attend(h, cfg, q, 4)
            K, V = pot_rows(h, cfg, n, rope)
            check_bounds(h, cfg, K, R)
            verify(cfg, q, K, V, R, 4, *got)
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
def test_some_layers_own_stream_and_replays():
    cfg = config("bf16", 4, 1, 8, 2, 128, 1000)
    g = torch.Generator(device="cuda").manual_seed(2)
    K, V = (torch.randn((4, 1, 2, 1000, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((4, 1, 8, 128), generator=g, device="cuda").bfloat16()
    h = make_pot(cfg)
    s = torch.cuda.Stream()
    try:
        ipot.ipot_enable_blocks(h, 32)
        ipot.ipot_append_chunk(h, K, V, 1000)
        verify(cfg, q[1:3], K[1:3], V[1:3], 32, 9, *attend(h, cfg, q[1:3].contiguous(), 9, layer=1))
        torch.cuda.synchronize()
        ipot.ipot_set_stream(h, s.cuda_stream)
        out, lse, blocks = attend(h, cfg, q, 9)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ipot.ipot_set_stream(h, s.cuda_stream)
            ipot.ipot_reset(h)
            ipot.ipot_append_chunk(h, K, V, 1000)     # the bounds are part of what is captured
            ipot.ipot_decode_attention_blocks(h, 0, 4, q, 9, out, lse, blocks)
        for seed in (5, 6):
            for x in (K, V, q):
                x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
            out.fill_(0)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                graph.replay()
            s.synchronize()
            verify(cfg, q, K, V, 32, 9, out, lse, blocks)
        del graph
    finally:
        torch.cuda.synchronize()
        ipot.ipot_destroy(h)


@pytest.mark.gpu
def test_refusals():
    cfg = config("bf16", 2, 1, 4, 2, 64, 100)
    L = ipot.lib()
    q, out = torch.ones((2, 1, 4, 64), device="cuda").bfloat16(), torch.zeros((2, 1, 4, 64), device="cuda")
    K = torch.ones((2, 1, 2, 20, 64), device="cuda").bfloat16()
    h = make_pot(cfg)
    try:
        def rc(h=h, layer=0, layers=2, q=q.data_ptr(), n=2, out=out.data_ptr(), lse=None, blocks=None):
            return L.ipot_decode_attention_blocks(h, layer, layers, q, n, out, lse, blocks)
        assert rc() == ipot.IPOT_E_STATE and L.ipot_view_blocks(h, None, None, None) == ipot.IPOT_E_STATE
        for bad in (0, 8, 17, 48, 256, -16):
            assert L.ipot_enable_blocks(h, bad) == ipot.IPOT_E_INVALID
        ipot.ipot_enable_blocks(h, 16)
        ipot.ipot_enable_blocks(h, 16)
        assert rc() == ipot.IPOT_E_STATE and ipot.ipot_view_blocks(h)[2] == 0   # empty
        cos = torch.ones((100, 32), device="cuda").bfloat16()
        assert L.ipot_enable_rope(h, cos.data_ptr(), cos.data_ptr(), 1) == ipot.IPOT_E_STATE   # the bounds would be those of other keys
        ipot.ipot_append_chunk(h, K, K, 20)
        for kw in (dict(h=None), dict(q=None), dict(out=None), dict(q=q.data_ptr() + 8), dict(out=out.data_ptr() + 2), dict(out=out.data_ptr() + 4), dict(lse=out.data_ptr() + 1), dict(blocks=out.data_ptr() + 2),
                   dict(layer=-1), dict(layers=0), dict(layer=1), dict(n=0), dict(n=8), dict(n=-1)):
            assert rc(**kw) == ipot.IPOT_E_INVALID, kw
        assert ipot.ipot_sync_status(h) == 0 and bool((out == 0).all())
        assert rc(n=7) == 0
    finally:
        ipot.ipot_destroy(h)


def test_refusals_without_a_pot():
    L = ipot.lib()
    assert L.ipot_enable_blocks(None, 16) == ipot.IPOT_E_INVALID
    assert L.ipot_view_blocks(None, None, None, None) == ipot.IPOT_E_INVALID
    assert L.ipot_decode_attention_blocks(None, 0, 1, 16, 1, 16, None, None) == ipot.IPOT_E_INVALID
