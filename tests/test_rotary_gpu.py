"""Rotary tables (ipot_rope_tables) and rows (ipot_rope_rows) against the definitions in 64 (80) bits, and their refusals.

Tolerances.  A table entry: the angle in turns is a product of two rounded 64-bit numbers (2^-52 of the angle), what is left of it
after whole turns, at most half a turn, becomes fp32 (2 x <= 1: half a step is 2^-25, times pi in radians), sincospif is within 1 ulp
(2^-23 of a value of at most 1), the magnitude is one rounded product (2^-24), and a bf16 entry is rounded once more (2^-8 of the value).
A rotated element, as in parity.py: half a step of the storage type + 2^-23 (|lo cos| + |hi sin|)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2410_01518_b200 import inputs, ipot
from parity import make_pot

DT = {"bf16": (torch.bfloat16, ipot.IPOT_BF16, 2.0 ** -8), "f32": (torch.float32, ipot.IPOT_F32, 2.0 ** -24)}
SCALINGS = {
    "plain": dict(scaling=ipot.IPOT_ROPE_PLAIN),
    "linear": dict(scaling=ipot.IPOT_ROPE_LINEAR, factor=4.0),
    "stretched": dict(scaling=ipot.IPOT_ROPE_STRETCHED, factor=8.0),
    "bands": dict(scaling=ipot.IPOT_ROPE_BANDS, factor=8.0, original_len=8192.0, low=1.0, high=4.0),
    "ramp": dict(scaling=ipot.IPOT_ROPE_RAMP, factor=16.0, original_len=4096.0, low=1.0, high=32.0),
    "ramp_given_magnitude": dict(scaling=ipot.IPOT_ROPE_RAMP, factor=16.0, original_len=4096.0, low=1.0, high=32.0, magnitude=0.75),
}


def frequencies(r, base, scaling, factor=1.0, original_len=0.0, low=0.0, high=0.0, magnitude=0.0):
    """The header's definitions, pair by pair, in extended precision: (radians per position, magnitude)."""
    ld = np.longdouble
    base, s, L = ld(base), ld(factor), ld(original_len)
    pi = ld("3.14159265358979323846264338327950288")
    out = []
    for i in range(r // 2):
        t = base ** (ld(-2 * i) / r)
        if scaling == ipot.IPOT_ROPE_LINEAR:
            t = t / s
        elif scaling == ipot.IPOT_ROPE_STRETCHED:
            t = (base * s ** (ld(r) / (r - 2))) ** (ld(-2 * i) / r)
        elif scaling == ipot.IPOT_ROPE_BANDS:
            turns = L * t / (2 * pi)
            if turns < low:
                t = t / s
            elif turns <= high:
                g = (turns - low) / (high - low)
                t = (1 - g) * t / s + g * t
        elif scaling == ipot.IPOT_ROPE_RAMP:
            def D(b):
                return r * np.log(L / (2 * pi * b)) / (2 * np.log(base))
            a, e = max(np.floor(D(high)), 0), min(np.ceil(D(low)), r - 1)
            g = 0 if i <= a else 1 if i >= e else (i - a) / (e - a)
            t = (1 - g) * t + g * t / s
        out.append(t)
    if magnitude == 0.0:
        magnitude = 0.1 * math.log(factor) + 1 if scaling == ipot.IPOT_ROPE_RAMP else 1.0
    return np.array(out), magnitude


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", list(SCALINGS))
@pytest.mark.parametrize("r,first,n,base", [(128, 0, 4096, 10000.0), (90, 1000003, 77, 500000.0), (32, 0, 1, 10000.0), (256, 65530, 33, 1e6), (6, 16777200, 50, 1e4),
                                            (128, (1 << 31) - 5, 5, 10000.0)])
def test_tables(kind, dtype, r, first, n, base):
    tdt, idt, half_step = DT[dtype]
    kw = dict(SCALINGS[kind])
    guard = 64
    cos, sin = (torch.full((n * (r // 2) + guard,), 7.0, dtype=tdt, device="cuda") for _ in range(2))
    ipot.ipot_rope_tables(cos, sin, first, n, r, idt, base=base, stream=torch.cuda.current_stream().cuda_stream, **kw)
    f, mag = frequencies(r, base, **kw)
    ang = np.arange(first, first + n, dtype=np.longdouble)[:, None] * f[None]
    for got, want in ((cos, np.cos(ang)), (sin, np.sin(ang))):
        assert (got[n * (r // 2):] == 7.0).all()
        g, w = got[:n * (r // 2)].double().cpu().numpy().reshape(n, -1), (want * mag).astype(np.float64)
        bound = mag * (2.0 ** -52 * ang.astype(np.float64) + math.pi * 2.0 ** -25 + 2.0 ** -23 + 2.0 ** -24) + half_step * np.abs(w) + 2.0 ** -130
        assert (np.abs(g - w) <= bound).all(), float(np.max(np.abs(g - w) / bound))


def test_tables_refusals():
    """Found on the host before anything is launched: no device needed."""
    L = ipot.lib()

    def rc(rotary=64, scaling=0, base=1e4, factor=2.0, original=4096.0, low=1.0, high=4.0, mag=0.0, first=0, n=8, dtype=ipot.IPOT_F32, cos=4096, sin=4096, spec=True):
        s = ipot.ipot_rope_spec_t(rotary, scaling, base, factor, original, low, high, mag)
        return L.ipot_rope_tables(C.byref(s) if spec else None, first, n, dtype, cos, sin, None)

    bad = [dict(spec=False), dict(cos=None), dict(sin=None), dict(cos=4100), dict(sin=4098), dict(rotary=63), dict(rotary=0), dict(rotary=258), dict(n=0),
           dict(first=-1), dict(first=(1 << 31) - 7), dict(first=1 << 62), dict(dtype=2), dict(scaling=-1), dict(scaling=5), dict(base=1.0), dict(base=math.inf), dict(base=math.nan),
           dict(mag=-1.0), dict(mag=math.nan), dict(scaling=1, factor=0.0), dict(scaling=1, factor=math.inf), dict(scaling=2, rotary=2), dict(scaling=2, base=1e300, factor=1e300),
           dict(scaling=3, original=0.0), dict(scaling=3, low=0.0), dict(scaling=3, low=4.0), dict(scaling=4, high=math.nan), dict(scaling=4, original=math.inf)]
    for kw in bad:
        assert rc(**kw) == ipot.IPOT_E_INVALID, kw


def rows_reference(x, pos, cos, sin, r, interleaved, out):
    """Rotated rows in 64 bits and the magnitude that bounds their error; [L, B, H, n, d], pos [B, n]."""
    z, mag = x.copy(), np.zeros_like(x)
    c, s = cos[np.maximum(pos, 0)][None, :, None], sin[np.maximum(pos, 0)][None, :, None]
    lo, hi = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    zl, zh = (z[..., 0:r:2], z[..., 1:r:2]) if interleaved else (z[..., :r // 2], z[..., r // 2:r])
    ml, mh = (mag[..., 0:r:2], mag[..., 1:r:2]) if interleaved else (mag[..., :r // 2], mag[..., r // 2:r])
    zl[...], zh[...] = lo * c - hi * s, hi * c + lo * s
    ml[...], mh[...] = np.abs(lo * c) + np.abs(hi * s), np.abs(hi * c) + np.abs(lo * s)
    skip = np.broadcast_to((pos < 0)[None, :, None, :, None], x.shape)
    return np.where(skip, out, z), np.where(skip, 0.0, mag)


def array(g, shape, dtype, layout):
    L, B, H, n, d = shape
    if layout == "packed":
        return torch.randn((L, B, n, H, d), generator=g, device="cuda").to(dtype).transpose(2, 3)
    if layout == "wide":   # queries, keys and values of a token side by side, rows of other types between them
        return torch.randn((L, B, n, H * 2, d + 16), generator=g, device="cuda").to(dtype)[:, :, :, ::2, 8:8 + d].transpose(2, 3)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


ROWS = [
    # L, B, Hq, Hkv, d, n, rotary
    (1, 1, 32, 8, 128, 1, 128), (2, 3, 12, 4, 96, 37, 96), (1, 2, 6, 2, 64, 65, 32), (1, 1, 3, 1, 256, 9, 250), (3, 1, 5, 5, 40, 129, 40),
    (1, 2, 8, 1, 128, 33, 26), (1, 1, 2, 2, 72, 200, 6), (1, 1, 8, 8, 32, 1000, 2),
]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", ROWS)
@pytest.mark.parametrize("dtype,table", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("pairing", [ipot.IPOT_ROPE_HALF, ipot.IPOT_ROPE_INTERLEAVED])
@pytest.mark.parametrize("layout,mode", [("dense", "out"), ("packed", "in place"), ("wide", "out")])
def test_rows(shape, dtype, table, pairing, layout, mode):
    L, B, Hq, Hkv, d, n, r = shape
    tdt, idt, half_step = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(11)
    cfg = inputs.small_config(cfg_id=990, pot_size=64, keep=16, nuc_slots=0, cap_rows=1, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, layers=1, batch=B)
    rows = 500
    ang = torch.rand((rows, r // 2), generator=g, device="cuda") * 7
    cos, sin = ang.cos().to(DT[table][0]), ang.sin().to(DT[table][0])
    pos = torch.randint(0, rows, (B, n), generator=g, device="cuda", dtype=torch.int32)
    if n > 2:
        pos[0, n // 2] = -1
        pos[-1, -1] = -2 ** 31
    q, k = array(g, (L, B, Hq, n, d), tdt, layout), array(g, (L, B, Hkv, n, d), tdt, layout)
    before = [x.double().cpu().numpy() for x in (q, k)]
    outs = [q, k] if mode == "in place" else [array(g, x.shape, tdt, "packed") for x in (q, k)]
    there = [x.double().cpu().numpy() for x in outs]
    h = make_pot(cfg)
    try:
        ipot.ipot_rope_rows(h, L, n, cos, sin, rows, r, pairing, DT[table][1], positions=pos, q=q, q_out=outs[0], k=k, k_out=outs[1], q_strides=q.stride()[:4],
                            k_strides=k.stride()[:4], q_out_strides=outs[0].stride()[:4], k_out_strides=outs[1].stride()[:4])
        assert ipot.ipot_sync_status(h) == 0
    finally:
        ipot.ipot_destroy(h)
    c, s = cos.double().cpu().numpy(), sin.double().cpu().numpy()
    for x, o, was in zip(before, outs, there):
        want, mag = rows_reference(x, pos.cpu().numpy(), c, s, r, pairing == ipot.IPOT_ROPE_INTERLEAVED, was)
        err = np.abs(o.double().cpu().numpy() - want)
        assert (err <= np.where(mag > 0, half_step * np.abs(want) + 2.0 ** -23 * (1 + half_step) * mag, 0.0)).all(), err.max()


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_agree_with_the_pot_s_own_copy(interleaved):
    """Keys rotated at the slots they will have equal the rotated copy bit for bit; tables come from ipot_rope_tables."""
    cfg = inputs.small_config(cfg_id=991, pot_size=300, keep=100, nuc_slots=0, cap_rows=1, Hq=8, Hkv=4, d=128, dtype="bf16", layers=2, batch=2)
    g = torch.Generator(device="cuda").manual_seed(3)
    pairing = ipot.IPOT_ROPE_INTERLEAVED if interleaved else ipot.IPOT_ROPE_HALF
    cos, sin = (torch.empty((300, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ipot.ipot_rope_tables(cos, sin, 0, 300, 128, ipot.IPOT_BF16)
    h = make_pot(cfg)
    try:
        ipot.ipot_enable_rope(h, cos, sin, pairing)
        K = torch.randn((2, 2, 4, 300, 128), generator=g, device="cuda").to(torch.bfloat16)
        ipot.ipot_append_chunk(h, K[:, :, :, :200].contiguous(), K[:, :, :, :200].contiguous(), 200)
        new = K[:, :, :, 200:].contiguous()
        out = torch.empty_like(new)
        ipot.ipot_rope_rows(h, 2, 100, cos, sin, 300, 128, pairing, ipot.IPOT_BF16, first=200, k=new, k_out=out)
        ipot.ipot_append_chunk(h, new, new, 100)
        assert ipot.ipot_sync_status(h) == 0
        copy = ipot.device_array(ipot.ipot_view_rope(h), (2, 2, 4, 300, 128), "bf16")
        assert torch.equal(copy[:, :, :, 200:].view(torch.int16), out.view(torch.int16))
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
def test_rows_refusals_positions_beyond_the_table_and_replay():
    cfg = inputs.small_config(cfg_id=992, pot_size=64, keep=16, nuc_slots=0, cap_rows=1, Hq=4, Hkv=2, d=64, dtype="bf16", batch=2)
    x, y = (torch.ones((1, 2, 4, 8, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    t = torch.ones((32, 32), dtype=torch.bfloat16, device="cuda")
    st = ipot.ipot_strides_t
    dense = (4096, 2048, 512, 64)
    h = make_pot(cfg)
    try:
        def rc(pot=h, rope=True, cos=t.data_ptr(), sin=t.data_ptr(), rows=32, rotary=64, pairing=1, dtype=ipot.IPOT_BF16, layers=1, n=8, positions=None, first=0, q=x.data_ptr(),
               qs=None, qo=y.data_ptr(), qos=None, k=None, ko=None):
            r = ipot.ipot_rope_t(cos, sin, rows, rotary, pairing, dtype)
            return ipot.lib().ipot_rope_rows(pot, C.byref(r) if rope else None, layers, n, positions, first, q, C.byref(st(*qs)) if qs else None, qo,
                                             C.byref(st(*qos)) if qos else None, k, None, ko, None)
        assert rc() == 0 and rc(qs=dense, qos=dense) == 0 and rc(qo=x.data_ptr()) == 0
        for kw in (dict(pot=None), dict(rope=False), dict(cos=None), dict(sin=t.data_ptr() + 2), dict(rows=0), dict(rotary=0), dict(rotary=33), dict(rotary=66), dict(pairing=0),
                   dict(pairing=3), dict(dtype=2), dict(layers=0), dict(layers=65536), dict(n=0), dict(positions=t.data_ptr() + 2), dict(first=-1), dict(first=25), dict(q=None),
                   dict(qo=None), dict(q=None, qo=None), dict(k=x.data_ptr()), dict(ko=x.data_ptr()), dict(q=x.data_ptr() + 2), dict(qo=y.data_ptr() + 8),
                   dict(qs=(4096, 2048, 512, 60)), dict(qs=(4096, 2048, -512, 64)), dict(qo=x.data_ptr(), qos=(4096, 2048, 64, 256)), dict(n=1 << 29, positions=t.data_ptr())):
            assert rc(**kw) == ipot.IPOT_E_INVALID, kw
        x.fill_(1)   # (the allowed calls above have rotated it in place)
        # a position beyond the table: its row stays, the others are rotated, the status is raised
        pos = torch.zeros((2, 8), dtype=torch.int32, device="cuda")
        out = torch.zeros_like(x)
        s = torch.cuda.Stream()
        ipot.ipot_rope_rows(h, 1, 8, t, t, 32, 64, 2, ipot.IPOT_BF16, positions=pos, q=x, q_out=out)   # (1, 1) -> (0, 2)
        torch.cuda.synchronize()
        assert ipot.ipot_sync_status(h) == 0
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ipot.ipot_set_stream(h, s.cuda_stream)
            ipot.ipot_rope_rows(h, 1, 8, t, t, 32, 64, 2, ipot.IPOT_BF16, positions=pos, q=x, q_out=out)
        out.fill_(9)
        pos[1, 3] = 32
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert ipot.ipot_sync_status(h) == ipot.IPOT_E_BOUNDS
        assert (out[0, 1, :, 3] == 9).all()
        out[0, 1, :, 3] = out[0, 0, :, 0]
        assert (out[..., 0::2] == 0).all() and (out[..., 1::2] == 2).all()
        del graph
    finally:
        ipot.ipot_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("pairing", [ipot.IPOT_ROPE_HALF, ipot.IPOT_ROPE_INTERLEAVED])
def test_rows_of_a_large_chunk_in_place_and_out(pairing):
    """More than L2 holds: the same rows as in pieces."""
    cfg = inputs.small_config(cfg_id=993, pot_size=64, keep=16, nuc_slots=0, cap_rows=1, Hq=16, Hkv=4, d=128, dtype="bf16", batch=4)
    g = torch.Generator(device="cuda").manual_seed(8)
    n, r = 4096, 96
    cos, sin = (torch.randn((n, r // 2), generator=g, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((1, 4, 16, n, 128), generator=g, device="cuda").bfloat16()
    out, pieces = torch.zeros_like(q), torch.zeros_like(q)
    h = make_pot(cfg)
    try:
        ipot.ipot_rope_rows(h, 1, n, cos, sin, n, r, pairing, ipot.IPOT_BF16, q=q, q_out=out)
        for a in range(0, n, 1024):
            x, y = q[:, :, :, a:a + 1024], pieces[:, :, :, a:a + 1024]
            ipot.ipot_rope_rows(h, 1, 1024, cos, sin, n, r, pairing, ipot.IPOT_BF16, first=a, q=x, q_out=y, q_strides=x.stride()[:4], q_out_strides=y.stride()[:4])
        assert torch.equal(out, pieces) and bool((out[..., r:] == q[..., r:]).all()) and not torch.equal(out[..., :r], q[..., :r])
        ipot.ipot_rope_rows(h, 1, n, cos, sin, n, r, pairing, ipot.IPOT_BF16, q=q, q_out=q)
        assert ipot.ipot_sync_status(h) == 0 and torch.equal(q, out)
    finally:
        ipot.ipot_destroy(h)
