"""Rotary tables (ipot_rope_tables) at the ends of their parameters' ranges; definitions and tolerances are those of test_rotary_gpu.py."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2410_01518_b200 import ipot
from test_rotary_gpu import DT, frequencies


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("factor", [1e-6, 2.0 ** -15, 0.5, 1.0, 1.5])
def test_a_ramp_that_does_not_stretch_has_magnitude_one(factor, dtype):
    """0.1 ln(s) + 1 belongs to contexts that were made longer (s > 1); below it would shrink, vanish and change sign."""
    tdt, idt, half_step = DT[dtype]
    r, n, kw = 64, 300, dict(scaling=ipot.IPOT_ROPE_RAMP, factor=factor, original_len=4096.0, low=1.0, high=32.0)
    cos, sin = (torch.full((n, r // 2), 7.0, dtype=tdt, device="cuda") for _ in range(2))
    ipot.ipot_rope_tables(cos, sin, 0, n, r, idt, base=10000.0, stream=torch.cuda.current_stream().cuda_stream, **kw)
    mag = 0.1 * math.log(factor) + 1 if factor > 1 else 1.0
    f, _ = frequencies(r, 10000.0, magnitude=mag, **kw)
    ang = np.arange(n, dtype=np.longdouble)[:, None] * f[None]
    for got, want in ((cos, np.cos(ang)), (sin, np.sin(ang))):
        g, w = got.double().cpu().numpy(), (want * mag).astype(np.float64)
        # the frequency's own roundings (exponent, power, 2 pi, quotient, blend) and the product's: (ln base + 8) 2^-53 < 2^-48 of the angle
        bound = mag * (2.0 ** -48 * ang.astype(np.float64) + math.pi * 2.0 ** -25 + 2.0 ** -23 + 2.0 ** -24) + half_step * np.abs(w) + 2.0 ** -130
        assert (np.abs(g - w) <= bound).all(), float(np.max(np.abs(g - w) / bound))


def test_tables_without_numbers_are_refused():
    """Angles or magnitudes that no longer are numbers; found on the host, no device needed."""
    L = ipot.lib()

    def rc(scaling, factor=2.0, base=1e4, mag=0.0, rotary=64, original=4096.0):
        s = ipot.ipot_rope_spec_t(rotary, scaling, base, factor, original, 1.0, 4.0, mag)
        return L.ipot_rope_tables(C.byref(s), 0, 8, ipot.IPOT_F32, 4096, 4096 << 8, None)

    for kw in (dict(scaling=ipot.IPOT_ROPE_LINEAR, factor=1e-307), dict(scaling=ipot.IPOT_ROPE_BANDS, factor=1e-307), dict(scaling=ipot.IPOT_ROPE_RAMP, factor=1e-307, original=1e-300),
               dict(scaling=ipot.IPOT_ROPE_LINEAR, factor=5e-324), dict(scaling=ipot.IPOT_ROPE_PLAIN, mag=3.5e38), dict(scaling=ipot.IPOT_ROPE_PLAIN, mag=1e300)):
        assert rc(**kw) == ipot.IPOT_E_INVALID, kw
