"""The range of a chunk's attention (ipot_chunk_attention): logits far from zero.

Tolerances as in test_chunk_attention_gpu.py.  Where a test's logits are exact in fp32 and differ by more than any weight resolves, every weight is
0 or the same for all keys that tie for the maximum, and what that file allows for the logits' own error (dx) is zero for the output."""
import pytest
import torch

from paper_2410_01518_b200 import ipot
from test_chunk_attention_gpu import Case, reference

SHAPES = [
    # d, rows in the pot, new tokens: tcgen05 with one query tile a block, with two, of wide heads; few rows; a cluster of blocks
    (128, 700, 200), (64, 1000, 2600), (256, 300, 70), (128, 900, 1), (96, 4000, 40),
]


def check_exact_logits(c):
    """Every row of the call against 64 bits, weights without an error of the logits."""
    half = 2.0 ** -8 if c.dtype == "bf16" else 0.0
    for h in range(c.Hq):
        kv = h // (c.Hq // c.Hkv)
        o, A, X, e = reference(c.q[0, 0, h], c.k[0, 0, kv], c.v[0, 0, kv], c.K[0, 0, kv], c.V[0, 0, kv], c.n)
        N = c.len + c.n
        tol = (A * (2.0 ** -20 + 2 * N * 2.0 ** -24 + half)) * (1 + half) + (half + 2.0 ** -24) * o.abs()
        err = (c.out[0, 0, h].double() - o).abs()
        assert bool((err <= tol).all()), f"head {h}: {(err / tol).max().item():.3g} of the tolerance"
        dx = (c.d + 4) * 2.0 ** -23 * X
        err = (c.lse[0, 0, h].double() - e).abs()
        assert bool((err <= 2 * dx + 2.0 ** -20 + N * 2.0 ** -24 + 2.0 ** -22 * e.abs()).all()), err.max().item()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power", [22, 26, 29, 34, 60, 100])
@pytest.mark.parametrize("d,length,n", SHAPES)
def test_logits_of_any_size(d, length, n, power, dtype):
    """q . k is 1, 2 or 3 times +-2^power: many keys tie for the maximum of a row, and 2^power / sqrt(d) in binary orders is no whole number, so a reference
    that is rounded and a logit that is not differ by up to half a step of the logit, far more than the exponential's range."""
    c = Case(dtype, 1, 1, 4, 2, d, length, n)
    try:
        g = torch.Generator(device="cuda").manual_seed(power + d)
        for x in (c.K, c.k):
            x.zero_()
            x[..., 0] = torch.randint(1, 4, x.shape[:-1], generator=g, device="cuda").to(x.dtype) * 2.0 ** (power // 2)
        c.q.zero_()
        c.q[..., 0] = 2.0 ** (power - power // 2)
        c.q[:, :, 1::2] *= -1
        ipot.ipot_reset(c.h)
        ipot.ipot_append_chunk(c.h, c.K, c.V, length)
        c.run()
        check_exact_logits(c)
    finally:
        c.close()
