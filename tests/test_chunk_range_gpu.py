"""The range of a chunk's attention (ipot_chunk_attention) and of generation over selected blocks: logits far from zero, values up to 2^127.

Tolerances as in test_chunk_attention_gpu.py.  Where a test's logits are exact in fp32 and differ by more than any weight resolves, every weight is
0 or the same for all keys that tie for the maximum, and what that file allows for the logits' own error (dx) is zero for the output."""
import math

import pytest
import torch

from paper_2410_01518_b200 import ipot
from test_chunk_attention_gpu import Case, check, reference

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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("logit", [-9.0, 0.0, 9.0, 12.25, 40.0])
@pytest.mark.parametrize("sign", ["one", "both"])
@pytest.mark.parametrize("d,length,n", SHAPES + [(128, 20000, 300), (256, 9000, 20)])
def test_values_up_to_two_to_the_127(d, length, n, sign, logit, dtype):
    """Every key counts (almost) the same, e^logit against no reference at all, and every value lies between 2^126 and 2^127: the result does too (or, with both signs,
    within), but neither the weights nor their number times a value does.  12.25 keeps the sum over 64 keys just below 2^24."""
    c = Case(dtype, 1, 1, 4, 2, d, length, n)
    try:
        g = torch.Generator(device="cuda").manual_seed(d + n)
        for x in (c.K, c.k):   # q . k / sqrt(d) = logit times a number between 1 - 2^-6 and 1
            x.copy_(1 - 2.0 ** -6 * torch.rand(x.shape[:-1] + (1,), generator=g, device="cuda").expand(x.shape))
        c.q.fill_(logit / math.sqrt(d))
        for x in (c.V, c.v):
            x.copy_(2.0 ** 126 * (1 + torch.rand(x.shape, generator=g, device="cuda") * (1 - 2.0 ** -7)))
            if sign == "both":
                x.mul_(1 - 2 * torch.randint(0, 2, x.shape, generator=g, device="cuda"))
        ipot.ipot_reset(c.h)
        ipot.ipot_append_chunk(c.h, c.K, c.V, length)
        c.run()
        for h in (0, 3):
            kv = h // 2
            check(c.out[0, 0, h], c.lse[0, 0, h], reference(c.q[0, 0, h], c.k[0, 0, kv], c.v[0, 0, kv], c.K[0, 0, kv], c.V[0, 0, kv], n), d, length + n, dtype)
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("logit", [0.0, 9.0, 40.0])
def test_values_up_to_two_to_the_127_over_selected_blocks(logit, dtype):
    """Half of the blocks of one unit of four heads; outputs in fp32, as test_blocks_gpu.py bounds them."""
    n, d, R, n_blocks = 30000, 128, 128, 100
    c = Case(dtype, 1, 1, 4, 1, d, n, 1)
    try:
        g = torch.Generator(device="cuda").manual_seed(5)
        c.K.copy_(1 - 2.0 ** -6 * torch.rand(c.K.shape[:-1] + (1,), generator=g, device="cuda").expand(c.K.shape))
        c.V.copy_(2.0 ** 126 * (1 + torch.rand(c.V.shape, generator=g, device="cuda") * (1 - 2.0 ** -7)))
        q = torch.full((1, 1, 4, d), logit / math.sqrt(d), device="cuda").to(c.K.dtype)
        ipot.ipot_reset(c.h)
        ipot.ipot_append_chunk(c.h, c.K, c.V, n)
        ipot.ipot_enable_blocks(c.h, R)
        out, lse, blocks = torch.zeros((1, 1, 4, d), device="cuda"), torch.zeros((1, 1, 4), device="cuda"), torch.zeros((1, 1, 1, n_blocks), dtype=torch.int32, device="cuda")
        ipot.ipot_decode_attention_blocks(c.h, 0, 1, q, n_blocks, out, lse, blocks)
        assert ipot.ipot_sync_status(c.h) == 0
        at = (blocks[0, 0, 0].long()[:, None] * R + torch.arange(R, device="cuda")).flatten()
        at = at[at < n]
        k, v, x = c.K[0, 0, 0][at].double(), c.V[0, 0, 0][at].double(), q[0, 0].double()
        z = x @ k.T / math.sqrt(d)
        p, N = torch.softmax(z, dim=1), len(at)
        o, A = p @ v, p @ v.abs()
        dx = (d + 4) * 2.0 ** -23 * (x.abs() @ k.abs().T / math.sqrt(d)).amax(dim=1)
        tol = A * (4 * dx + 2.0 ** -20 + 2 * N * 2.0 ** -24 + (2.0 ** -22 if dtype == "bf16" else 0))[:, None] + 2.0 ** -24 * o.abs()
        assert bool(((out[0, 0].double() - o).abs() <= tol).all())
        e = torch.logsumexp(z, dim=1)
        assert bool(((lse[0, 0].double() - e).abs() <= 2 * dx + 2.0 ** -20 + N * 2.0 ** -24 + 2.0 ** -22 * e.abs()).all())
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d,length,n", [(64, 700, 200), (128, 700, 200), (64, 100, 1500)])
@pytest.mark.parametrize("power,below", [(24, b) for b in (-3, 0, 1, 2, 3, 17, 38, 39, 64, 65, 66, 104, 105)] + [(12, b) for b in (-3, 0, 1, 2, 39, 40, 41)] + [(p, 1) for p in (10, 11, 13, 16, 20, 22)])
def test_references_far_from_zero(power, below, d, length, n):
    """All logits equal and 2^power - below - 1/2 in binary orders: whatever form a tile takes, every key weighs the same."""
    c = Case("bf16", 1, 1, 4, 2, d, length, n)
    try:
        orders = 1.4426950408889634 / math.sqrt(d)   # of a unit of q . k (the kernel's own differs in the eighth digit: at 2^24 by less than 2)
        whole = round((2.0 ** power - below - 0.5) / orders)
        for i in range(4):   # the number in base 256, a digit a channel
            for x in (c.K, c.k):
                x[..., i] = (whole >> 8 * i) & 255
            c.q[..., i] = 2.0 ** (8 * i)
        for x in (c.K, c.k, c.q):
            x[..., 4:] = 0
        ipot.ipot_reset(c.h)
        ipot.ipot_append_chunk(c.h, c.K, c.V, length)
        c.run()
        check_exact_logits(c)
    finally:
        c.close()
