"""The order of blocks whose scores agree in their first 32 differing bits (ipot_decode_attention_blocks): what lies below decides, and only then the lower index.

Scores are exact: one head, queries of ones, and the rows of a block all equal, so that a block's score is the sum of a key's channels, a few terms of one sign in 64 bits."""
import pytest
import torch

from test_blocks_gpu import attend, config
from parity import make_pot
from paper_2410_01518_b200 import ipot


def lists(first, second, n_blocks, d=32, R=16):
    """Per block a score of `first` (exact in fp32) + `second` (exact in fp32): the list that the library takes of them."""
    total = len(first)
    cfg = config("f32", 1, 1, 1, 1, d, total * R)
    K = torch.zeros((1, 1, 1, total, R, d), device="cuda")
    K[..., 0] = torch.tensor(first, dtype=torch.float32, device="cuda")[:, None]
    K[..., 7] = torch.tensor(second, dtype=torch.float32, device="cuda")[:, None]
    K = K.view(1, 1, 1, total * R, d)
    h = make_pot(cfg)
    try:
        ipot.ipot_append_chunk(h, K, torch.zeros_like(K), total * R)
        ipot.ipot_enable_blocks(h, R)
        return attend(h, cfg, torch.ones((1, 1, 1, d), device="cuda"), n_blocks)[2][0, 0, 0].tolist()
    finally:
        ipot.ipot_destroy(h)


def best(first, second, n_blocks):
    s = [a + b for a, b in zip(first, second)]   # (Python's floats: exact here)
    others = sorted(range(len(s) - 1), key=lambda b: (-s[b], b))[:n_blocks - 1]
    return sorted(others + [len(s) - 1])


@pytest.mark.gpu
@pytest.mark.parametrize("total", [200, 257, 258, 1000, 2048])   # up to 2 blocks a thread, and more
@pytest.mark.parametrize("step", [2.0 ** -23, 2.0 ** -32, 2.0 ** -40, 2.0 ** -50])
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_differ_far_behind_the_first_differing_bit(falling, step, total):
    """A few blocks score 2^20 more, so that the highest differing bit is one of the exponent; of the rest, 1 + i step, the larger are in, wherever they lie."""
    g = torch.Generator().manual_seed(total)
    far = set(torch.randperm(total - 1, generator=g)[:5].tolist())
    order = list(range(total)) if not falling else list(range(total, 0, -1))
    first = [2.0 ** 20 if b in far else 1.0 for b in range(total)]
    second = [0.0 if b in far else order[b] * step for b in range(total)]
    for n_blocks in (1 + 5 + 1, 1 + 5 + 60, total // 2, total - 1):
        assert lists(first, second, n_blocks) == best(first, second, n_blocks), n_blocks


@pytest.mark.gpu
@pytest.mark.parametrize("total", [250, 1500])
def test_ties_among_scores_that_differ_far_behind(total):
    """Pairs of neighbouring blocks tie in all 64 bits: the border runs through one of them."""
    first = [2.0 ** 20 if b % 97 == 5 else 1.0 for b in range(total)]
    second = [0.0 if b % 97 == 5 else (b // 2) * 2.0 ** -45 for b in range(total)]
    for n_blocks in (40, 41, 42, 43, total // 3, total // 3 + 1):
        assert lists(first, second, n_blocks) == best(first, second, n_blocks), n_blocks


@pytest.mark.gpu
@pytest.mark.parametrize("total", [150, 600])
def test_negative_and_mixed_scores(total):
    """Scores on both sides of zero, apart by less than a 32-bit window shows on either."""
    first = [(-1.0) ** b for b in range(total)]
    second = [first[b] * ((b * 37) % total) * 2.0 ** -42 for b in range(total)]
    for n_blocks in (2, total // 4, total // 2, total // 2 + 9, total - 2):
        assert lists(first, second, n_blocks) == best(first, second, n_blocks), n_blocks
