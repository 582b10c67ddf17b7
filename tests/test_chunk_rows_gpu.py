"""Chunk attention of 9 to 16 query rows a KV head, on either side of the rule that sends them to the kernel of few rows or to that of many, against the
definition in 64 bits with the tolerances of test_chunk_attention_gpu.py."""
import pytest

from test_chunk_attention_gpu import Case

CALLS = [
    # layers, streams, query heads, KV heads, channels, rows in the pot, new tokens
    (1, 1, 16, 4, 128, 9000, 4), (1, 5, 4, 1, 128, 900, 3), (33, 1, 8, 2, 128, 130, 4), (32, 1, 8, 2, 64, 600, 3), (65, 1, 4, 1, 256, 40, 4),
    (1, 17, 9, 1, 256, 77, 1), (97, 1, 5, 1, 96, 50, 3), (12, 1, 32, 8, 64, 33, 4), (16, 1, 64, 8, 32, 20, 2), (1, 1, 16, 1, 200, 3000, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("call", CALLS)
def test_nine_to_sixteen_rows(call, dtype):
    c = Case(dtype, *call, seed=call[5])
    try:
        layers = [0, call[0] // 2, call[0] - 1]
        c.run().verify(layers=layers)
    finally:
        c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("call,tokens", [((2, 3, 16, 4, 128, 300, 4), [4, 0, 3]), ((40, 2, 16, 4, 128, 60, 4), [1, 4]), ((70, 2, 4, 1, 192, 30, 3), [3, 2])])
def test_nine_to_sixteen_rows_of_padded_streams(call, tokens, dtype):
    c = Case(dtype, *call, tokens=tokens, layout="packed")
    try:
        c.run().verify(layers=[0, call[0] - 1])
    finally:
        c.close()
