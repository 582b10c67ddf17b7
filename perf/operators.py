"""The operators a model's forward needs around the memory pot, as cases that can be timed and compared.

``chunk``    a chunk of new tokens attends to the pot's rows and, causally, to itself (``ipot_chunk_attention``): what a
             layer does with every chunk of a prompt between two distillations, and with every generated token;
``blocks``   one generated token attends to the blocks of the pot that a cheap bound selects (``ipot_decode_attention_blocks``);
``append``   rows go into a pot that keeps those bounds (``ipot_append_chunk`` after ``ipot_enable_blocks``);
``rotate``   a chunk's queries and keys are rotated at their positions (``ipot_rope_rows``);
``tables``   the cosines and sines for that (``ipot_rope_tables``).

Sizes are those of ``inputs.CONFIGS``, of the benchmark's workloads and of the tests, and generic odd ones.  With ``own`` false
every operator is computed from elementary torch operations.  ``exact`` computes it unit by unit in 64 bits.
"""
import math

import numpy as np
import torch

own = False

_HEADS = dict(dtype="bf16", layers=1, batch=1, Hq=32, Hkv=8, d=128)
# "len" rows in the pot, "n" new tokens; "packed": rows of a token lie together ([.., token, head, d]) instead of those of a
# head; "padded": the streams of the batch have different numbers of tokens, the rows behind them are padding
_CHUNK = dict(_HEADS, kind="chunk", packed=False, padded=False)
_TABLES = dict(kind="tables", base=10000.0, factor=1.0, original=0, low=0.0, high=0.0)


def listed():
    return [
        # a serving batch: four streams' chunks over a pot of 8192 slots that is three quarters full
        dict(_CHUNK, name="chunk_batch4", batch=4, len=6144, n=2048),
        # one generated token of one layer, together with its own key and value: launch and latency
        dict(_CHUNK, name="chunk_one_token", len=4095, n=1),
        # nothing is a multiple of anything, three prompts of different lengths, rows as a projection leaves them
        dict(_CHUNK, name="chunk_ragged", layers=2, batch=3, Hq=12, Hkv=4, d=96, len=1999, n=333, packed=True, padded=True),
        # a toy model in fp32
        dict(_CHUNK, name="chunk_f32", dtype="f32", Hq=8, d=64, Hkv=2, len=256, n=256),
        # a token of generation over a long pot, one layer of a 70B model, an eighth of the rows
        dict(_HEADS, name="blocks_one_layer", kind="blocks", Hq=64, len=16384, rows=64, blocks=32),
        # all 32 layers of a 7B model's pot in one call, a quarter of the rows
        dict(_HEADS, name="blocks_32_layers", kind="blocks", layers=32, len=4096, rows=32, blocks=32),
        # a chunk's rows into the pot of all 32 layers, bounds kept
        dict(_HEADS, name="append_32_layers", kind="append", layers=32, n=2048, rows=32),
        # the same for a few odd rows in fp32
        dict(_HEADS, name="append_ragged_f32", kind="append", dtype="f32", layers=5, batch=3, Hq=12, Hkv=4, d=64, n=999, rows=16),
        # queries and keys of one generated token: launch and latency
        dict(_HEADS, name="rotate_one_token", kind="rotate", n=1, rotary=128, pairing="half", packed=False, padded=False),
        # queries and keys of 16 streams' chunks, half of every head rotated
        dict(_HEADS, name="rotate_batch16", kind="rotate", batch=16, n=2048, rotary=64, pairing="interleaved", packed=True, padded=True),
        # the tables of the largest pot, scaled for long contexts by wavelength
        dict(_TABLES, name="tables_pot", dtype="bf16", rotary=128, first=0, n=32768, base=500000.0, scaling="bands", factor=8.0,
             original=8192, low=1.0, high=4.0),
        # far positions in fp32, an odd number of frequencies
        dict(_TABLES, name="tables_far_f32", dtype="f32", rotary=90, first=1000003, n=999, scaling="ramp", factor=16.0, original=4096,
             low=1.0, high=32.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_heads(rng):
    f32, hkv = rng.random() < 0.2, rng.choice((1, 2, 4, 4, 8, 8, 8))
    return dict(dtype="f32" if f32 else "bf16", layers=_log_int(rng, 1, 32), batch=_log_int(rng, 1, 16),
                Hq=hkv * rng.choice((1, 2, 3, 4, 4, 4, 5, 7, 8)), Hkv=hkv, d=rng.choice((32, 64, 96, 128, 128, 128, 128, 256)))


def _draw_chunk(rng):
    n = rng.choice((1, 1, _log_int(rng, 2, 64), _log_int(rng, 64, 4096), _log_int(rng, 64, 4096)))
    return dict(_CHUNK, **_draw_heads(rng), len=rng.choice((0, _log_int(rng, 1, 16384), _log_int(rng, 500, 16384))), n=n,
                packed=rng.random() < 0.5, padded=rng.random() < 0.25)


def _draw_blocks(rng):
    n, rows = _log_int(rng, 100, 32768), rng.choice((16, 32, 64, 128))
    total = -(-n // rows)
    return dict(_draw_heads(rng), kind="blocks", len=n, rows=rows, blocks=max(1, min(total, int(total * rng.uniform(0.03, 0.5)))))


def _draw_append(rng):
    return dict(_draw_heads(rng), kind="append", n=_log_int(rng, 1, 8192), rows=rng.choice((16, 32, 64, 128)))


def _draw_rotate(rng):
    c = _draw_heads(rng)
    return dict(c, kind="rotate", n=_log_int(rng, 1, 4096), rotary=rng.choice((c["d"], c["d"], c["d"] // 2, c["d"] // 4, c["d"] - 6)),
                pairing=rng.choice(("half", "interleaved")), packed=rng.random() < 0.5, padded=rng.random() < 0.25)


def _draw_tables(rng):
    scaling = rng.choice(("plain", "linear", "stretched", "bands", "ramp"))
    return dict(_TABLES, dtype=rng.choice(("bf16", "f32")), rotary=2 * rng.randint(8, 128), first=rng.choice((0, 0, rng.randrange(1 << 24))),
                n=_log_int(rng, 16, 131072), base=rng.choice((10000.0, 500000.0, 1000000.0)), scaling=scaling,
                factor=1.0 if scaling == "plain" else rng.choice((2.0, 4.0, 8.0, 16.0, 40.0)), original=rng.choice((4096, 8192, 32768)), low=1.0,
                high=4.0 if scaling == "bands" else 32.0)


def _cost(c):
    """Rough seconds of the plain form, to keep drawn cases below the largest listed one of their kind."""
    w = work(c)
    if c["kind"] != "chunk":
        return w["bytes"]
    return c["layers"] * c["batch"] * c["Hq"] * c["n"] * (c["len"] + c["n"]) * (c["d"] + 64)


def draw(rng):
    kind = rng.choice((_draw_chunk, _draw_chunk, _draw_chunk, _draw_blocks, _draw_blocks, _draw_append, _draw_rotate, _draw_tables))
    while True:
        c = kind(rng)
        if _cost(c) <= max(_cost(x) for x in listed() if x["kind"] == c["kind"]):
            return c


def _units(c):
    return c["layers"] * c["batch"] * c["Hkv"]


def _elem(c):
    return 4 if c["dtype"] == "f32" else 2


def _tokens(c):
    """Tokens of every stream: all of them, or fewer and fewer, down to none where the batch is large."""
    B, n = c["batch"], c["n"]
    return [n - (n * b) // B for b in range(B)] if c["padded"] else [n] * B


def work(case):
    c = case
    if c["kind"] == "tables":
        entries = c["n"] * (c["rotary"] // 2)
        return {"bytes": 2 * entries * _elem(c), "flops": 4 * entries}
    units, G, row = _units(c), c["Hq"] // c["Hkv"], c["d"] * _elem(c)
    if c["kind"] == "chunk":
        heads, out = c["layers"] * c["Hkv"], {"bytes": 0, "flops": 0}
        for t in _tokens(c):
            if t:
                out["bytes"] += heads * ((2 * c["len"] + 2 * t + 2 * G * t) * row + 4 * G * t)
                out["flops"] += heads * 4 * c["d"] * G * (t * c["len"] + t * (t + 1) // 2)
        return out
    if c["kind"] == "blocks":
        total = -(-c["len"] // c["rows"])
        used = min(c["len"], c["blocks"] * c["rows"])
        return {"bytes": units * ((2 * total + 2 * used + G) * row + G * (4 * c["d"] + 4) + 4 * c["blocks"]),
                "flops": units * c["d"] * (4 * total + 4 * G * used)}
    if c["kind"] == "append":
        return {"bytes": units * (4 * c["n"] + 2 * -(-c["n"] // c["rows"])) * row, "flops": 2 * units * c["n"] * c["d"]}
    rows = c["layers"] * (c["Hq"] + c["Hkv"]) * sum(_tokens(c))
    return {"bytes": rows * 2 * row + min(4096, c["n"] + 17 * c["batch"]) * c["rotary"] * _elem(c), "flops": 3 * rows * c["rotary"]}


# ------------------------------------------------------------------ inputs


class _State:
    """Device buffers of the caller and, with ``own``, one pot."""


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _rows(g, c, heads, scale=1.0):
    """[layers][batch][heads][n][d], in memory as the case has it."""
    L, B, n, d = c["layers"], c["batch"], c["n"], c["d"]
    if c["packed"]:
        return (scale * _normal(g, (L, B, n, heads, d), _dtype(c))).transpose(2, 3)
    return scale * _normal(g, (L, B, heads, n, d), _dtype(c))


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _like(x):
    """Zeros with the strides of x."""
    return torch.zeros_like(x, memory_format=torch.preserve_format)


def _prepare_chunk(c, g, s):
    L, B, d = c["layers"], c["batch"], c["d"]
    shape = (L, B, c["Hkv"], c["len"], d)
    s.K, s.V = _normal(g, shape, _dtype(c)), _normal(g, shape, _dtype(c))
    s.q, s.k, s.v = _rows(g, c, c["Hq"], 1.5), _rows(g, c, c["Hkv"]), _rows(g, c, c["Hkv"])
    s.out = _like(s.q)
    s.lse = torch.zeros((L, B, c["Hq"], c["n"]), device="cuda")
    s.tokens = torch.tensor(_tokens(c), dtype=torch.int32, device="cuda") if c["padded"] else None


def _prepare_blocks(c, g, s):
    shape = (c["layers"], c["batch"], c["Hkv"], c["len"], c["d"])
    # neighbouring tokens resemble each other: every 64 rows share half of their variance
    common = _normal(g, shape[:3] + (-(-c["len"] // 64), c["d"]), torch.float32).repeat_interleave(64, dim=3)[:, :, :, :c["len"]]
    s.K = (0.7 * common + 0.7 * _normal(g, shape, torch.float32)).to(_dtype(c))
    s.V = _normal(g, shape, _dtype(c))
    s.lo, s.hi = _bounds(s.K, c["rows"])   # a program keeps them beside its rows
    s.q = 1.5 * _normal(g, (c["layers"], c["batch"], c["Hq"], c["d"]), _dtype(c))
    s.out = torch.zeros(s.q.shape, device="cuda")
    s.lse = torch.zeros(s.q.shape[:3], device="cuda")
    s.idx = torch.zeros(shape[:3] + (c["blocks"],), dtype=torch.int32, device="cuda")


def _prepare_append(c, g, s):
    shape = (c["layers"], c["batch"], c["Hkv"], c["n"], c["d"])
    s.K, s.V = _normal(g, shape, _dtype(c)), _normal(g, shape, _dtype(c))


def _prepare_rotate(c, g, s):
    B, n, half = c["batch"], c["n"], c["rotary"] // 2
    s.q, s.k = _rows(g, c, c["Hq"]), _rows(g, c, c["Hkv"])
    s.q_out, s.k_out = _like(s.q), _like(s.k)
    # every stream is somewhere else in its pot; the positions of padding are negative
    first = torch.randint(0, 17 * B, (B, 1), generator=g, device="cuda")
    at = torch.arange(n, device="cuda")[None, :]
    count = torch.tensor(_tokens(c), device="cuda")[:, None]
    s.positions = torch.where(at < count, first + at, torch.full_like(at, -1)).to(torch.int32)
    ang = torch.arange(n + 17 * B, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    s.cos, s.sin = ang.cos().to(_dtype(c)), ang.sin().to(_dtype(c))


def _prepare_tables(c, g, s):
    # the positions are the input: where the tables start depends on the seed
    s.first = c["first"] + int(torch.randint(0, 1024, (1,), generator=g, device="cuda"))
    s.cos, s.sin = (torch.zeros((c["n"], c["rotary"] // 2), dtype=_dtype(c), device="cuda") for _ in range(2))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = _State()
    s.c = case
    {"chunk": _prepare_chunk, "blocks": _prepare_blocks, "append": _prepare_append, "rotate": _prepare_rotate,
     "tables": _prepare_tables}[case["kind"]](case, g, s)
    if own:
        _own_state(case, s)
    return s


# ------------------------------------------------------------------ the plain forms


def _bounds(K, rows):
    """Smallest and largest value of every channel over blocks of `rows` rows."""
    n = K.shape[3]
    whole = -(-n // rows) * rows
    at = torch.arange(whole, device=K.device).clamp(max=n - 1)   # the last row again: it changes no bound
    x = K[:, :, :, at].unflatten(3, (whole // rows, rows))
    return x.amin(dim=4), x.amax(dim=4)


def _softmax(x, v):
    """(softmax(x) v, log sum exp x) over the last dimension of x."""
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, v) / l, (m + torch.log(l)).squeeze(-1)


def _grouped(q, c):
    """[L, B, Hq, n, d] -> [L, B, Hkv, G * n, d] in fp32, scaled."""
    L, B, n, d = c["layers"], c["batch"], q.shape[3], c["d"]
    return q.float().reshape(L, B, c["Hkv"], (c["Hq"] // c["Hkv"]) * n, d) / math.sqrt(d)


def _plain_chunk(c, s):
    L, B, n, N, d = c["layers"], c["batch"], c["n"], c["len"], c["d"]
    K, V = torch.cat([s.K, s.k], dim=3).float(), torch.cat([s.V, s.v], dim=3).float()
    x = torch.matmul(_grouped(s.q, c), K.transpose(3, 4)).view(L, B, c["Hkv"], -1, n, N + n)
    later = torch.arange(N + n, device="cuda")[None, :] > N + torch.arange(n, device="cuda")[:, None]
    x.masked_fill_(later, -math.inf)
    o, lse = _softmax(x.flatten(3, 4), V)
    o, lse = o.view(L, B, c["Hq"], n, d).to(_dtype(c)), lse.view(L, B, c["Hq"], n)
    if s.tokens is None:
        return o, lse
    there = torch.arange(n, device="cuda")[None, :] < s.tokens[:, None]   # rows of padding stay as they were
    return torch.where(there[None, :, None, :, None], o, s.out), torch.where(there[None, :, None, :], lse, s.lse)


def _plain_blocks(c, s):
    q = s.q.double().unflatten(2, (c["Hkv"], -1))
    # sum over the heads of sum_c max(q lo, q hi); in 64 bits, so that values next to the border fall on the same side
    bound = (s.hi.double() * q.clamp(min=0).sum(dim=3)[:, :, :, None]).sum(-1) + (s.lo.double() * q.clamp(max=0).sum(dim=3)[:, :, :, None]).sum(-1)
    bound[..., -1] = math.inf   # the newest block always
    order = torch.sort(bound, dim=-1, descending=True, stable=True).indices
    idx = torch.sort(order[..., :c["blocks"]], dim=-1).values
    rows = (idx[..., None] * c["rows"] + torch.arange(c["rows"], device="cuda")).flatten(3)
    there = rows < c["len"]
    at = rows.clamp(max=c["len"] - 1)[..., None].expand(-1, -1, -1, -1, c["d"])
    K, V = s.K.gather(3, at).float(), s.V.gather(3, at).float()
    x = torch.matmul(_grouped(s.q[:, :, :, None], c), K.transpose(3, 4)).masked_fill(~there[:, :, :, None], -math.inf)
    o, lse = _softmax(x, V)
    return o.reshape(s.out.shape), lse.reshape(s.lse.shape), idx.to(torch.int32)


def _plain_append(c, s):
    lo, hi = _bounds(s.K, c["rows"])
    return s.K.clone(), s.V.clone(), lo, hi


def _rotated(x, c, s, out):
    r = c["rotary"]
    at = s.positions.long().clamp(min=0)
    cos, sin = s.cos[at].float()[None, :, None], s.sin[at].float()[None, :, None]
    y = x.float()
    if c["pairing"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        z = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        z = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    z = torch.cat([z, y[..., r:]], dim=-1).to(_dtype(c))
    return torch.where((s.positions >= 0)[None, :, None, :, None], z, out)


def _frequencies(c):
    """Turns per position of every channel pair, in radians, and the factor on cosines and sines."""
    r, f = c["rotary"], c["factor"]
    i = torch.arange(r // 2, device="cuda", dtype=torch.float64)
    plain = c["base"] ** (-2.0 * i / r)
    if c["scaling"] == "linear":
        return plain / f, 1.0
    if c["scaling"] == "stretched":
        return (c["base"] * f ** (r / (r - 2.0))) ** (-2.0 * i / r), 1.0
    if c["scaling"] == "bands":
        turns = c["original"] * plain / (2 * math.pi)   # of a pair within the original context
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
        return plain * keep + plain / f * (1 - keep), 1.0
    if c["scaling"] == "ramp":
        at = lambda turns: r * math.log(c["original"] / (2 * math.pi * turns)) / (2 * math.log(c["base"]))  # noqa: E731
        first, last = max(math.floor(at(c["high"])), 0), min(math.ceil(at(c["low"])), r - 1)
        drop = ((i - first) / max(last - first, 0.001)).clamp(0, 1)
        return plain * (1 - drop) + plain / f * drop, 0.1 * math.log(f) + 1.0
    return plain, 1.0


def _plain_tables(c, s):
    w, magnitude = _frequencies(c)
    ang = (s.first + torch.arange(c["n"], device="cuda", dtype=torch.float64))[:, None] * w
    return (torch.cos(ang) * magnitude).to(_dtype(c)), (torch.sin(ang) * magnitude).to(_dtype(c))


# ------------------------------------------------------------------ the framework's calls


def _own_state(c, s):
    """The pot that a program holds, filled, and views of what a call leaves in it."""
    import sys

    from paper_2410_01518_b200 import ipot

    s.ipot = ipot
    if c["kind"] == "tables":
        return
    n = c["len"] if "len" in c else c["n"]

    class Pot:
        def __init__(self):
            self.h = None
            self.h = ipot.ipot_create_ex(max(n, 2), max(1, n // 2), c["layers"], c["Hq"], c["Hkv"], c["d"], batch=c["batch"],
                                         dtype=ipot.IPOT_F32 if c["dtype"] == "f32" else ipot.IPOT_BF16, nuc_slots=0, max_cap_rows=1)

        def __del__(self):
            if self.h is not None and not sys.is_finalizing():   # (at exit the binding is gone before the pots, and memory goes with the process)
                ipot.ipot_destroy(self.h)

        def view(self, addr, shape, dtype):
            memory = type("Memory", (), {})()
            memory.pot = self
            memory.__cuda_array_interface__ = {"shape": (math.prod(shape) * dtype.itemsize,), "typestr": "|u1", "data": (addr, False), "version": 2}
            return torch.as_tensor(memory, device="cuda").view(dtype).view(shape)

    s.pot = Pot()
    if c["kind"] in ("blocks", "append"):
        ipot.ipot_enable_blocks(s.pot.h, c["rows"])
    if c["kind"] in ("blocks", "chunk") and n:
        ipot.ipot_append_chunk(s.pot.h, s.K, s.V, n)
        ipot.ipot_sync_status(s.pot.h)
    if c["kind"] == "append":
        shape, slots = s.K.shape[:3], max(n, 2)
        K, V, _ = ipot.ipot_view(s.pot.h)
        lo, hi, _ = ipot.ipot_view_blocks(s.pot.h)
        blocks, used = -(-slots // c["rows"]), -(-n // c["rows"])
        s.views = [s.pot.view(a, shape + (slots, c["d"]), _dtype(c))[:, :, :, :n] for a in (K, V)]
        s.views += [s.pot.view(a, shape + (blocks, c["d"]), _dtype(c))[:, :, :, :used] for a in (lo, hi)]


def _own_chunk(c, s):
    s.ipot.ipot_chunk_attention(s.pot.h, 0, c["layers"], c["n"], s.q, s.k, s.v, s.out, s.lse, tokens=s.tokens,
                                q_strides=s.q.stride()[:4], k_strides=s.k.stride()[:4], v_strides=s.v.stride()[:4], out_strides=s.out.stride()[:4])
    return s.out, s.lse


def _own_blocks(c, s):
    s.ipot.ipot_decode_attention_blocks(s.pot.h, 0, c["layers"], s.q, c["blocks"], s.out, s.lse, s.idx)
    return s.out, s.lse, s.idx


def _own_append(c, s):
    s.ipot.ipot_reset(s.pot.h)
    s.ipot.ipot_append_chunk(s.pot.h, s.K, s.V, c["n"])
    return s.views


def _own_rotate(c, s):
    i = s.ipot
    i.ipot_rope_rows(s.pot.h, c["layers"], c["n"], s.cos, s.sin, s.cos.shape[0], c["rotary"],
                     i.IPOT_ROPE_HALF if c["pairing"] == "half" else i.IPOT_ROPE_INTERLEAVED, i.IPOT_F32 if c["dtype"] == "f32" else i.IPOT_BF16,
                     positions=s.positions, q=s.q, q_out=s.q_out, k=s.k, k_out=s.k_out, q_strides=s.q.stride()[:4], q_out_strides=s.q_out.stride()[:4],
                     k_strides=s.k.stride()[:4], k_out_strides=s.k_out.stride()[:4])
    return s.q_out, s.k_out


def _own_tables(c, s):
    i = s.ipot
    scaling = {"plain": i.IPOT_ROPE_PLAIN, "linear": i.IPOT_ROPE_LINEAR, "stretched": i.IPOT_ROPE_STRETCHED, "bands": i.IPOT_ROPE_BANDS,
               "ramp": i.IPOT_ROPE_RAMP}[c["scaling"]]
    i.ipot_rope_tables(s.cos, s.sin, s.first, c["n"], c["rotary"], i.IPOT_F32 if c["dtype"] == "f32" else i.IPOT_BF16, base=c["base"],
                       scaling=scaling, factor=c["factor"], original_len=c["original"], low=c["low"], high=c["high"])
    return s.cos, s.sin


def run(state):
    s, c = state, state.c
    if own:
        return {"chunk": _own_chunk, "blocks": _own_blocks, "append": _own_append, "rotate": _own_rotate, "tables": _own_tables}[c["kind"]](c, s)
    if c["kind"] == "chunk":
        return _plain_chunk(c, s)
    if c["kind"] == "blocks":
        return _plain_blocks(c, s)
    if c["kind"] == "append":
        return _plain_append(c, s)
    if c["kind"] == "rotate":
        return _rotated(s.q, c, s, s.q_out), _rotated(s.k, c, s, s.k_out)
    return _plain_tables(c, s)


# ------------------------------------------------------------------ the definitions, unit by unit in 64 bits


def _attend64(q, k, v, limit=None):
    """One query head over its rows; row t of q sees the first limit + t + 1 of them, or all."""
    x = torch.einsum("td,jd->tj", q.double(), k.double()) * q.shape[1] ** -0.5
    if limit is not None:
        x = torch.where(torch.ones_like(x, dtype=torch.bool).tril(limit), x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, dim=1)
    return torch.einsum("tj,jd->td", torch.exp(x - lse[:, None]), v.double()), lse


def _exact_attention(c, s, out, lse, rows_of):
    for l in range(c["layers"]):
        for b in range(c["batch"]):
            for h in range(c["Hq"]):
                t, k, v, limit = rows_of(l, b, h // (c["Hq"] // c["Hkv"]))
                q = s.q[l, b, h] if s.q.dim() == 5 else s.q[l, b, h:h + 1]
                if t:
                    o, e = _attend64(q[:t], k, v, limit)
                    if s.q.dim() == 5:
                        out[l, b, h, :t], lse[l, b, h, :t] = o, e
                    else:
                        out[l, b, h], lse[l, b, h] = o[0], e[0]


def _exact_chunk(c, s):
    tokens = _tokens(c)
    out, lse = torch.zeros(s.q.shape, device="cuda", dtype=torch.float64), torch.zeros(s.lse.shape, device="cuda", dtype=torch.float64)

    def rows_of(l, b, kv):
        t = tokens[b]
        return t, torch.cat([s.K[l, b, kv], s.k[l, b, kv, :t]]), torch.cat([s.V[l, b, kv], s.v[l, b, kv, :t]]), c["len"]

    _exact_attention(c, s, out, lse, rows_of)
    return out, lse


def _exact_blocks(c, s):
    total = -(-c["len"] // c["rows"])
    G = c["Hq"] // c["Hkv"]
    out, lse = torch.zeros(s.q.shape, device="cuda", dtype=torch.float64), torch.zeros(s.lse.shape, device="cuda", dtype=torch.float64)
    chosen = np.zeros(tuple(s.idx.shape), dtype=np.int32)
    for u in np.ndindex(*chosen.shape[:3]):
        q = s.q[u[0], u[1], u[2] * G:(u[2] + 1) * G].double().cpu().numpy()
        lo, hi = s.lo[u].double().cpu().numpy(), s.hi[u].double().cpu().numpy()
        bound = np.maximum(q[:, None] * lo[None], q[:, None] * hi[None]).sum(axis=(0, 2))
        best = sorted(range(total - 1), key=lambda b: (-bound[b], b))[:c["blocks"] - 1]
        chosen[u] = sorted(best + [total - 1])

    def rows_of(l, b, kv):
        at = (torch.from_numpy(chosen[l, b, kv]).cuda()[:, None] * c["rows"] + torch.arange(c["rows"], device="cuda")).flatten()
        at = at[at < c["len"]]
        return 1, s.K[l, b, kv][at], s.V[l, b, kv][at], None

    _exact_attention(c, s, out, lse, rows_of)
    return out, lse, torch.from_numpy(chosen)


def _exact_rotate(c, s):
    def turn(x):
        y, r = x.double().cpu().numpy().copy(), c["rotary"]
        w = s.cos.double().cpu().numpy() + 1j * s.sin.double().cpu().numpy()
        for b in range(c["batch"]):
            p = s.positions[b].cpu().numpy()
            for l in range(c["layers"]):
                z = y[l, b]
                first, second = (z[..., :r // 2], z[..., r // 2:r]) if c["pairing"] == "half" else (z[..., 0:r:2], z[..., 1:r:2])
                turned = (first + 1j * second) * w[np.maximum(p, 0)][None]
                first[...], second[...] = turned.real, turned.imag
            y[:, b, :, p < 0] = 0.0
        return torch.from_numpy(y)

    return turn(s.q), turn(s.k)


def _exact_tables(c, s):
    r, f, L = c["rotary"], c["factor"], c["original"]
    w = []
    for i in range(r // 2):
        plain = math.exp(-2.0 * i / r * math.log(c["base"]))
        slow, wave = plain / f, 2 * math.pi / plain
        if c["scaling"] == "plain":
            w.append(plain)
        elif c["scaling"] == "linear":
            w.append(slow)
        elif c["scaling"] == "stretched":   # the last pair turns `factor` times slower, the first as before
            w.append(plain * math.exp(-math.log(f) * 2 * i / (r - 2)))
        elif c["scaling"] == "bands":
            t = (L / wave - c["low"]) / (c["high"] - c["low"])
            w.append(plain if wave < L / c["high"] else slow if wave > L / c["low"] else (1 - t) * slow + t * plain)
        else:
            pair = [r * math.log(L / (turns * 2 * math.pi)) / (2 * math.log(c["base"])) for turns in (c["high"], c["low"])]
            first, last = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), r - 1)
            ramp = min(1.0, max(0.0, (i - first) / (last - first if last > first else 0.001)))
            w.append(slow * ramp + plain * (1 - ramp))
    magnitude = 0.1 * math.log(f) + 1.0 if c["scaling"] == "ramp" else 1.0
    z = magnitude * np.exp(1j * np.outer(np.arange(s.first, s.first + c["n"], dtype=np.float64), np.array(w)))
    return z.real.copy(), z.imag.copy()


def exact(case, seed):
    heads = case.get("layers", 1) * case.get("batch", 1) * case.get("Hq", 1)
    if (case["kind"] in ("chunk", "blocks") and heads > 8192) or (case["kind"] == "rotate" and work(case)["bytes"] > 1.5e9):
        return None   # too many units to go through one by one
    global own
    was, own = own, False   # the inputs alone
    s = prepare(case, seed)
    own = was
    if case["kind"] == "append":
        shape, n = s.K.shape, case["n"]
        pieces = [s.K[:, :, :, i:i + case["rows"]].double() for i in range(0, n, case["rows"])]
        return s.K.double(), s.V.double(), torch.stack([-(-p).amax(3) for p in pieces], 3), torch.stack([p.amax(3) for p in pieces], 3)
    return {"chunk": _exact_chunk, "blocks": _exact_blocks, "rotate": _exact_rotate, "tables": _exact_tables}[case["kind"]](case, s)
