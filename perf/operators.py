"""The operators of the language model's decode step: what they compute, in plain torch, beside the calls of the library.

Four operators (include/earlytom_decode.h):

  append     rows of keys and values go into a paged cache, rotated on the way and quantised to e4m3 if the cache is
  read       rows of the cache come back as bf16
  attention  one new token of each sequence against its cached keys and values
  linear     a dense layer for few rows, with bias, activation, residual or gate in its epilogue

A cache is data [n_pages][2 (keys, values)][kv_heads][page_size][head_dim], bf16 or e4m3; an e4m3 cache has one power of
two for each (position, head) of keys and of values: scale [n_pages][2][kv_heads][page_size], a byte b for 2^(b - 127).
block_table [n_seq][max_pages] names the pages of a sequence in order.

Sizes: 28 query heads on 4 key / value heads of 128, hidden 3584, feed-forward 18944 are the language model that the
framework's prefill is measured with (7 675 tokens is its uncompressed 32-frame prompt); the others are generic.
"""
import math
import random
from collections import namedtuple

import torch

own = False

F8 = torch.float8_e4m3fn
Run = namedtuple("Run", "n start")          # a sequence's appended or read rows: how many, from which position


# ---- cases ------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one more token of one conversation after a 32-frame video: launch latency
        dict(name="append 1 token", op="append", n_seq=1, rows=1, far=7675, heads=28, kv_heads=4, head_dim=128,
             page=64, e4m3=False, theta=1e6, mix=1),
        # one more token of 64 conversations, into a quantised cache
        dict(name="append 64 tokens e4m3", op="append", n_seq=64, rows=1, far=16000, heads=28, kv_heads=4, head_dim=128,
             page=16, e4m3=True, theta=1e6, mix=2),
        # the keys and values that a prefill left behind (rotated already) move into a quantised cache
        dict(name="append prompt 7675 e4m3", op="append", n_seq=1, rows=7675, far=0, heads=0, kv_heads=4, head_dim=128,
             page=64, e4m3=True, theta=0.0, mix=3),
        # chunks of eight prompts, ragged, rotated on their way into the cache
        dict(name="append 8 prompts bf16", op="append", n_seq=8, rows=4001, far=9000, heads=28, kv_heads=4, head_dim=128,
             page=32, e4m3=False, theta=1e6, mix=4),
        # a cached prompt comes back as rows
        dict(name="read 7675 e4m3", op="read", n_seq=1, rows=7675, far=0, kv_heads=4, head_dim=128, page=64, e4m3=True, mix=5),
        # ragged parts of sixteen caches, full-width heads of a small model
        dict(name="read 16 ragged bf16", op="read", n_seq=16, rows=5003, far=700, kv_heads=16, head_dim=64, page=16,
             e4m3=False, mix=6),
        # the first words of one conversation: launch latency
        dict(name="attention 1 x 61 bf16", op="attention", n_seq=1, longest=61, ragged=False, heads=28, kv_heads=4,
             head_dim=128, page=16, e4m3=False, mix=7),
        # one long video: a single sequence has to fill the card
        dict(name="attention 1 x 100003 bf16", op="attention", n_seq=1, longest=100003, ragged=False, heads=28, kv_heads=4,
             head_dim=128, page=64, e4m3=False, mix=8),
        # a serving batch of conversations about videos, lengths spread, some slots empty, quantised cache
        dict(name="attention 64 ragged e4m3", op="attention", n_seq=64, longest=16001, ragged=True, heads=28, kv_heads=4,
             head_dim=128, page=32, e4m3=True, mix=9),
        # a small model with as many key / value heads as query heads
        dict(name="attention 24 mha bf16", op="attention", n_seq=24, longest=2049, ragged=True, heads=16, kv_heads=16,
             head_dim=64, page=16, e4m3=False, mix=10),
        # query / key / value projection of one token
        dict(name="linear 1 x 3584 x 4608", op="linear", m=1, k=3584, n=4608, epilogue=0),
        # gate and up projection of a batch, gated in the epilogue
        dict(name="linear 19 x 3584 x 37888 gated", op="linear", m=19, k=3584, n=37888, epilogue=4),
    ]


def _log(rng, lo, hi):
    """A whole number, spread evenly over the logarithm of its range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attention", "attention", "linear"])
    if op == "linear":
        epilogue = rng.choice([0, 1, 2, 4])
        k = 8 * _log(rng, 16, 18944 // 8)
        n = 256 * _log(rng, 1, 37888 // 256) if epilogue == 4 else _log(rng, 64, 37888)
        return dict(op="linear", m=rng.randint(1, 32), k=k, n=max(256 if epilogue == 4 else 64, min(n, 100_000_000 // k // 256 * 256)),
                    epilogue=epilogue)
    kv_heads, group = rng.choice([(1, 8), (2, 1), (2, 6), (4, 7), (4, 4), (8, 1), (8, 4), (8, 5), (16, 1), (1, 23), (3, 12)])
    head_dim, page, e4m3, mix = rng.choice([64, 128]), rng.choice([16, 32, 64, 128]), rng.random() < 0.5, rng.randrange(1 << 20)
    width = kv_heads * head_dim
    if op == "attention":
        n_seq = _log(rng, 1, 96)
        longest = _log(rng, 1, max(16, min(100_000, 150_000_000 // (width * n_seq))))
        return dict(op=op, n_seq=n_seq, longest=longest, ragged=rng.random() < 0.7, heads=group * kv_heads, kv_heads=kv_heads,
                    head_dim=head_dim, page=page, e4m3=e4m3, mix=mix)
    n_seq = _log(rng, 1, 64)
    if op == "append":
        heads = group * kv_heads
        rows = _log(rng, 1, max(2, min(8000, 60_000_000 // ((heads + 2 * kv_heads) * head_dim * n_seq))))
        return dict(op=op, n_seq=n_seq, rows=rows, far=_log(rng, 1, 60_000), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                    page=page, e4m3=e4m3, theta=rng.choice([1e4, 5e5, 1e6]), mix=mix)
    rows = _log(rng, 1, max(2, min(8000, 30_000_000 // (width * n_seq))))
    return dict(op=op, n_seq=n_seq, rows=rows, far=_log(rng, 1, 60_000), kv_heads=kv_heads, head_dim=head_dim, page=page,
                e4m3=e4m3, mix=mix)


def _runs(case):
    """The rows of each sequence: between half and all of case["rows"], from a position up to case["far"]."""
    r = random.Random(case["mix"])
    n, most, far = case["n_seq"], case["rows"], case["far"]
    return [Run(most if n == 1 else r.randint((most + 1) // 2, most), far if n == 1 else r.randint(0, far)) for _ in range(n)]


def _lengths(case):
    """Cached positions of each sequence; a ragged batch has short and long ones and an empty slot."""
    if not case["ragged"]:
        return [case["longest"]] * case["n_seq"]
    r = random.Random(case["mix"])
    got = [int(round(case["longest"] * r.random() ** 2)) for _ in range(case["n_seq"])]
    got[0] = case["longest"]
    if case["n_seq"] > 2:
        got[1], got[2] = 0, 1
    return got


def work(case):
    if case["op"] == "linear":
        m, k, n, e = case["m"], case["k"], case["n"], case["epilogue"]
        out = m * n * (8 if e == 2 else 2) // (2 if e == 4 else 1)
        return {"bytes": 2 * k * (m + n) + 4 * n + out, "flops": 2 * m * k * n}
    width = case["kv_heads"] * case["head_dim"]
    cell = 2 * (width + case["kv_heads"]) if case["e4m3"] else 4 * width      # a position's keys and values
    if case["op"] == "attention":
        total, q = sum(_lengths(case)), case["heads"] * case["head_dim"]
        return {"bytes": total * cell + case["n_seq"] * (4 * q + 4 * case["heads"]), "flops": 4 * total * q}
    rows = sum(x.n for x in _runs(case))
    if case["op"] == "read":
        return {"bytes": rows * (cell + 4 * width), "flops": rows * 2 * width}
    q = case["heads"] * case["head_dim"]
    return {"bytes": rows * (cell + 4 * width + 4 * q), "flops": rows * 3 * (q + width)}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "linear":
        return _prepare_linear(case, gen)
    page, kv_heads, head_dim = case["page"], case["kv_heads"], case["head_dim"]
    s = dict(case=case, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if case["op"] == "attention":
        lens = _lengths(case)
        used, first = [-(-n // page) for n in lens], [0] * len(lens)
        max_pages = max(1, max(used))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["q"] = _normal(gen, case["n_seq"], case["heads"] * head_dim)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((case["n_seq"], case["heads"]), dtype=torch.float32, device="cuda")
        s["workspace"] = torch.empty(4 << 20, dtype=torch.uint8, device="cuda")
    else:
        runs = _runs(case)
        first = [x.start // page for x in runs]
        used = [(x.start + x.n - 1) // page + 1 - f for x, f in zip(runs, first)]
        max_pages = max(f + u for f, u in zip(first, used))
        offsets = [0]
        for x in runs:
            offsets.append(offsets[-1] + x.n)
        s["start"] = torch.tensor([x.start for x in runs], dtype=torch.int32, device="cuda")
        # a decode step has one row for each sequence and needs no offsets
        s["offsets"] = None if case["rows"] == 1 else torch.tensor(offsets, dtype=torch.int32, device="cuda")
        s["rows"] = offsets[-1]
    n_pages = sum(used) + 3
    # the pages that matter are scattered over the cache; the other entries of the table name page 0
    perm = torch.randperm(n_pages - 1, device="cuda", generator=gen).to(torch.int32) + 1
    table = torch.zeros((case["n_seq"], max_pages), dtype=torch.int32, device="cuda")
    at = 0
    for i, (f, u) in enumerate(zip(first, used)):
        table[i, f:f + u] = perm[at:at + u]
        at += u
    s["table"] = table
    s["cache"], s["scale"] = _random_cache(gen, n_pages, kv_heads, page, head_dim, case["e4m3"])
    if case["op"] == "append":
        s["qkv"] = _normal(gen, s["rows"], (case["heads"] + 2 * kv_heads) * head_dim)
        s["q_out"] = torch.empty((s["rows"], case["heads"] * head_dim), dtype=torch.bfloat16, device="cuda") if case["heads"] else None
    elif case["op"] == "read":
        s["out"] = torch.empty((s["rows"], 2 * kv_heads * head_dim), dtype=torch.bfloat16, device="cuda")
    return s


def _normal(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16)


def _random_cache(gen, n_pages, kv_heads, page, head_dim, e4m3):
    data = _normal(gen, n_pages, 2, kv_heads, page, head_dim)
    if not e4m3:
        return data, None
    codes, scale = torch.empty_like(data, dtype=F8), torch.empty(data.shape[:-1], dtype=torch.uint8, device="cuda")
    for at in range(0, n_pages, 4096):
        x = data[at:at + 4096].float()
        # tokens differ in size, as keys and values do
        x = x * torch.exp2(torch.randint(-3, 4, x.shape[:-1], device="cuda", generator=gen).float()).unsqueeze(-1)
        c, b = _quantise(x)
        codes[at:at + 4096].view(torch.uint8).copy_(c.view(torch.uint8))
        scale[at:at + 4096] = b
    return codes, scale


def _prepare_linear(case, gen):
    m, k, n, e = case["m"], case["k"], case["n"], case["epilogue"]
    w = torch.randn((n, k), device="cuda", generator=gen, dtype=torch.bfloat16).mul_(1 / math.sqrt(k))
    s = dict(case=case, a=_normal(gen, m, k), w=w, bias=torch.randn(n, device="cuda", generator=gen) * 0.02)
    if e == 2:
        s["c"] = torch.randn((m, n), device="cuda", generator=gen)
    else:
        s["c"] = torch.empty((m, n // 2 if e == 4 else n), dtype=torch.bfloat16, device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2605_30010_b200 import binding as B
    case = s["case"]
    if case["op"] == "linear":
        return B.et_linear_rows(s["a"], s["w"], s["bias"], case["epilogue"], c=s["c"])
    if case["op"] == "append":
        B.et_kv_append(s["cache"], s["scale"], s["qkv"], case["heads"], s["table"], s["start"], row_offsets=s["offsets"],
                       theta=case["theta"], q_out=s["q_out"], status=s["status"])
        return _append_outputs(s)
    if case["op"] == "read":
        return B.et_kv_read(s["cache"], s["scale"], s["table"], s["start"], s["rows"], row_offsets=s["offsets"], out=s["out"],
                            status=s["status"])
    B.et_attention_paged(s["q"], case["heads"], s["cache"], s["scale"], s["table"], s["lens"], out=s["out"], lse=s["lse"],
                         workspace=s["workspace"], status=s["status"])
    return dict(out=s["out"], lse=s["lse"])


def _append_outputs(s):
    out = dict(cache=s["cache"])
    if s["scale"] is not None:
        out["scale"] = s["scale"].view(torch.float8_e8m0fnu)
    if s["q_out"] is not None:
        out["q"] = s["q_out"]
    return out


def _run_plain(s):
    return {"linear": _plain_linear, "append": _plain_append, "read": _plain_read, "attention": _plain_attention}[s["case"]["op"]](s)


def _plain_linear(s):
    e = s["case"]["epilogue"]
    y = s["a"].float() @ s["w"].float().T + s["bias"]
    if e == 1:
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    elif e == 2:
        return s["c"].add_(y)
    elif e == 4:      # weight rows: 32 of the gate, then 32 of the same outputs' up projection, and so on
        y = y.view(y.shape[0], -1, 2, 32)
        gate, up = y[:, :, 0].reshape(y.shape[0], -1), y[:, :, 1].reshape(y.shape[0], -1)
        y = gate / (1 + torch.exp(-gate)) * up
    return s["c"].copy_(y)


def _pow2(e):
    """2^e as fp32 for whole e in [-127, 127], exactly: by its bits, since a library's power may be one step off."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _quantise(x):
    """fp32 rows [..., d] -> (e4m3 codes, byte b): the smallest power of two 2^(b - 127) that brings the row within +-448."""
    top = x.abs().amax(-1)
    mantissa, exponent = torch.frexp(top)                    # top = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875).to(exponent.dtype)  # 448 = 0.875 * 2^9
    e = torch.where(top > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    return (x * _pow2(-e).unsqueeze(-1)).to(F8), (e + 127).to(torch.uint8)


def _values(data, scale):
    """Cached rows as the fp32 values that they stand for."""
    if scale is None:
        return data.float()
    return data.float() * _pow2(scale.to(torch.int32) - 127).unsqueeze(-1)


def _places(s, rows):
    """(page, place in the page, position) of each row."""
    r = torch.arange(rows, device="cuda")
    if s["offsets"] is None:
        seq, pos = r, s["start"].long()
    else:
        off = s["offsets"].long()
        seq = torch.searchsorted(off[1:], r, right=True)
        pos = s["start"].long()[seq] + r - off[seq]
    page = s["case"]["page"]
    return s["table"].long()[seq, pos // page], pos % page, pos


def _rotate(x, pos, theta):
    """Rotate-half rotary embedding of x [rows][heads][d]; angles in 64 bits, since positions are far."""
    half = x.shape[-1] // 2
    turn = theta ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    angle = pos.double().unsqueeze(-1) * turn
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_append(s):
    case = s["case"]
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["head_dim"]
    page, place, pos = _places(s, s["rows"])
    x = s["qkv"].float().view(s["rows"], heads + 2 * kv_heads, d)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    if case["theta"] > 0:
        q, k = _rotate(q, pos, case["theta"]), _rotate(k, pos, case["theta"])
    if s["q_out"] is not None:
        s["q_out"].copy_(q.reshape(s["rows"], -1))
    both = torch.stack([k, v], 1)                            # [rows][2][kv_heads][d]
    if case["e4m3"]:
        codes, b = _quantise(both)
        s["cache"].view(torch.uint8).permute(0, 3, 1, 2, 4)[page, place] = codes.view(torch.uint8)
        s["scale"].permute(0, 3, 1, 2)[page, place] = b
    else:
        s["cache"].permute(0, 3, 1, 2, 4)[page, place] = both.to(torch.bfloat16)
    return _append_outputs(s)


def _plain_read(s):
    page, place, _ = _places(s, s["rows"])
    data = s["cache"].view(torch.uint8 if s["case"]["e4m3"] else torch.bfloat16).permute(0, 3, 1, 2, 4)[page, place]
    if s["case"]["e4m3"]:
        data = _values(data.view(F8), s["scale"].permute(0, 3, 1, 2)[page, place])
    return s["out"].copy_(data.reshape(s["rows"], -1))


def _plain_attention(s):
    case = s["case"]
    n, heads, kv_heads, d, table = case["n_seq"], case["heads"], case["kv_heads"], case["head_dim"], s["table"].long()
    longest = table.shape[1] * case["page"]
    data = s["cache"].view(torch.uint8 if case["e4m3"] else torch.bfloat16)[table]      # [n][pages][2][kv_heads][page][d]
    data = _values(data.view(F8), s["scale"][table]) if case["e4m3"] else data.float()
    data = data.permute(2, 0, 3, 1, 4, 5).reshape(2, n, kv_heads, longest, d)
    live = torch.arange(longest, device="cuda") < s["lens"].unsqueeze(1)
    score = s["q"].float().view(n, kv_heads, -1, d) @ data[0].transpose(-1, -2) / math.sqrt(d)
    score = score.masked_fill(~live[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    out = p @ data[1].masked_fill(~live[:, None, :, None], 0) / torch.where(total > 0, total, torch.ones_like(total))
    s["out"].copy_(out.reshape(n, heads * d))
    s["lse"].copy_((torch.log(total) + top).reshape(n, heads))
    return dict(out=s["out"], lse=s["lse"])


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "append": _exact_append, "read": _exact_read, "attention": _exact_attention}[case["op"]](s)


def _exact_linear(s):
    e, bias = s["case"]["epilogue"], s["bias"].double()
    y = torch.cat([torch.nn.functional.linear(s["a"].double(), s["w"][i:i + 4096].double(), bias[i:i + 4096])
                   for i in range(0, s["w"].shape[0], 4096)], 1)
    if e == 1:
        return torch.nn.functional.gelu(y, approximate="tanh")
    if e == 2:
        return s["c"].double() + y
    if e == 4:
        parts = y.split(32, 1)
        return torch.cat([torch.nn.functional.silu(g) * u for g, u in zip(parts[::2], parts[1::2])], 1)
    return y


def _code_values():
    """What each of the 256 e4m3 codes stands for."""
    got = []
    for c in range(256):
        sign, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        got.append(math.nan if c & 127 == 127 else sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)))
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _two_to(e):
    """2^e in 64 bits for whole e in [-160, 160], from a table of exact powers."""
    return torch.tensor([2.0 ** i for i in range(-160, 161)], dtype=torch.float64, device="cuda")[e.long() + 160]


def _seq_rows(s, i, first, n):
    """Positions first .. first + n - 1 of sequence i as row numbers of the cache's (page, place) pairs."""
    page = s["case"]["page"]
    pos = torch.arange(first, first + n, device="cuda")
    return s["table"][i].long()[torch.div(pos, page, rounding_mode="floor")], pos - torch.div(pos, page, rounding_mode="floor") * page


def _seq_values(s, which, i, first, n):
    """[kv_heads][n][d] in 64 bits."""
    pages, place = _seq_rows(s, i, first, n)
    if s["scale"] is None:
        return torch.stack([s["cache"][pages, which, h, place].double() for h in range(s["cache"].shape[2])])
    codes = s["cache"].view(torch.uint8)
    return torch.stack([_code_values()[codes[pages, which, h, place].long()]
                        * _two_to(s["scale"][pages, which, h, place].long() - 127).unsqueeze(-1) for h in range(codes.shape[2])])


def _exact_attention(s):
    case = s["case"]
    n, heads, kv_heads, d = case["n_seq"], case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.zeros((n, heads, d), dtype=torch.float64, device="cuda")
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device="cuda")
    for i, length in enumerate(_lengths(case)):
        if length == 0:
            continue
        k, v = (_seq_values(s, which, i, 0, length).repeat_interleave(heads // kv_heads, 0) for which in (0, 1))
        z = torch.einsum("hd,hnd->hn", s["q"][i].view(heads, d).double(), k) * d ** -0.5
        lse[i] = torch.logsumexp(z, -1)
        out[i] = torch.einsum("hn,hnd->hd", torch.softmax(z, -1), v)
    return dict(out=out.view(n, heads * d), lse=lse)


def _exact_read(s):
    parts = [torch.stack([_seq_values(s, which, i, x.start, x.n) for which in (0, 1)]) for i, x in enumerate(_runs(s["case"]))]
    return torch.cat([p.permute(2, 0, 1, 3).reshape(p.shape[2], -1) for p in parts])


def _exact_append(s):
    case = s["case"]
    heads, kv_heads, d, half = case["heads"], case["kv_heads"], case["head_dim"], case["head_dim"] // 2
    cache = _code_values()[s["cache"].view(torch.uint8).long()] if case["e4m3"] else s["cache"].double()
    scale = _two_to(s["scale"].long() - 127) if case["e4m3"] else None
    x = s["qkv"].double().view(s["rows"], heads + 2 * kv_heads, d)
    pos = torch.cat([torch.arange(r.start, r.start + r.n, device="cuda") for r in _runs(case)]).double()
    if case["theta"] > 0:
        i = torch.arange(half, device="cuda", dtype=torch.float64)
        turned = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[:, None] * torch.exp(-2 * i / d * math.log(case["theta"])))
        z = torch.complex(x[:, :heads + kv_heads, :half], x[:, :heads + kv_heads, half:]) * turned[:, None]
        x = torch.cat([torch.cat([z.real, z.imag], -1), x[:, heads + kv_heads:]], 1)
    at = 0
    for i, r in enumerate(_runs(case)):
        pages, place = _seq_rows(s, i, r.start, r.n)
        for which in (0, 1):
            for h in range(kv_heads):
                row = x[at:at + r.n, heads + which * kv_heads + h]
                if case["e4m3"]:
                    size = _two_to(torch.ceil(torch.log2(row.abs().amax(-1) / 448)).clamp(-127, 127))
                    y = row / size[:, None]
                    step = _two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)      # three mantissa bits
                    cache[pages, which, h, place] = torch.round(y / step) * step
                    scale[pages, which, h, place] = size
                else:
                    cache[pages, which, h, place] = row
        at += r.n
    got = dict(cache=cache)
    if scale is not None:
        got["scale"] = scale
    if heads:
        got["q"] = x[:, :heads].reshape(s["rows"], heads * d)
    return got
