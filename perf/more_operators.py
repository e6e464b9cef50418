"""The operators of serving from a paged cache: what they compute, in plain torch, beside the calls of the library.

Five operators (include/earlytom_decode.h, include/earlytom_pages.h):

  store      rows of keys and values go into a cache of 4 bits, rotated on the way, and come back as bf16
  attention  one new token of each sequence against its keys and values in a cache of 4 bits
  pages      sequences give pages back and take others; their tables, rows' offsets and slots follow
  select     beam search: the best continuations of each request's beams over the vocabulary
  reorder    the beams' tables follow the selection: pages are shared, half-filled ones are copied

A cache of 4 bits is codes [n_pages][2 (keys, values)][kv_heads][page_size][head_dim / 2], two a byte, the even value in the low
bits, and scale bf16 [n_pages][2][kv_heads][page_size][head_dim / 32]: a code c stands for (c - 8) times the scale of its 32.
block_table [n_seq][max_pages] names the pages of a sequence in order; refs [n_pages] counts the table entries that name a page.

Sizes: 28 query heads on 4 key / value heads of 128 and a vocabulary of 152 064 are the language model that the framework's
prefill is measured with (7 675 tokens is its uncompressed 32-frame prompt); the others are generic.
"""
import math
import random
from collections import namedtuple

import numpy as np
import torch

own = False

Run = namedtuple("Run", "n start")          # a sequence's stored rows: how many, from which position


# ---- cases ------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one more token of one conversation after a 32-frame video: launch latency
        dict(name="store 1 token", op="store", n_seq=1, rows=1, far=7675, heads=28, kv_heads=4, head_dim=128, page=64, theta=1e6,
             mix=1),
        # the keys and values that a prefill left behind (rotated already) move into the cache
        dict(name="store prompt 7675", op="store", n_seq=1, rows=7675, far=0, heads=0, kv_heads=4, head_dim=128, page=64, theta=0.0,
             mix=2),
        # chunks of eight prompts, ragged, rotated on their way
        dict(name="store 8 prompts", op="store", n_seq=8, rows=4001, far=9000, heads=28, kv_heads=4, head_dim=128, page=32, theta=1e6,
             mix=3),
        # the first words of one conversation: launch latency
        dict(name="attention 1 x 61", op="attention", n_seq=1, longest=61, ragged=False, heads=28, kv_heads=4, head_dim=128, page=16,
             mix=4),
        # one long video: a single sequence has to fill the card
        dict(name="attention 1 x 100003", op="attention", n_seq=1, longest=100003, ragged=False, heads=28, kv_heads=4, head_dim=128,
             page=64, mix=5),
        # a serving batch of conversations about videos, lengths spread, some slots empty
        dict(name="attention 64 ragged", op="attention", n_seq=64, longest=16001, ragged=True, heads=28, kv_heads=4, head_dim=128,
             page=32, mix=6),
        # a decode step: every conversation one token more or, after rejected drafts, a few
        dict(name="pages 64 x few tokens", op="pages", n_seq=64, longest=16001, page=64, turnover=0.0, mix=7),
        # a prefill step of a large server: most slots get a new prompt
        dict(name="pages 700 prompts", op="pages", n_seq=700, longest=7675, page=32, turnover=0.8, mix=8),
        # four beams of one request
        dict(name="select 1 x 4 bf16", op="select", n_req=1, beams=4, k=4, vocab=152064, fp32=False, done=0.0, mix=9),
        # a batch, some beams ended, twice as many candidates as beams
        dict(name="select 32 x 8 fp32", op="select", n_req=32, beams=8, k=16, vocab=152064, fp32=True, done=0.1, mix=10),
        # the four beams' pages after it, one layer of a 4-bit cache
        dict(name="reorder 1 x 4", op="reorder", n_req=1, beams=4, prompt=7675, grown=50, page=64, kv_heads=4, head_dim=128, bits=4,
             layers=1, mix=11),
        # a batch of beams, four layers of a bf16 cache
        dict(name="reorder 32 x 8", op="reorder", n_req=32, beams=8, prompt=1501, grown=77, page=32, kv_heads=4, head_dim=128, bits=16,
             layers=4, mix=12),
    ]


def _log(rng, lo, hi):
    """A whole number, spread evenly over the logarithm of its range."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "attention", "attention", "pages", "select", "reorder"])
    mix = rng.randrange(1 << 20)
    if op == "pages":
        n_seq, page = _log(rng, 1, 700), rng.choice([16, 32, 64, 128])
        longest = _log(rng, 1, max(2, min(30_000, 5_000_000 // n_seq)))
        return dict(op=op, n_seq=n_seq, longest=longest, page=page, turnover=rng.choice([0.0, 0.2, 0.8]), mix=mix)
    if op == "select":
        beams, vocab = rng.choice([1, 2, 3, 4, 5, 8, 12, 16]), _log(rng, 500, 200_000)
        return dict(op=op, n_req=_log(rng, 1, max(1, min(64, 30_000_000 // (beams * vocab)))), beams=beams,
                    k=rng.choice([beams, beams, 2 * beams, rng.randint(1, 32)]), vocab=vocab, fp32=rng.random() < 0.5,
                    done=rng.choice([0.0, 0.1, 0.4]), mix=mix)
    kv_heads, group = rng.choice([(1, 8), (2, 1), (2, 6), (4, 7), (4, 4), (8, 1), (8, 4), (8, 5), (16, 1), (1, 23), (3, 12)])
    head_dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    width = kv_heads * head_dim
    if op == "attention":
        n_seq = _log(rng, 1, 96)
        return dict(op=op, n_seq=n_seq, longest=_log(rng, 1, max(16, min(100_000, 150_000_000 // (width * n_seq)))),
                    ragged=rng.random() < 0.7, heads=group * kv_heads, kv_heads=kv_heads, head_dim=head_dim, page=page, mix=mix)
    if op == "store":
        n_seq, heads = _log(rng, 1, 64), group * kv_heads
        rows = _log(rng, 1, max(2, min(8000, 60_000_000 // ((heads + 2 * kv_heads) * head_dim * n_seq))))
        return dict(op=op, n_seq=n_seq, rows=rows, far=_log(rng, 1, 60_000), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                    page=page, theta=rng.choice([1e4, 5e5, 1e6]), mix=mix)
    n_req, beams = _log(rng, 1, 32), rng.choice([1, 2, 3, 4, 5, 8])
    most = max(page, 40_000_000 // (width * n_req))
    return dict(op=op, n_req=n_req, beams=beams, prompt=_log(rng, 1, min(20_000, most)), grown=_log(rng, 1, max(1, min(300, most // beams))),
                page=page, kv_heads=kv_heads, head_dim=head_dim, bits=rng.choice([4, 8, 16]), layers=rng.randint(1, 3), mix=mix)


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


def _turns(case):
    """(len, keep) of each sequence: the positions that it holds, and those that stay.  It gets as many as it gives up, so that a
    pass leaves as many pages in use as it found: a new prompt in place of an old one, drafts in place of rejected ones."""
    r = random.Random(case["mix"])
    got = []
    for i in range(case["n_seq"]):
        n = case["longest"] if i == 0 else int(round(case["longest"] * r.random()))
        if i % 16 == 5:
            got.append((-1, -1))                                       # a slot that is not in use
        elif r.random() < case["turnover"]:
            got.append((n, 0))
        else:
            got.append((n, max(0, n - (1 if i == 0 or r.random() < 0.7 else r.randint(0, 8)))))
    return got


def _beams(case):
    """Parents of a step's beams, as rows of the step before: some have several children, some none, one slot ends."""
    r = random.Random(case["mix"])
    got = []
    for q in range(case["n_req"]):
        got += [q * case["beams"] + int(case["beams"] * r.random() ** 1.7) for _ in range(case["beams"])]
    if len(got) > 8:
        got[r.randrange(len(got))] = -1
    return got


def _pages(n, page):
    return -(-n // page)


def _cell(case):
    """Bytes of a position's keys and values."""
    width = 2 * case["kv_heads"] * case["head_dim"]
    bits = case.get("bits", 4)
    return width * 2 if bits == 16 else width + 2 * case["kv_heads"] if bits == 8 else width // 2 + width // 16


def work(case):
    op = case["op"]
    if op == "select":
        rows = case["n_req"] * case["beams"]
        return {"bytes": rows * case["vocab"] * (4 if case["fp32"] else 2) + 5 * rows + 13 * case["n_req"] * case["k"],
                "flops": 3 * rows * case["vocab"]}
    if op == "pages":
        turns = _turns(case)
        moved = sum(_pages(max(n, 0), case["page"]) - _pages(max(k, 0), case["page"]) for n, k in turns)
        rows = sum(n - k for n, k in turns)
        return {"bytes": 4 * _pool(case) + 16 * moved + 20 * len(turns) + 4 * rows, "flops": _pool(case) + 4 * rows}
    if op == "reorder":
        n, parents = case["prompt"] + case["grown"], _beams(case)
        copies = sum(p >= 0 and p in parents[:b] for b, p in enumerate(parents)) if n % case["page"] else 0
        table = _pages(n, case["page"]) * len(parents)
        return {"bytes": 8 * table + 4 * _beam_pool(case) + copies * 2 * (n % case["page"]) * _cell(case) * case["layers"],
                "flops": 4 * table}
    width = case["kv_heads"] * case["head_dim"]
    q = case["heads"] * case["head_dim"]
    if op == "attention":
        total = sum(_lengths(case))
        return {"bytes": total * _cell(case) + case["n_seq"] * (4 * q + 4 * case["heads"]), "flops": 4 * total * q}
    rows = sum(x.n for x in _runs(case))
    return {"bytes": rows * (2 * _cell(case) + 8 * width + 4 * q), "flops": rows * (3 * (q + width) + 4 * width)}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"store": _prepare_store, "attention": _prepare_attention, "pages": _prepare_pages, "select": _prepare_select,
            "reorder": _prepare_reorder}[case["op"]](case, gen, np.random.default_rng(seed))


def _normal(gen, *shape):
    return torch.randn(shape, device="cuda", generator=gen, dtype=torch.bfloat16)


def _ints(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device="cuda")


def _random_cache(gen, n_pages, kv_heads, page, head_dim):
    """Codes and scales of rows whose sizes differ, as those of keys and values do."""
    codes = torch.empty((n_pages, 2, kv_heads, page, head_dim // 2), dtype=torch.uint8, device="cuda")
    scale = torch.empty((n_pages, 2, kv_heads, page, head_dim // 32), dtype=torch.bfloat16, device="cuda")
    for at in range(0, n_pages, 2048):
        x = _normal(gen, *scale[at:at + 2048].shape, 32).float()
        size = torch.exp2(torch.randint(-3, 4, x.shape[:-2], device="cuda", generator=gen).float())
        top = x.abs().amax(-1, keepdim=True)
        n = (torch.round(x * (7 / top)) + 8).to(torch.uint8)
        n = n.reshape(*n.shape[:-2], head_dim)
        codes[at:at + 2048] = n[..., ::2] | (n[..., 1::2] << 4)
        scale[at:at + 2048] = top[..., 0] / 7 * size[..., None]
    return codes, scale


def _scattered(gen, n_seq, first, used, spare=3):
    """A table whose entries first .. first + used - 1 name pages scattered over a cache; the others name page 0."""
    n_pages = sum(used) + spare
    perm = torch.randperm(n_pages - 1, device="cuda", generator=gen).to(torch.int32) + 1
    table = torch.zeros((n_seq, max(1, max(f + u for f, u in zip(first, used)))), dtype=torch.int32, device="cuda")
    at = 0
    for i, (f, u) in enumerate(zip(first, used)):
        table[i, f:f + u] = perm[at:at + u]
        at += u
    return table, n_pages


def _prepare_store(case, gen, rng):
    page, kv_heads, head_dim, heads = case["page"], case["kv_heads"], case["head_dim"], case["heads"]
    runs = _runs(case)
    first = [x.start // page for x in runs]
    table, n_pages = _scattered(gen, case["n_seq"], first, [(x.start + x.n - 1) // page + 1 - f for x, f in zip(runs, first)])
    rows = sum(x.n for x in runs)
    codes, scale = _random_cache(gen, n_pages, kv_heads, page, head_dim)
    return dict(case=case, rows=rows, table=table, codes=codes, scale=scale, status=_ints([0]), start=_ints([x.start for x in runs]),
                # a decode step has one row for each sequence and needs no offsets
                offsets=None if case["rows"] == 1 else _ints(np.cumsum([0] + [x.n for x in runs])),
                qkv=_normal(gen, rows, (heads + 2 * kv_heads) * head_dim),
                q_out=torch.empty((rows, heads * head_dim), dtype=torch.bfloat16, device="cuda") if heads else None,
                back=torch.empty((rows, 2 * kv_heads * head_dim), dtype=torch.bfloat16, device="cuda"))


def _prepare_attention(case, gen, rng):
    lens, n, heads = _lengths(case), case["n_seq"], case["heads"]
    table, n_pages = _scattered(gen, n, [0] * n, [_pages(x, case["page"]) for x in lens])
    codes, scale = _random_cache(gen, n_pages, case["kv_heads"], case["page"], case["head_dim"])
    q = _normal(gen, n, heads * case["head_dim"])
    return dict(case=case, lens=_ints(lens), table=table, codes=codes, scale=scale, status=_ints([0]), q=q, out=torch.empty_like(q),
                lse=torch.empty((n, heads), dtype=torch.float32, device="cuda"),
                workspace=torch.empty(4 << 20, dtype=torch.uint8, device="cuda"))


def _pool(case):
    """Pages of the cache: half as many again as the sequences hold."""
    return sum(_pages(max(n, 0), case["page"]) for n, _ in _turns(case)) * 3 // 2 + 64


def _prepare_pages(case, gen, rng):
    turns, page, n_pages, n_seq = _turns(case), case["page"], _pool(case), case["n_seq"]
    lens, keep = np.array([t[0] for t in turns]), np.array([t[1] for t in turns])
    used = -(-np.maximum(lens, 0) // page)
    live = np.arange(max(1, used.max())) < used[:, None]
    table = np.full(live.shape, -1)
    table[live] = rng.permutation(n_pages)[:used.sum()]
    # every fourth sequence shares the pages of its first words with the one before
    for s in range(1, n_seq, 4):
        same = min(used[s], used[s - 1], 3)
        table[s, :same] = table[s - 1, :same]
    # and somebody else holds some of the pages: beginnings of prompts that are kept for later ones
    refs = np.bincount(table[live], minlength=n_pages)
    refs[rng.random(n_pages) < 0.15] += 1
    rows = int((lens - keep).sum())
    return dict(case=case, refs=_ints(refs), table=_ints(table), lens=_ints(lens), keep=_ints(keep), add=_ints(lens - keep), rows=rows,
                new_len=_ints(lens), offsets=_ints([0] * (n_seq + 1)), slots=_ints([0] * rows), status=_ints([0]),
                workspace=torch.empty(4 * n_pages + 8 * n_seq, dtype=torch.uint8, device="cuda"))


def _prepare_select(case, gen, rng):
    n_req, beams, vocab, k = case["n_req"], case["beams"], case["vocab"], case["k"]
    rows = n_req * beams
    x = torch.empty((rows, vocab), dtype=torch.float32 if case["fp32"] else torch.bfloat16, device="cuda")
    for at in range(0, rows, 64):                                      # a few likely tokens stand out of the rest
        y = torch.randn(x[at:at + 64].shape, device="cuda", generator=gen)
        x[at:at + 64] = 2 * y + y.abs() ** 2.2 * 0.4
    score = torch.rand((n_req, beams), device="cuda", generator=gen).mul_(-20)
    done = torch.rand((n_req, beams), device="cuda", generator=gen) < case["done"]
    if beams > 2 and rows > 8:
        score[-1, 1] = -math.inf                                       # a beam that found no continuation
    return dict(case=case, logits=x, score=score.view(-1), done=done.view(-1), eos=2, parent=_ints([0] * (n_req * k)),
                token=_ints([0] * (n_req * k)), new_score=torch.empty(n_req * k, device="cuda"),
                new_done=torch.empty(n_req * k, dtype=torch.bool, device="cuda"),
                workspace=torch.empty(rows * -(-vocab // 4096) * (8 * k + 16), dtype=torch.uint8, device="cuda"))


def _beam_pool(case):
    whole = case["prompt"] // case["page"]
    n = _pages(case["prompt"] + case["grown"], case["page"])
    return case["n_req"] * (whole + case["beams"] * (n - whole + 1)) + 5


def _prepare_reorder(case, gen, rng):
    n_req, beams, page, kv_heads, head_dim = case["n_req"], case["beams"], case["page"], case["kv_heads"], case["head_dim"]
    n, whole, n_pages = case["prompt"] + case["grown"], case["prompt"] // page, _beam_pool(case)
    columns = _pages(n, page)
    # the beams of a request share the prompt's whole pages and have grown apart since
    perm = rng.permutation(n_pages)
    shared = perm[:n_req * whole].reshape(n_req, 1, whole).repeat(beams, 1)
    grown = perm[n_req * whole:n_req * whole + n_req * beams * (columns - whole)].reshape(n_req, beams, columns - whole)
    table = np.concatenate([shared, grown], 2).reshape(n_req * beams, columns)
    table = np.concatenate([table, np.zeros((len(table), 2), table.dtype)], 1)          # room for what is still to come
    refs0 = _ints(np.bincount(table[:, :columns].ravel(), minlength=n_pages))
    caches = []
    for _ in range(case["layers"]):
        if case["bits"] == 4:
            caches.append(_random_cache(gen, n_pages, kv_heads, page, head_dim))
        else:
            data = _normal(gen, n_pages, 2, kv_heads, page, head_dim)
            eight = case["bits"] == 8
            caches.append((data.to(torch.float8_e4m3fn) if eight else data,
                           torch.randint(120, 134, data.shape[:-1], device="cuda", generator=gen).to(torch.uint8) if eight else None))
    rows = n_req * beams
    return dict(case=case, refs0=refs0, refs=refs0.clone(), table=_ints(table), lens=_ints([n] * rows), parent=_ints(_beams(case)),
                new_table=torch.zeros_like(_ints(table)), new_len=_ints([0] * rows), copies=_ints(np.zeros((rows, 3))), caches=caches,
                status=_ints([0]), workspace=torch.empty(4 * n_pages + 16 * rows, dtype=torch.uint8, device="cuda"))


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2605_30010_b200 import binding as B
    case = s["case"]
    op = case["op"]
    if op == "store":
        B.et_kv_append(s["codes"], s["scale"], s["qkv"], case["heads"], s["table"], s["start"], row_offsets=s["offsets"],
                       theta=case["theta"], q_out=s["q_out"], status=s["status"])
        B.et_kv_read(s["codes"], s["scale"], s["table"], s["start"], s["rows"], row_offsets=s["offsets"], out=s["back"],
                     status=s["status"])
    elif op == "attention":
        B.et_attention_paged(s["q"], case["heads"], s["codes"], s["scale"], s["table"], s["lens"], out=s["out"], lse=s["lse"],
                             workspace=s["workspace"], status=s["status"])
    elif op == "pages":
        B.et_pages_update(s["refs"], case["page"], s["table"], s["lens"], keep=s["keep"], add=s["add"], new_len=s["new_len"],
                          row_offsets=s["offsets"], slots=s["slots"], status=s["status"], workspace=s["workspace"])
    elif op == "select":
        B.et_beam_select(s["logits"], case["beams"], case["k"], scores=s["score"], done=s["done"], eos=s["eos"], parent=s["parent"],
                         token=s["token"], new_scores=s["new_score"], new_done=s["new_done"], workspace=s["workspace"])
    else:
        s["refs"].copy_(s["refs0"])               # every pass begins with the same counts
        B.et_pages_fork(s["refs"], case["page"], s["table"], s["lens"], s["parent"], s["new_table"], new_len=s["new_len"],
                        copies=s["copies"], status=s["status"], workspace=s["workspace"])
        for data, scale in s["caches"]:
            B.et_kv_copy(data, scale, s["copies"], status=s["status"])
    return _outputs(s)


def _outputs(s):
    op = s["case"]["op"]
    if op == "store":
        return dict(rows=s["back"]) if s["q_out"] is None else dict(rows=s["back"], q=s["q_out"])
    if op == "attention":
        return dict(out=s["out"], lse=s["lse"])
    if op == "pages":
        return dict(refs=s["refs"], table=s["table"], new_len=s["new_len"], offsets=s["offsets"], slots=s["slots"])
    if op == "select":
        return dict(parent=s["parent"], token=s["token"], score=s["new_score"], done=s["new_done"])
    got = dict(refs=s["refs"], table=s["new_table"], new_len=s["new_len"], copies=s["copies"])
    for i, (data, scale) in enumerate(s["caches"]):
        got["data%d" % i] = data                  # codes of 4 bits are moved, not computed: the same bytes
        if scale is not None:
            got["scale%d" % i] = scale
    return got


def _run_plain(s):
    {"store": _plain_store, "attention": _plain_attention, "pages": _plain_pages, "select": _plain_select,
     "reorder": _plain_reorder}[s["case"]["op"]](s)
    return _outputs(s)


def _quantise(x):
    """64-bit rows [..., d] -> (codes [..., d / 2], scale [..., d / 32])."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    least = y.abs().amax(-1) / 7
    scale = least.to(torch.bfloat16)
    scale = torch.where(scale.double() < least, (scale.view(torch.int16) + 1).view(torch.bfloat16), scale)      # the next one up
    size = scale.double().unsqueeze(-1)
    n = torch.where(size > 0, torch.round(y / torch.where(size > 0, size, 1.0)), 0.0).clamp(-7, 7)
    n = (n + 8).to(torch.uint8).reshape(x.shape)
    return n[..., ::2] | (n[..., 1::2] << 4), scale


def _values(codes, scale):
    """Cached rows as the fp32 values that they stand for."""
    n = torch.stack([codes & 15, codes >> 4], -1).reshape(*scale.shape, 32).float() - 8
    return (n * scale.float().unsqueeze(-1)).reshape(*codes.shape[:-1], -1)


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
    """Rotate-half rotary embedding of x [rows][heads][d], in 64 bits: positions are far, and keys lie next to borders."""
    half = x.shape[-1] // 2
    turn = theta ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    angle = (pos.double().unsqueeze(-1) * turn).unsqueeze(1)
    cos, sin = torch.cos(angle), torch.sin(angle)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_store(s):
    case = s["case"]
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["head_dim"]
    page, place, pos = _places(s, s["rows"])
    x = s["qkv"].double().view(s["rows"], heads + 2 * kv_heads, d)
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    if case["theta"] > 0:
        q, k = _rotate(q, pos, case["theta"]), _rotate(k, pos, case["theta"])
    if s["q_out"] is not None:
        s["q_out"].copy_(q.reshape(s["rows"], -1))
    codes, scale = _quantise(torch.stack([k, v], 1))          # [rows][2][kv_heads]...
    s["codes"].permute(0, 3, 1, 2, 4)[page, place] = codes
    s["scale"].permute(0, 3, 1, 2, 4)[page, place] = scale
    got = _values(s["codes"].permute(0, 3, 1, 2, 4)[page, place], s["scale"].permute(0, 3, 1, 2, 4)[page, place])
    s["back"].copy_(got.reshape(s["rows"], -1))


def _plain_attention(s):
    case = s["case"]
    n, heads, kv_heads, d, table = case["n_seq"], case["heads"], case["kv_heads"], case["head_dim"], s["table"].long()
    longest = table.shape[1] * case["page"]
    data = _values(s["codes"][table], s["scale"][table])      # [n][pages][2][kv_heads][page][d]
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


def _free_first(refs):
    """Page numbers, those that nothing names first, in ascending order."""
    return torch.sort((refs != 0).to(torch.int8), stable=True).indices


def _plain_pages(s):
    page, refs, table = s["case"]["page"], s["refs"], s["table"]
    column = torch.arange(table.shape[1], device="cuda")
    held = s["lens"].clamp(min=0).long()
    kept = torch.minimum(s["keep"].long(), held)
    add = torch.where(kept >= 0, s["add"].clamp(min=0).long(), 0)
    stays = ((kept.clamp(min=0) + page - 1) // page).unsqueeze(1)
    drop = (column >= stays) & (column < ((held + page - 1) // page).unsqueeze(1))
    refs.scatter_add_(0, torch.where(drop, table, 0).long().view(-1), -drop.view(-1).to(torch.int32))
    take = (column >= stays) & (column < ((kept + add + page - 1) // page).unsqueeze(1))
    rank = take.view(-1).long().cumsum(0) - 1
    got = torch.where(take.view(-1), _free_first(refs)[rank.clamp(min=0)], 0)
    refs.scatter_add_(0, got, take.view(-1).to(torch.int32))
    table.copy_(torch.where(take, got.view(take.shape).to(torch.int32), torch.where(drop, -1, table)))
    s["new_len"].copy_(torch.where(kept >= 0, kept + add, -1))
    s["offsets"][1:] = add.cumsum(0)
    row = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(s["offsets"][1:].long(), row, right=True)
    pos = kept[seq] + row - s["offsets"].long()[seq]
    s["slots"].copy_(table.long()[seq, pos // page] * page + pos % page)


def _plain_select(s):
    case = s["case"]
    n_req, beams, vocab, k = case["n_req"], case["beams"], case["vocab"], case["k"]
    x = s["logits"].view(n_req, beams, vocab).double()        # borders between candidates are near
    top = x.amax(-1, keepdim=True)
    lse = torch.log(torch.exp(x - top).sum(-1, keepdim=True)) + top
    score = s["score"].view(n_req, beams, 1).double()
    ended = s["done"].view(n_req, beams, 1)
    x = torch.where(ended, -math.inf, score + x - lse)
    x[:, :, s["eos"]] = torch.where(ended, score, x[:, :, s["eos"]:s["eos"] + 1])[..., 0]
    best, at = torch.sort(x.view(n_req, -1), dim=1, descending=True, stable=True)
    best, at = best[:, :k], at[:, :k]
    fine = best > -math.inf
    first = torch.arange(n_req, device="cuda").unsqueeze(1) * beams
    parent, token = torch.where(fine, first + at // vocab, -1), torch.where(fine, at % vocab, -1)
    s["parent"].copy_(parent.view(-1))
    s["token"].copy_(token.view(-1))
    s["new_score"].copy_(best.reshape(-1))
    s["new_done"].copy_(((token == s["eos"]) | ~fine).view(-1))


def _plain_reorder(s):
    page, refs, table, new, parent = s["case"]["page"], s["refs"], s["table"], s["new_table"], s["parent"].long()
    rows = parent.numel()
    refs.copy_(s["refs0"])
    column = torch.arange(table.shape[1], device="cuda")
    p = parent.clamp(min=0)
    length = torch.where(parent >= 0, s["lens"].long()[p], -1)
    was = column < ((s["lens"].long().clamp(min=0) + page - 1) // page).unsqueeze(1)
    now = column < ((length.clamp(min=0) + page - 1) // page).unsqueeze(1)
    new.copy_(torch.where(now, table[p], new))
    refs.scatter_add_(0, torch.where(was, table, 0).long().view(-1), -was.view(-1).to(torch.int32))
    refs.scatter_add_(0, torch.where(now, new, 0).long().view(-1), now.view(-1).to(torch.int32))
    # a half-filled last page stays with the first child of its parent, if nobody else has it
    row = torch.arange(rows, device="cuda")
    live = length > 0
    children = torch.zeros(len(table), dtype=torch.int64, device="cuda").scatter_add_(0, p, live.long())
    eldest = torch.full_like(children, rows).scatter_reduce_(0, p, torch.where(live, row, rows), "amin")
    part = length.clamp(min=0) % page
    last = (length.clamp(min=0) // page).clamp(max=table.shape[1] - 1)
    old = torch.where(part > 0, new[row, last].long(), 0)
    copied = (part > 0) & ~((row == eldest[p]) & (refs[old] == children[p]))
    fresh = torch.where(copied, _free_first(refs)[(copied.long().cumsum(0) - 1).clamp(min=0)], 0)
    refs.scatter_add_(0, old, -copied.to(torch.int32))
    refs.scatter_add_(0, fresh, copied.to(torch.int32))
    new[row, last] = torch.where(copied, fresh.to(torch.int32), new[row, last])
    s["new_len"].copy_(length)
    s["copies"].copy_(torch.where(copied.unsqueeze(1), torch.stack([old, fresh, part], 1), torch.tensor([-1, -1, 0], device="cuda")))
    # a row without a copy makes another row's once more
    pick = torch.where(copied, row, copied.to(torch.int8).argmax())
    filled = (torch.arange(page, device="cuda") < part[pick].unsqueeze(1)) & copied[pick].unsqueeze(1)
    for data, scale in s["caches"]:
        _copy_rows(data.view(torch.uint8) if data.dtype == torch.float8_e4m3fn else data, old[pick], fresh[pick], filled)
        if scale is not None:
            _copy_rows(scale.unsqueeze(-1) if scale.dim() == 4 else scale, old[pick], fresh[pick], filled)


def _copy_rows(x, source, target, filled):
    x[target] = torch.where(filled[:, None, None, :, None], x[source], x[target])


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("pages", "reorder"):
        return None                               # nothing is computed but whole numbers
    return {"store": _exact_store, "attention": _exact_attention, "select": _exact_select}[case["op"]](s)


def _seq_rows(s, i, first, n):
    """Positions first .. first + n - 1 of sequence i as the cache's (page, place) pairs."""
    page = s["case"]["page"]
    pos = torch.arange(first, first + n, device="cuda")
    column = torch.div(pos, page, rounding_mode="floor")
    return s["table"][i].long()[column], pos - column * page


def _seq_values(s, which, i, n):
    """The first n keys or values of sequence i: [kv_heads][n][d] in 64 bits."""
    pages, place = _seq_rows(s, i, 0, n)
    level = torch.tensor([c - 8.0 for c in range(16)], dtype=torch.float64, device="cuda")
    got = []
    for h in range(s["codes"].shape[2]):
        byte = s["codes"][pages, which, h, place].long()
        pair = torch.stack([level[byte % 16], level[torch.div(byte, 16, rounding_mode="floor")]], 2)
        got.append(pair.flatten(1) * s["scale"][pages, which, h, place].double().repeat_interleave(32, 1))
    return torch.stack(got)


def _exact_attention(s):
    case = s["case"]
    n, heads, kv_heads, d = case["n_seq"], case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.zeros((n, heads, d), dtype=torch.float64, device="cuda")
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device="cuda")
    for i, length in enumerate(_lengths(case)):
        if length == 0:
            continue
        k, v = (_seq_values(s, which, i, length).repeat_interleave(heads // kv_heads, 0) for which in (0, 1))
        z = torch.einsum("hd,hnd->hn", s["q"][i].view(heads, d).double(), k) * d ** -0.5
        lse[i] = torch.logsumexp(z, -1)
        out[i] = torch.einsum("hn,hnd->hd", torch.softmax(z, -1), v)
    return dict(out=out.view(n, heads * d), lse=lse)


def _exact_store(s):
    case = s["case"]
    heads, kv_heads, d, half = case["heads"], case["kv_heads"], case["head_dim"], case["head_dim"] // 2
    x = s["qkv"].double().view(s["rows"], heads + 2 * kv_heads, d)
    pos = torch.cat([torch.arange(r.start, r.start + r.n, device="cuda") for r in _runs(case)]).double()
    if case["theta"] > 0:
        i = torch.arange(half, device="cuda", dtype=torch.float64)
        turned = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos[:, None] * torch.exp(-2 * i / d * math.log(case["theta"])))
        z = torch.complex(x[:, :heads + kv_heads, :half], x[:, :heads + kv_heads, half:]) * turned[:, None]
        x = torch.cat([torch.cat([z.real, z.imag], -1), x[:, heads + kv_heads:]], 1)
    parts = []
    for block in x[:, heads:].reshape(s["rows"], -1).split(32, 1):
        m, e = torch.frexp(block.abs().amax(1) / 7)
        size = torch.ldexp(torch.ceil(m * 256), e - 8)                 # eight bits, upwards
        parts.append(torch.round(block / size[:, None].clamp(min=1e-300)) * size[:, None])
    got = dict(rows=torch.cat(parts, 1))
    if heads:
        got["q"] = x[:, :heads].reshape(s["rows"], heads * d)
    return got


def _exact_select(s):
    case = s["case"]
    n_req, beams, vocab, k = case["n_req"], case["beams"], case["vocab"], case["k"]
    best = torch.empty((n_req, k), dtype=torch.float64, device="cuda")
    for q in range(n_req):
        pool = []
        for b in range(q * beams, (q + 1) * beams):
            if s["done"][b]:
                pool.append(s["score"][b:b + 1].double())
            else:
                pool.append(torch.log_softmax(s["logits"][b].double(), 0).topk(min(k, vocab)).values + s["score"][b].double())
        pool = torch.cat(pool + [torch.full((k,), -math.inf, dtype=torch.float64, device="cuda")])
        best[q] = pool.topk(k).values
    return dict(parent=None, token=None, score=best.view(-1), done=None)
