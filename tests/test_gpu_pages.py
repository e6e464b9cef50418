"""Pages of the cache and beam search (include/earlytom_pages.h) against plain implementations: sequential ones for tables and counts,
whose results have to be the same whole numbers, and 64-bit ones for what is computed.  Then all of them together with the decode
step's operators as a beam search over a small model's attention."""
import math

import numpy as np
import pytest

from tests.test_gpu_decode import bf16, f64, i32
from tests.test_gpu_kv_int4 import Cache4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2605_30010_b200 import binding
    return binding


# ---- et_pages_update --------------------------------------------------------------------------------------------------

def up(n, page):
    return -(-n // page)


def update_reference(refs, page, table, lens, keep, add, most=1 << 20):
    """One sequence after the other: (refs, table, new_len, offsets, slots, codes of the status that may be there)."""
    refs, table = refs.copy(), table.copy()
    n_seq, max_pages = table.shape
    cap, codes = max_pages * page, set()
    turns = []
    for s in range(n_seq):
        held = min(max(lens[s], 0), cap)
        kept = (lens[s] if lens[s] < 0 else held) if keep is None else min(keep[s], held)
        kept = max(kept, -1)
        want = 0 if kept < 0 else 1 if add is None else max(add[s], 0)
        for j in range(up(max(kept, 0), page), up(held, page)):
            p, table[s, j] = table[s, j], -1
            if not 0 <= p < len(refs):
                codes.add(5)
            elif refs[p] <= 0:
                codes.add(7)
            else:
                refs[p] -= 1
        turns.append((kept, want))
    free = list(np.nonzero(refs == 0)[0])
    at, new_len, offsets, slots = 0, [], [0], []
    for s, (kept, want) in enumerate(turns):
        first, got = up(max(kept, 0), page), True
        if kept + want > cap:
            codes.add(3)
            got = False
        else:
            columns = range(first, up(max(kept, 0) + want, page))
            at += len(columns)
            got = len(columns) == 0 or at <= len(free)
            if not got:
                codes.add(6)
            for i, j in enumerate(columns):
                table[s, j] = free[at - len(columns) + i] if got else -1
                if got:
                    refs[table[s, j]] = 1
        new_len.append(-1 if kept < 0 else kept + want * got)
        offsets.append(offsets[-1] + want)
        for pos in range(kept, kept + min(want, most - len(slots))):
            p = table[s, pos // page] if got else -1
            if got and not 0 <= p < len(refs):
                codes.add(5)
            slots.append(p * page + pos % page if 0 <= p < len(refs) else -1)
    return refs, table, np.array(new_len), np.array(offsets), np.array(slots, dtype=np.int64), codes


def random_state(rng, n_seq, longest, page, spare, room=2, shared=True):
    lens = (longest * rng.random(n_seq)).astype(int)
    lens[0] = longest
    lens[rng.random(n_seq) < 0.1] = 0
    lens[rng.random(n_seq) < 0.1] = -1
    used = up(np.maximum(lens, 0), page)
    table = np.full((n_seq, used.max() + room), -7)
    live = np.arange(table.shape[1]) < used[:, None]
    n_pages = int(used.sum()) + spare
    table[live] = rng.permutation(n_pages)[:used.sum()]
    if shared:
        for s in range(1, n_seq, 3):
            m = min(used[s], used[s - 1], 2)
            table[s, :m] = table[s - 1, :m]
    refs = np.bincount(table[live], minlength=n_pages)
    refs[rng.random(n_pages) < 0.05] += 1
    return lens, table, refs


def check_update(B, page, lens, table, refs, keep, add, rows=None, in_place=False, with_offsets=True, fill=255):
    import torch
    want = update_reference(refs, page, table, lens, keep, add, 1 << 20 if rows is None else rows)
    r, t, l = i32(refs), i32(table), i32(lens)
    rows = len(want[4]) if rows is None else rows
    offsets = i32([-9] * (len(lens) + 1)) if with_offsets else None
    slots, status = i32([-9] * rows) if rows else None, i32([0])
    ws = torch.full((B.ET_PAGES_WORKSPACE(len(refs), len(lens)),), fill, dtype=torch.uint8, device="cuda")
    new = B.et_pages_update(r, page, t, l, None if keep is None else i32(keep), None if add is None else i32(add), l if in_place else None, offsets,
                            slots, status, ws)
    torch.cuda.synchronize()
    assert np.array_equal(r.cpu().numpy(), want[0])
    assert np.array_equal(t.cpu().numpy(), want[1])
    assert np.array_equal(new.cpu().numpy(), want[2]) and (new is l) == in_place
    if with_offsets:
        assert np.array_equal(offsets.cpu().numpy(), want[3])
    if rows:
        n = min(rows, len(want[4]))
        got = slots.cpu().numpy()
        assert np.array_equal(got[:n], want[4][:n]) and (got[n:] == -1).all()
    codes = set(want[5]) | ({3} if rows and rows < want[3][-1] else set())
    assert status.item() == max(codes, default=0)
    return r, t, new


@pytest.mark.parametrize("n_seq,longest,page,spare", [(1, 1, 16, 3), (1, 100_000, 16, 9000), (3, 130, 64, 10), (64, 16_000, 64, 3000), (150, 700, 32, 900),
                                                      (1023, 90, 16, 4000), (1025, 64, 128, 1500), (9000, 40, 16, 20_000), (65_536, 20, 32, 70_000)])
def test_update(B, n_seq, longest, page, spare):
    """Decode steps, drafts that are rejected, prompts that come and go, slots that open and close; counts above one."""
    rng = np.random.default_rng(n_seq + longest)
    lens, table, refs = random_state(rng, n_seq, longest, page, spare)
    cap = table.shape[1] * page
    check_update(B, page, lens, table, refs, None, None, in_place=True)
    keep = np.where(rng.random(n_seq) < 0.2, -1, np.maximum(lens - rng.integers(0, 9, n_seq), 0))
    keep[rng.random(n_seq) < 0.2] = 0
    add = rng.integers(-2, 7, n_seq)
    check_update(B, page, lens, table, refs, keep, add)
    new = (longest * rng.random(n_seq) * 0.8).astype(int)
    keep = np.where(rng.random(n_seq) < 0.5, 0, lens + 5)
    check_update(B, page, lens, table, refs, keep, np.minimum(new, np.maximum(cap - np.minimum(np.maximum(lens, 0), keep), 0)) * (keep == 0), in_place=True)


def test_update_without_room(B):
    """Pages run out in the middle of the sequences; a table is full; more is asked for than can be said."""
    rng = np.random.default_rng(4)
    for spare in (0, 1, 7, 40):
        lens, table, refs = random_state(rng, 200, 100, 16, spare, shared=False)
        refs[refs == 0] = rng.integers(0, 2, (refs == 0).sum())
        check_update(B, 16, lens, table, refs, None, rng.integers(0, 40, 200))
    lens, table, refs = random_state(rng, 30, 100, 16, 300, room=0)
    check_update(B, 16, lens, table, refs, None, None)
    add = np.zeros(30, int)
    add[3], add[7], add[9] = 2 ** 30, 10 ** 6, 3
    check_update(B, 16, lens, table, refs, None, add, rows=50)
    check_update(B, 16, lens, table, refs, np.zeros(30, int), np.full(30, 20), rows=1000)
    check_update(B, 16, np.full(30, 10_000), table, np.full(len(refs), 3), None, None)


def test_update_with_entries_and_counts_that_are_wrong(B):
    rng = np.random.default_rng(5)
    lens, table, refs = random_state(rng, 20, 200, 16, 50)
    lens[:6] = [200, 100, 64, 40, 33, 90]
    table[0, 3], table[1, 2], table[2, 3], table[4, 1] = -1, len(refs), 2 ** 31 - 1, -2 ** 31
    check_update(B, 16, lens, table, np.maximum(refs, 1), np.full(20, 5), np.full(20, 17))
    refs[table[3, 1]], refs[table[5, 2]] = 0, -4
    check_update(B, 16, lens, table, refs, np.zeros(20, int), np.zeros(20, int))


@pytest.mark.parametrize("rows", [0, 1, 16_383, 16_384, 16_385, 40_001])
def test_update_slots(B, rows):
    """Slots of few rows and of many, fewer and more than there are; with offsets and without."""
    rng = np.random.default_rng(6)
    lens, table, refs = random_state(rng, 40, 3000, 32, 2000)
    add = np.minimum(rng.integers(0, 900, 40), table.shape[1] * 32 - np.maximum(lens, 0))
    for with_offsets in (True, False):
        check_update(B, 32, lens, table, refs, None, add, rows=rows, with_offsets=with_offsets, fill=rows % 251)


def test_update_in_a_graph_on_a_side_stream(B):
    """Three captured updates in a row, replayed: each sees the one before, as the same calls one by one do."""
    import torch
    rng = np.random.default_rng(7)
    lens, table, refs = random_state(rng, 50, 60, 16, 900, room=30)
    state = [i32(refs), i32(table), i32(lens)]
    ws, status, slots = torch.empty(B.ET_PAGES_WORKSPACE(len(refs), 50), dtype=torch.uint8, device="cuda"), i32([0]), i32([0] * 50)
    add = i32(rng.integers(0, 5, 50))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        for a in (None, add, None):
            B.et_pages_update(state[0], 16, state[1], state[2], add=a, new_len=state[2], slots=slots, status=status, workspace=ws)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for a in [None, add.cpu().numpy(), None] * 2:
        refs, table, lens, _, _, codes = update_reference(refs, 16, table, lens, None, a)
        assert not codes - {3}
    assert np.array_equal(state[0].cpu().numpy(), refs) and np.array_equal(state[1].cpu().numpy(), table) and np.array_equal(state[2].cpu().numpy(), lens)


# ---- et_pages_fork, et_kv_copy ----------------------------------------------------------------------------------------

def fork_reference(refs, page, table, lens, parent, new_table):
    refs, new_table = refs.copy(), new_table.copy()
    n_old, max_pages = table.shape
    codes, lengths, kids = set(), [], {}
    good = lambda p: 0 <= p < len(refs)                                                           # noqa: E731
    for b, p in enumerate(parent):
        if p >= n_old:
            codes.add(8)
        if 0 <= p < n_old:
            kids.setdefault(p, []).append(b)
        lengths.append(max(lens[p], -1) if 0 <= p < n_old else -1)
    for p in range(n_old):
        for j in range(min(up(max(lens[p], 0), page), max_pages)):
            g = table[p, j]
            if not good(g):
                codes.add(5)
            else:
                refs[g] += len(kids.get(p, [])) - 1
                assert refs[g] >= 0
            for b in kids.get(p, []):
                new_table[b, j] = g
    last = {}
    for b, n in enumerate(lengths):
        if n > 0 and n % page and n // page < max_pages and good(new_table[b, n // page]):
            g = new_table[b, n // page]
            family = kids[parent[b]]
            if not (b == family[0] and refs[g] == len(family)):
                last[b] = g
    free = list(np.nonzero(refs == 0)[0])
    copies = np.array([[-1, -1, 0]] * len(parent))
    for i, (b, g) in enumerate(last.items()):
        j = lengths[b] // page
        refs[g] -= 1
        new_table[b, j] = -1
        if i < len(free):
            new_table[b, j] = free[i]
            refs[free[i]] = 1
            copies[b] = g, free[i], lengths[b] % page
        else:
            codes.add(6)
    return refs, new_table, np.array(lengths), copies, codes


def beam_state(rng, n_req, beams, prompt, grown, page, spare, room=1):
    """Tables of requests whose beams share the prompt's whole pages."""
    whole, columns = prompt // page, up(prompt + grown, page)
    n_pages = n_req * (whole + beams * (columns - whole)) + spare
    perm = rng.permutation(n_pages)
    table = np.full((n_req, beams, columns + room), -3)
    table[:, :, :whole] = perm[:n_req * whole].reshape(n_req, 1, whole)
    table[:, :, whole:columns] = perm[n_req * whole:n_req * (whole + beams * (columns - whole))].reshape(n_req, beams, columns - whole)
    table = table.reshape(n_req * beams, -1)
    return np.full(n_req * beams, prompt + grown), table, np.bincount(table[:, :columns].ravel(), minlength=n_pages)


def check_fork(B, page, lens, table, refs, parent, fill=255):
    import torch
    new = np.full((len(parent), table.shape[1]), -5)
    want = fork_reference(refs, page, table, lens, parent, new)
    r, t, status = i32(refs), i32(new), i32([0])
    ws = torch.full((B.ET_FORK_WORKSPACE(len(refs), len(parent)),), fill, dtype=torch.uint8, device="cuda")
    old = i32(table)
    new_len, copies = B.et_pages_fork(r, page, old, i32(lens), i32(parent), t, status=status, workspace=ws)
    torch.cuda.synchronize()
    assert np.array_equal(new_len.cpu().numpy(), want[2])
    assert np.array_equal(t.cpu().numpy(), want[1])
    assert np.array_equal(copies.cpu().numpy(), want[3])
    assert np.array_equal(r.cpu().numpy(), want[0])
    assert np.array_equal(old.cpu().numpy(), table) and status.item() == max(want[4], default=0)
    return r, t, new_len, copies


@pytest.mark.parametrize("n_req,beams,prompt,grown,page", [(1, 1, 5, 0, 16), (1, 4, 7675, 50, 64), (1, 3, 15, 1, 16), (7, 5, 33, 20, 16), (32, 8, 700, 77, 32),
                                                           (3, 2, 128, 0, 128), (300, 4, 40, 3, 16), (2048, 8, 20, 9, 16)])
def test_fork(B, n_req, beams, prompt, grown, page):
    """Beams that go on, branch and end, in whole pages and in the middle of one; rows of several requests, and with fewer and more
    rows than before."""
    rng = np.random.default_rng(n_req + prompt)
    rows = n_req * beams
    lens, table, refs = beam_state(rng, n_req, beams, prompt, grown, page, rows + 5)
    own = np.arange(rows) // beams * beams
    check_fork(B, page, lens, table, refs, np.arange(rows))
    parent = own + (beams * rng.random(rows) ** 2).astype(int)
    check_fork(B, page, lens, table, refs, parent)
    check_fork(B, page, lens, table, refs, own)                                   # one beam takes all
    parent[rng.random(rows) < 0.2] = -1
    check_fork(B, page, lens, table, refs, parent, fill=0)
    if rows <= 8192:
        check_fork(B, page, lens, table, refs, np.repeat(parent, 2))              # pages may run out here
    check_fork(B, page, lens, table, refs, parent[:(rows + 1) // 2])
    check_fork(B, page, lens, table, refs, np.full(rows, -1))
    lens = np.maximum(lens - rng.integers(0, page, rows), -1)
    lens[rng.random(rows) < 0.1] = -1
    refs = np.bincount(table[np.arange(table.shape[1]) < up(np.maximum(lens, 0), page)[:, None]], minlength=len(refs))
    check_fork(B, page, lens, table, refs, parent)


def test_fork_of_pages_that_others_hold_and_of_bad_ones(B):
    rng = np.random.default_rng(1)
    lens, table, refs = beam_state(rng, 5, 3, 40, 9, 16, 40)
    parent = np.array([0, 0, 2, 3, 4, 5, 6, 6, 6, 9, 11, 11, -1, 99, 2 ** 31 - 1])
    held = refs.copy()
    held[table[:, 3]] += 1                                                       # everybody's last page is kept elsewhere as well
    check_fork(B, 16, lens, table, held, parent)
    table[0, 3] = table[2, 0] = -1
    table[3, 1], table[6, 3] = len(refs), 2 ** 31 - 1
    check_fork(B, 16, lens, table, refs + 1, parent)
    lens[9] = 10_000                                                             # longer than its table
    check_fork(B, 16, lens, table, refs + 1, parent)


def cache_bytes(B, rng, n_pages, kvh, page, d, fmt):
    import torch
    shape = (n_pages, 2, kvh, page)
    data = torch.from_numpy(rng.integers(0, 256, (*shape, (2 * d, d, d // 2)[fmt]), dtype=np.uint8)).cuda()
    data = data.view({0: torch.bfloat16, 1: torch.float8_e4m3fn, 2: torch.uint8}[fmt])
    scale = None
    if fmt == 1:
        scale = torch.from_numpy(rng.integers(0, 255, shape, dtype=np.uint8)).cuda()
    elif fmt == 2:
        scale = torch.from_numpy(rng.integers(0, 256, (*shape, d // 16), dtype=np.uint8)).cuda().view(torch.bfloat16)
    return data, scale


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("kvh,page,d", [(1, 16, 64), (4, 64, 128), (3, 128, 64), (16, 32, 128)])
def test_copy(B, fmt, kvh, page, d):
    """From one position to a whole page, entries that are skipped; nothing else changes."""
    import torch
    rng = np.random.default_rng(kvh + fmt)
    n_pages = 60
    data, scale = cache_bytes(B, rng, n_pages, kvh, page, d, fmt)
    perm = rng.permutation(n_pages)
    copies = [[perm[0], perm[1], 1], [perm[0], perm[2], page], [perm[3], perm[4], page - 1], [-1, -1, 0], [perm[5], perm[6], 0], [perm[7], -1, 5],
              [perm[8], perm[9], page + 9], [-3, perm[10], 4], [perm[11], perm[12], -2]] + [[perm[13 + 2 * i], perm[14 + 2 * i], 1 + i % page] for i in range(20)]
    want, want_scale = data.view(torch.uint8).clone(), None if scale is None else scale.view(torch.uint8).clone()
    for a, b, n in copies:
        if a >= 0 and b >= 0 and n > 0:
            want[b, :, :, :n] = want[a, :, :, :n]
            if scale is not None:
                want_scale[b, :, :, :n] = want_scale[a, :, :, :n]
    status = i32([0])
    B.et_kv_copy(data, scale, i32(copies), status)
    assert torch.equal(data.view(torch.uint8), want) and (scale is None or torch.equal(scale.view(torch.uint8), want_scale)) and status.item() == 0
    B.et_kv_copy(data, scale, i32([[0, n_pages, 3], [n_pages, 0, 3], [2 ** 31 - 1, 2 ** 31 - 1, 3]]), status)
    assert torch.equal(data.view(torch.uint8), want) and status.item() == B.ET_PAGED_BAD_PAGE


# ---- et_beam_select ---------------------------------------------------------------------------------------------------

def select_reference(x, scores, done, eos, beams, k):
    """(parent, token, score, done, margins): the best k in 64 bits, and how far each is from the next one."""
    rows, vocab = x.shape
    out = []
    for q in range(rows // beams):
        pool = []
        for b in range(beams):
            r = q * beams + b
            if not math.isfinite(scores[r]):
                continue
            if done[r]:
                pool.append((scores[r], r, eos))
                continue
            with np.errstate(all="ignore"):
                top = x[r].max()
                total = scores[r] + x[r] - (np.log(np.exp(x[r] - top).sum()) + top)
            if not math.isfinite(top):
                continue
            order = np.lexsort((np.arange(vocab), -x[r]))[:k]
            pool += [(total[t], r, t) for t in order if x[r, t] > -math.inf]
        pool.sort(key=lambda e: (-e[0], e[1]))
        got = pool[:k] + [(-math.inf, -1, -1)] * (k - len(pool))
        gaps = [abs(a[0] - b[0]) if a[1] != b[1] else math.inf for a, b in zip(pool, pool[1:])][:k] + [math.inf]
        out += [(p, t, s, t == eos or p < 0, min(gaps)) for s, p, t in got]
    return out


def check_select(B, x, beams, k, scores=None, done=None, eos=-1, ties=False, fill=255):
    """x: a tensor on the GPU.  Where two beams' candidates are within 2^-18 of one another (the logarithm's 2^-20 and the reference's
    rounding, twice) the request's order is not compared unless the beams are alike (`ties`)."""
    import torch
    rows = x.shape[0]
    s = np.zeros(rows) if scores is None else np.asarray(scores, dtype=np.float32).astype(float)
    dn = np.zeros(rows, bool) if done is None else np.asarray(done)
    want = select_reference(f64(x), s, dn, eos, beams, k)
    ws = torch.full((B.ET_BEAM_WORKSPACE(rows, x.shape[1], k),), fill, dtype=torch.uint8, device="cuda")
    got = B.et_beam_select(x, beams, k, None if scores is None else torch.tensor(s, dtype=torch.float32, device="cuda"),
                           None if done is None else torch.tensor(dn, device="cuda"), eos, workspace=ws)
    parent, token, score, ended = (t.tolist() for t in got)
    skipped = 0
    for i, (p, t, v, e, gap) in enumerate(want):
        if gap < 2.0 ** -18 and not ties:
            skipped += 1
            continue
        assert (parent[i], token[i], ended[i]) == (p, t, e), (i, parent[i], token[i], p, t)
        assert score[i] == v or abs(score[i] - v) <= 2.0 ** -20 + 2.0 ** -24 * abs(v)
    assert skipped <= len(want) // 8
    return got


@pytest.mark.parametrize("fp32", [False, True])
@pytest.mark.parametrize("n_req,beams,k,vocab", [(1, 1, 1, 1), (2, 3, 7, 2), (1, 4, 4, 4095), (3, 1, 5, 4096), (2, 2, 33, 4097), (1, 5, 64, 9001), (4, 32, 32, 777),
                                                 (40, 4, 8, 12_289), (1, 2, 64, 100_003), (300, 2, 2, 31), (2, 4, 20, 262_147), (1, 1, 3, 1 << 20)])
def test_select(B, n_req, beams, k, vocab, fp32):
    """Odd vocabularies, whose rows begin anywhere, one chunk to 256 of them, one candidate to 64; bf16 logits with many equal values."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(vocab + k)
    rng = np.random.default_rng(vocab + k)
    rows = n_req * beams
    x = torch.randn((rows, vocab), device="cuda", generator=gen) * 3
    x = x if fp32 else x.to(torch.bfloat16)
    check_select(B, x, beams, k)
    scores = -20 * rng.random(rows)
    scores[rng.random(rows) < 0.15] = -math.inf
    check_select(B, x, beams, k, scores, rng.random(rows) < 0.3, eos=vocab // 2, fill=0)


@pytest.mark.parametrize("order", ["rising", "falling", "equal", "few levels", "one group", "negative"])
@pytest.mark.parametrize("k", [1, 4, 32, 50, 64])
def test_select_of_unlucky_orders(B, order, k):
    """Logits in the orders that put many of them on the list of candidates; equal ones in the order of their tokens."""
    import torch
    vocab = 3 * 4096 + 55
    i = torch.arange(vocab, device="cuda").float()
    x = {"rising": i / 64, "falling": -i / 64, "equal": torch.ones_like(i), "few levels": (i * 7919 % 3), "negative": -3e38 + i * 1e33,
         "one group": torch.where((i % 4096 // 4 % 256) < 8, 50 - i / 1000, -i / 100)}[order]
    x = torch.stack([x, x, torch.where(i % 3 == 0, x, -math.inf)])
    check_select(B, x, 3, k, scores=[-1.0, -1.0, -1e9], ties=True)
    check_select(B, x[:1], 1, k)
    check_select(B, x.to(torch.bfloat16), 3, k, scores=[-1.0, -3.3, -1.7], ties=order == "negative")


def test_select_of_logits_that_are_not_finite(B):
    """Banned tokens, rows with none left, with NaN or an infinity; zeros of both signs are equal."""
    import torch
    inf, nan = math.inf, math.nan
    x = torch.full((8, 9000), -inf, device="cuda")
    x[0, [5, 8999]] = torch.tensor([1.0, 2.0], device="cuda")
    x[2] = torch.randn(9000, device="cuda")
    x[2, 77] = nan
    x[3] = torch.randn(9000, device="cuda")
    x[3, 8000] = inf
    x[4] = 0.0
    x[4, 100] = -0.0
    x[5, 0] = -3e38
    x[6] = nan
    x[7] = inf
    parent, token, score, done = check_select(B, x, 8, 10, eos=5, ties=True)
    assert set(parent.tolist()) <= {0, 4, 5} and token.tolist()[0] == 0 and parent.tolist()[0] == 5
    got = check_select(B, x[4:5].to(torch.bfloat16), 1, 64, ties=True)
    assert got[1].tolist() == list(range(64))
    got = check_select(B, x[[1, 3, 6, 7]], 4, 5)
    assert got[0].tolist() == [-1] * 5 and got[3].tolist() == [True] * 5 and (got[2] == -inf).all()
    check_select(B, x[[0, 4]], 2, 4, scores=[inf, nan])
    check_select(B, x[[0, 4]], 2, 4, scores=[nan, -1.0], done=[True, False], eos=3, ties=True)


def test_select_from_strided_rows(B):
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.randn((6, 10_007), device="cuda").to(dtype)
        for first in (0, 1, 3, 7):
            part = wide[:, first:first + 9_001]
            a, b = B.et_beam_select(part, 3, 8), B.et_beam_select(part.contiguous(), 3, 8)
            assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_select_accurate_sums(B):
    """Scores of distributions from flat to peaked, beside large offsets, within the documented 2^-20."""
    import torch
    vocab = 152_064
    i = torch.arange(vocab, device="cuda").double()
    x = torch.stack([torch.zeros_like(i), -i / 1000, -(i / 40) ** 0.5, torch.sin(i) * 30, torch.cos(i) + 1000, -torch.log1p(i) * 1.01]).float()
    for r in range(len(x)):
        _, token, score, _ = B.et_beam_select(x[r:r + 1], 1, 64)
        y = x[r].double()
        want = y[token.long()] - torch.logsumexp(y, 0)
        assert ((score.double() - want).abs() <= 2.0 ** -20 + 2.0 ** -24 * want.abs()).all(), r


# ---- together ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["int4", "bf16"])
def test_beam_search_over_paged_caches(B, fmt):
    """Three requests of different prompts, four beams, 40 tokens, two layers of attention, all of it captured as one graph that is
    replayed: pages handed out, rows appended, attention, output head, selection, fork and copies.  Against the same search with
    each beam's keys and values in tensors of its own, moved about as the beams are, whose attention is computed in 64 bits from the rows that the
    cache stored; the search goes on from the graph's selection, which has to be right to the logits' rounding."""
    import torch
    rng = np.random.default_rng(2)
    n_req, beams, heads, kvh, d, page, vocab, layers, steps = 3, 4, 4, 2, 64, 16, 1000, 2, 40
    rows, hidden, eos, max_pages = n_req * beams, 256, 7, 12
    prompts = [30, 64, 1]
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)                                # noqa: E731
    embed = rand(vocab, hidden).to(torch.bfloat16)
    wqkv = [(rand((heads + 2 * kvh) * d, hidden) / math.sqrt(hidden)).to(torch.bfloat16) for _ in range(layers)]
    wo = [(rand(hidden, heads * d) / math.sqrt(heads * d)).to(torch.bfloat16) for _ in range(layers)]
    head = (rand(vocab, hidden) * 0.3).to(torch.bfloat16)
    n_pages = 120
    caches = []
    for _ in range(layers):
        if fmt == "int4":
            caches.append((torch.zeros((n_pages, 2, kvh, page, d // 2), dtype=torch.uint8, device="cuda"),
                           torch.zeros((n_pages, 2, kvh, page, d // 32), dtype=torch.bfloat16, device="cuda")))
        else:
            caches.append((torch.zeros((n_pages, 2, kvh, page, d), dtype=torch.bfloat16, device="cuda"), None))
    refs, status = i32([0] * n_pages), i32([0])
    # the prompts' rows, one sequence a request, and then a row for each beam
    first = i32(np.full((n_req, max_pages), -1))
    start, offsets = i32([0] * n_req), i32([0] * (n_req + 1))
    lens = B.et_pages_update(refs, page, first, start, add=i32(prompts), row_offsets=offsets, status=status)
    x0 = embed[torch.randint(0, vocab, (sum(prompts),), device="cuda", generator=gen)]
    for (data, scale), w in zip(caches, wqkv):
        qkv = (x0.float() @ w[heads * d:].float().T).to(torch.bfloat16)
        B.et_kv_append(data, scale, qkv, 0, first, start, offsets, status=status)
    table, spare = i32(np.full((rows, max_pages), -1)), i32(np.full((rows, max_pages), -1))
    parents = i32(np.repeat(np.arange(n_req), beams))
    lens, copies = B.et_pages_fork(refs, page, first, lens, parents, table, status=status)
    for data, scale in caches:
        B.et_kv_copy(data, scale, copies, status)
    token = i32(rng.integers(0, vocab, rows))
    score, done = torch.zeros(rows, device="cuda"), torch.zeros(rows, dtype=torch.bool, device="cuda")
    score[1::beams] = -1
    score[2::beams], score[3::beams] = -2, -math.inf                             # a beam that is not there yet
    new = dict(len=i32([0] * rows), parent=i32([0] * rows), token=i32([0] * rows), score=torch.empty(rows, device="cuda"),
               done=torch.zeros(rows, dtype=torch.bool, device="cuda"))
    ws = dict(att=torch.empty(B.ET_PAGED_WORKSPACE, dtype=torch.uint8, device="cuda"), pages=torch.empty(4 * n_pages + 16 * rows, dtype=torch.uint8, device="cuda"),
              beam=torch.empty(B.ET_BEAM_WORKSPACE(rows, vocab, beams), dtype=torch.uint8, device="cuda"))
    logits = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda")
    seen = dict(q=[torch.empty((rows, heads * d), dtype=torch.bfloat16, device="cuda") for _ in range(layers)],
                att=[torch.empty((rows, heads * d), dtype=torch.bfloat16, device="cuda") for _ in range(layers)])
    old_len = torch.empty_like(lens)

    def step():
        old_len.copy_(lens)
        B.et_pages_update(refs, page, table, lens, new_len=lens, status=status, workspace=ws["pages"])
        x = embed[token.clamp(min=0).long()]
        for i, (data, scale) in enumerate(caches):
            qkv = B.et_linear_rows(x, wqkv[i])
            B.et_kv_append(data, scale, qkv, heads, table, old_len, theta=1e4, q_out=seen["q"][i], status=status)
            B.et_attention_paged(seen["q"][i], heads, data, scale, table, lens, out=seen["att"][i], workspace=ws["att"], status=status)
            x = (x + B.et_linear_rows(seen["att"][i], wo[i])) * 0.7
        B.et_linear_rows(x.contiguous(), head, c=logits)
        B.et_beam_select(logits, beams, beams, score, done, eos, new["parent"], new["token"], new["score"], new["done"], ws["beam"])
        B.et_pages_fork(refs, page, table, lens, new["parent"], spare, new["len"], copies, status, ws["pages"])
        for data, scale in caches:
            B.et_kv_copy(data, scale, copies, status)
        table.copy_(spare)
        for a, b in ((lens, "len"), (token, "token"), (score, "score"), (done, "done")):
            a.copy_(new[b])

    def held(which):
        """Each beam's stored keys and values: [layer][row] -> [n, 2, kvh, d], read from the cache row by row."""
        at = which.tolist()
        got = []
        for data, scale in caches:
            got.append([B.et_kv_read(data, scale, table[r:r + 1].contiguous(), i32([0]), n, i32([0, n]), status=status).view(n, 2, kvh, d) if n > 0 else None
                        for r, n in enumerate(at)])
        return got

    torch.cuda.synchronize()
    state = [t.clone() for t in (refs, table, lens, token, score, done)] + [t.clone() for c in caches for t in c if t is not None]
    step()                                                                       # (outside the graph first: allocations, and the same result)
    torch.cuda.synchronize()
    one = [t.clone() for t in (refs, table, lens, token, score, done)]
    for a, b in zip([refs, table, lens, token, score, done] + [t for c in caches for t in c if t is not None], state):
        a.copy_(b)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        step()
    own = held(lens)                                                             # what each beam's memory has to be
    for turn in range(steps):
        before = lens.tolist()
        ended = done.clone()
        old_score = score.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert status.item() == 0
        if turn == 0:
            assert all(torch.equal(a, b) for a, b in zip((refs, table, lens, token, score, done), one))
        parent = new["parent"].tolist()
        # tables and counts belong together, and no page that is still written to has two rows
        t, n = table.cpu().numpy(), lens.cpu().numpy()
        live = np.arange(max_pages) < up(np.maximum(n, 0), page)[:, None]
        assert np.array_equal(np.bincount(t[live], minlength=n_pages), refs.cpu().numpy())
        for r in range(rows):
            assert n[r] == (before[parent[r]] + 1 if parent[r] >= 0 and before[parent[r]] >= 0 else -1)
            if n[r] > 0 and n[r] % page:
                assert refs[t[r, n[r] // page]].item() == 1
        # the beams' memories: the parent's, and one row more
        now = held(lens)
        for i in range(layers):
            for r in range(rows):
                if n[r] > 0:
                    assert torch.equal(now[i][r][:-1], own[i][parent[r]])
        # attention of the parents over them, in 64 bits (a row's memory is that of any of its children)
        for i in range(layers):
            for p in set(parent) - {-1}:
                kv = now[i][parent.index(p)].double()
                q = seen["q"][i][p].double().view(kvh, heads // kvh, d)
                z = torch.einsum("hgd,nhd->hgn", q, kv[:, 0]) / math.sqrt(d)
                w = torch.softmax(z, -1)
                want, mass = torch.einsum("hgn,nhd->hgd", w, kv[:, 1]), torch.einsum("hgn,nhd->hgd", w, kv[:, 1].abs())
                # (int4: what is read back is the stored value rounded to bf16, 2^-9 of keys and values, of the score 2^-9 of its size)
                size = torch.einsum("hgd,nhd->hgn", q.abs(), kv[:, 0].abs()).amax(-1, keepdim=True) / math.sqrt(d)
                loose = 2.0 ** -8 * (1 + 2 * size) if fmt == "int4" else 0
                off = (seen["att"][i][p].double().view_as(want) - want).abs()
                assert (off <= 2.0 ** -8 * want.abs() + (2.0 ** -15 + loose + 2 * d * 2.0 ** -23 * size) * mass).all()
        # the selection, from the logits as they are
        want = select_reference(f64(logits), f64(old_score), ended.cpu().numpy(), eos, beams, beams)
        for r, (p, tok, sc, dn, gap) in enumerate(want):
            if gap > 2.0 ** -18:
                assert (parent[r], token[r].item(), done[r].item()) == (p, tok, dn)
            assert score[r].item() == sc or abs(score[r].item() - sc) <= 2.0 ** -19 + 2.0 ** -23 * abs(sc)
        own = now
    # the requests end: every page comes back
    B.et_pages_update(refs, page, table, lens, keep=i32([-1] * rows), status=status)
    assert refs.tolist() == [0] * n_pages and status.item() == 0


def test_calls_on_a_stream_of_their_own(B):
    """Results on a side stream, created there, behind work that takes a while."""
    import torch
    rng = np.random.default_rng(3)
    lens, table, refs = random_state(rng, 30, 200, 16, 100)
    x = torch.randn((6, 5000), device="cuda")
    want = B.et_beam_select(x, 3, 6)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        y = torch.zeros_like(x)
        torch.cuda._sleep(20_000_000)
        y.copy_(x)
        t, r, l = i32(table), i32(refs), i32(lens)
        new_table = torch.zeros_like(t)
    got = B.et_beam_select(y, 3, 6, stream=stream)
    new = B.et_pages_update(r, 16, t, l, stream=stream)
    parent = torch.arange(30, dtype=torch.int32, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    new_len, copies = B.et_pages_fork(r, 16, t, new, parent, new_table, stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ref = update_reference(refs, 16, table, lens, None, None)
    assert np.array_equal(new.cpu().numpy(), ref[2]) and torch.equal(new_len, new)
    ref = fork_reference(ref[0], 16, ref[1], ref[2], np.arange(30), np.zeros_like(table))      # (pages that others hold are copied)
    assert np.array_equal(r.cpu().numpy(), ref[0]) and np.array_equal(new_table.cpu().numpy(), ref[1])
    assert np.array_equal(copies.cpu().numpy(), ref[3])


def test_update_of_sums_beyond_32_bits_writes_nothing_outside(B):
    """More positions asked for than numbers can say: offsets are any, but slots are written within their buffer only."""
    import torch
    rng = np.random.default_rng(12)
    lens, table, refs = random_state(rng, 40, 100, 16, 50)
    for rows in (100, 30_000):
        wide = i32([-77] * (rows + 2_000))
        add = i32([2 ** 31 - 1 - 7 * i if i % 3 else 5 for i in range(40)])
        status, state = i32([0]), [i32(refs), i32(table), i32(lens)]
        B.et_pages_update(*state[:1], 16, *state[1:], add=add, row_offsets=i32([0] * 41), slots=wide[1000:1000 + rows], status=status)
        assert status.item() == B.ET_PAGED_CAPACITY or status.item() == B.ET_PAGED_NO_PAGE
        assert (wide[:1000] == -77).all() and (wide[1000 + rows:] == -77).all()


@pytest.mark.parametrize("n", [1, 700])
def test_update_of_large_tables(B, n):
    """Tables whose entries are given back by a kernel of their own; as many slots as make a thread's rows cross pages and sequences."""
    rng = np.random.default_rng(n)
    longest, page = (300_000, 16) if n == 1 else (900, 16)
    lens, table, refs = random_state(rng, n, longest, page, 25_000)
    assert table.size > 1 << 14
    keep = np.maximum(lens - rng.integers(0, longest, n), 0)
    add = np.minimum(rng.integers(0, longest, n), table.shape[1] * page - np.minimum(np.maximum(lens, 0), keep))
    check_update(B, page, lens, table, refs, keep, add)
    check_update(B, page, lens, table, refs, np.full(n, -1), None, in_place=True)


@pytest.mark.parametrize("n,longest,page", [(1500, 900, 16), (20_000, 70, 16), (2, 640_000, 16)])
def test_update_of_tables_for_the_larger_cluster(B, n, longest, page):
    """Tables of more than 2^16 entries, also with more sequences than the cluster's threads and with fewer than it has CTAs."""
    rng = np.random.default_rng(n)
    lens, table, refs = random_state(rng, n, longest, page, 3_000)
    assert table.size > 1 << 16
    keep = np.maximum(lens - rng.integers(0, longest, n), 0)
    add = np.minimum(rng.integers(0, longest, n), table.shape[1] * page - np.minimum(np.maximum(lens, 0), keep))
    check_update(B, page, lens, table, refs, keep, add)
    check_update(B, page, lens, table, refs, None, None, in_place=True)


@pytest.mark.parametrize("k", [10, 16, 32, 64])
@pytest.mark.parametrize("vocab,allowed", [(300, 1.0), (721, 1.0), (2500, 1.0), (9001, 0.01), (4096, 0.02)])
def test_select_of_few_tokens(B, vocab, allowed, k):
    """Vocabularies and grammars that leave most of a block's threads without a token."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(vocab + k)
    x = torch.randn((6, vocab), device="cuda", generator=gen) * 4
    x = torch.where(torch.rand((6, vocab), device="cuda", generator=gen) < allowed, x, -math.inf)
    x[5, vocab // 3:] = -math.inf
    check_select(B, x, 3, k, scores=[-1.0, -2.0, -3.0, -1.0, -2.0, -3.0])
