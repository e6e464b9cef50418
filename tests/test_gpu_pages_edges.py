"""Pages of the cache and beam search (include/earlytom_pages.h) where numbers, counts and orders are unlucky: against the plain
implementations of test_gpu_pages.py, with buffers between guards."""
import math

import numpy as np
import pytest

from tests.test_gpu_decode import i32
from tests.test_gpu_pages import B, random_state, up, update_reference                            # noqa: F401

pytestmark = pytest.mark.gpu

GUARD = 4096


def guarded(values):
    """(the whole buffer, the part that holds `values`): int32 on the GPU between guards of -77."""
    v = np.asarray(values)
    wide = i32(np.full(v.size + 2 * GUARD, -77))
    part = wide[GUARD:GUARD + v.size].view(v.shape)
    part.copy_(i32(v))
    return wide, part


def guards_hold(wide):
    return bool((wide[:GUARD] == -77).all()) and bool((wide[-GUARD:] == -77).all())


# ---- et_pages_update --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_seq,longest,rows", [(5, 144, 0), (40, 100, 100), (40, 100, 33_000), (700, 900, 50), (1500, 900, 40_000), (9000, 40, 64),
                                                (20_000, 70, 33_000)])
def test_update_of_sums_beyond_32_bits_leaves_tables_right(B, n_seq, longest, rows):              # noqa: F811
    """Many sequences ask for nearly 2^31 positions each: none of them gets one, and tables, counts and lengths are what they are without
    them.  Full sequences among them, the last one too, whose entries end where the next row or the buffer's end is."""
    rng = np.random.default_rng(n_seq + rows)
    page = 16
    lens, table, refs = random_state(rng, n_seq, longest, page, 4000, room=0)
    cap = table.shape[1] * page
    full = rng.random(n_seq) < 0.3
    full[-1] = full[n_seq // 2] = True
    keep = np.where(full, cap, np.maximum(lens - 3, -1))
    lens = np.where(full, cap, lens)
    table[full] = rng.integers(0, len(refs), (int(full.sum()), table.shape[1]))
    refs = np.maximum(refs, 0) + np.bincount(table[full].ravel(), minlength=len(refs))
    add = np.where(rng.random(n_seq) < 0.6, 2 ** 31 - 1 - rng.integers(0, 9, n_seq), rng.integers(0, 9, n_seq))
    want = update_reference(refs, page, table, lens, keep, add.astype(object), most=0)
    bufs = [guarded(x) for x in (refs, table, np.full(n_seq, -9), np.full(n_seq + 1, -9), np.full(max(rows, 1), -9))]
    status = i32([0])
    B.et_pages_update(bufs[0][1], page, bufs[1][1], i32(lens), i32(keep), i32(add), bufs[2][1], bufs[3][1], bufs[4][1] if rows else None, status)
    assert all(guards_hold(wide) for wide, _ in bufs)
    for (_, got), expected in zip(bufs, want[:3]):
        assert np.array_equal(got.cpu().numpy(), expected)
    assert status.item() >= max(want[5])                  # (rows of no order may meet entries that are no pages)


def rows_of(B, cache, table, lens):                                                               # noqa: F811
    """Each sequence's stored rows."""
    return [B.et_kv_read(cache, None, table[i:i + 1].contiguous(), i32([0]), n, i32([0, n])) if n > 0 else None for i, n in enumerate(lens.tolist())]


def test_sequences_grow_behind_a_shared_beginning(B):                                             # noqa: F811
    """Three conversations go on from 40 positions that a fourth holder keeps, a fifth gives drafts back into a shared page: each one gets
    its last page from et_pages_fork before it grows.  No two have a place in common, and nobody's stored rows change."""
    import torch
    page, n_pages, kvh, d = 16, 60, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(3)
    cache = torch.randn((n_pages, 2, kvh, page, d), device="cuda", generator=gen).to(torch.bfloat16)
    table = np.full((5, 8), -1)
    table[:4, :3] = [7, 30, 12]                                                                  # 40 positions, the last 8 in page 12
    table[4, :4] = [7, 30, 12, 5]                                                                # 55 of which 41 stay, 9 in page 12
    refs = np.bincount(table[table >= 0], minlength=n_pages)
    refs[12] += 1                                                                                # kept for later ones
    r, t, lens, status = i32(refs), i32(table), i32([40, 40, 40, 40, 55]), i32([0])
    before = rows_of(B, cache, t, i32([40, 40, 40, 40, 41]))
    lens = B.et_pages_update(r, page, t, lens, keep=i32([40, 40, 40, 40, 41]), add=i32([0] * 5), status=status)
    other = i32(np.full((5, 8), -1))
    lens, copies = B.et_pages_fork(r, page, t, lens, i32(range(5)), other, status=status)
    B.et_kv_copy(cache, None, copies, status)
    add, offsets, slots = i32([1, 25, 8, 0, 3]), i32([0] * 6), i32([-9] * 37)
    new = B.et_pages_update(r, page, other, lens, add=add, row_offsets=offsets, slots=slots, status=status)
    qkv = torch.randn((37, 2 * kvh * d), device="cuda", generator=gen).to(torch.bfloat16)
    B.et_kv_append(cache, None, qkv, 0, other, lens, offsets, status=status)
    assert status.item() == 0 and new.tolist() == [41, 65, 48, 40, 44]
    places = slots.tolist()
    assert min(places) >= 0 and len(set(places)) == 37 and not {p // page for p in places} & {7, 30, 12}
    now, first = rows_of(B, cache, other, new), offsets.tolist()
    for i in range(5):
        n = len(before[i])
        assert torch.equal(now[i][:n], before[i]) and torch.equal(now[i][n:], qkv[first[i]:first[i + 1]])
    live = np.arange(8) < up(new.cpu().numpy(), page)[:, None]
    held = np.bincount(other.cpu().numpy()[live], minlength=n_pages)
    held[12] += 1
    assert np.array_equal(r.cpu().numpy(), held)


def test_rows_of_a_sequence_that_got_no_place_are_not_written(B):                                # noqa: F811
    """A sequence asks for more than its table holds; its entries behind the used ones name another one's pages, as they may after a fork.
    Appended with a negative start, nothing of its rows is stored anywhere."""
    import torch
    page, n_pages, kvh, d = 16, 20, 1, 64
    gen = torch.Generator(device="cuda").manual_seed(4)
    cache = torch.randn((n_pages, 2, kvh, page, d), device="cuda", generator=gen).to(torch.bfloat16)
    table = np.array([[3, 9, 4, 11], [8, 2, 3, 9]])                                              # 50 positions; 20, and two old entries
    refs = np.zeros(n_pages, int)
    refs[[3, 9, 4, 11, 8, 2]] = 1
    r, t, keep, add, offsets, status = i32(refs), i32(table), i32([50, 20]), i32([3, 60]), i32([0] * 3), i32([0])
    new = B.et_pages_update(r, page, t, keep, add=add, row_offsets=offsets, status=status)
    assert new.tolist() == [53, 20] and status.item() == B.ET_PAGED_CAPACITY
    qkv = torch.randn((63, 2 * kvh * d), device="cuda", generator=gen).to(torch.bfloat16)
    want = cache.clone()
    want[11, :, :, 2:5] = qkv[:3].view(3, 2, kvh, d).permute(1, 2, 0, 3)
    B.et_kv_append(cache, None, qkv, 0, t, torch.where(new - keep == add, keep, -1), offsets)
    assert torch.equal(cache, want)


@pytest.mark.parametrize("n_pages,page", [((1 << 27) - 1, 16), ((1 << 24) - 1, 128)])
def test_update_of_the_largest_pools(B, n_pages, page):                                          # noqa: F811
    """As many pages as slots can name, the free ones far apart and at the very end."""
    import torch
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    free = sorted({0, 77, n_pages // 3, n_pages - 1, n_pages - 2, n_pages - 40_000, n_pages // 2 + 1})
    refs[free] = 0
    table, lens, status = i32(np.full((3, 4), -1)), i32([0, 0, 0]), i32([0])
    add, slots = i32([2 * page, page + 1, 3 * page - 2]), i32([-9] * (6 * page - 1))
    new = B.et_pages_update(refs, page, table, lens, add=add, slots=slots, status=status)
    assert status.item() == 0 and new.tolist() == add.tolist() and not (refs == 0).any() and not (refs != 1).any()
    assert table.tolist() == [free[:2] + [-1, -1], free[2:4] + [-1, -1], free[4:] + [-1]]
    want = [p * page + t for entries, n in zip((free[:2], free[2:4], free[4:]), add.tolist()) for p, t in
            [(entries[i // page], i % page) for i in range(n)]]
    assert slots.tolist() == want


def test_update_of_the_longest_table(B):                                                         # noqa: F811
    """2^30 positions are given back and as many taken, each with its slot."""
    import torch
    page, columns = 128, 1 << 23
    n_pages, cap = columns + 5, 1 << 30
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    refs[-5:] = 0
    table = torch.arange(columns - 1, -1, -1, dtype=torch.int32, device="cuda").view(1, -1)
    status, slots = i32([0]), torch.full((cap,), -9, dtype=torch.int32, device="cuda")
    new = B.et_pages_update(refs, page, table, i32([cap]), keep=i32([0]), add=i32([cap]), slots=slots, status=status)
    assert status.item() == 0 and new.tolist() == [cap]
    assert torch.equal(table[0], torch.arange(columns, dtype=torch.int32, device="cuda"))
    assert torch.equal(slots, torch.arange(cap, dtype=torch.int32, device="cuda"))
    assert (refs[:columns] == 1).all() and (refs[columns:] == 0).all()


@pytest.mark.parametrize("first", [1, 2, 3])
@pytest.mark.parametrize("rows", [2_000, 40_001])
def test_update_into_slots_that_begin_anywhere(B, rows, first):                                  # noqa: F811
    import torch
    rng = np.random.default_rng(rows + first)
    lens, table, refs = random_state(rng, 40, 3000, 32, 2000)
    add = np.minimum(rng.integers(0, 900, 40), table.shape[1] * 32 - np.maximum(lens, 0))
    want = update_reference(refs, 32, table, lens, None, add, rows)
    wide = torch.full((rows + 8,), -77, dtype=torch.int32, device="cuda")
    B.et_pages_update(i32(refs), 32, i32(table), i32(lens), add=i32(add), slots=wide[first:first + rows])
    got, n = wide.cpu().numpy(), len(want[4])
    assert np.array_equal(got[first:first + n], want[4]) and (got[first + n:first + rows] == -1).all()
    assert (got[:first] == -77).all() and (got[first + rows:] == -77).all()


# ---- et_pages_fork ----------------------------------------------------------------------------------------------------

def fork_of_low_counts(refs, page, table, lens, parent, new_table):
    """As fork_reference, for counts that may be lower than the entries that name their pages."""
    refs, new_table = refs.copy(), new_table.copy()
    codes, lengths, kids = set(), [], {}
    for b, p in enumerate(parent):
        if p >= 0:
            kids.setdefault(p, []).append(b)
        lengths.append(max(lens[p], -1) if p >= 0 else -1)

    def down(g):
        if refs[g] <= 0:
            codes.add(7)
        else:
            refs[g] -= 1
    for p in range(len(table)):
        for j in range(up(max(lens[p], 0), page)):
            family = kids.get(p, [])
            if family:
                refs[table[p, j]] += len(family) - 1
            else:
                down(table[p, j])
            for b in family:
                new_table[b, j] = table[p, j]
    last = {}
    for b, n in enumerate(lengths):
        if n > 0 and n % page:
            g, family = new_table[b, n // page], kids[parent[b]]
            if refs[g] <= 0:
                codes.add(7)
            elif not (b == family[0] and refs[g] == len(family)):
                last[b] = g
    free = list(np.nonzero(refs == 0)[0])
    copies = np.array([[-1, -1, 0]] * len(parent))
    for i, (b, g) in enumerate(last.items()):
        down(g)
        assert i < len(free)
        new_table[b, lengths[b] // page] = free[i]
        copies[b] = g, free[i], lengths[b] % page
    for i in range(len(last)):
        refs[free[i]] = 1
    return refs, new_table, np.array(lengths), copies, codes


@pytest.mark.parametrize("wide", [0, 200])
def test_fork_with_counts_that_are_too_low(B, wide):                                              # noqa: F811
    """Half-filled last pages whose counts are 0, below it, or lower than the rows that leave them: no count becomes negative, and no page
    that is copied is another row's new one.  In one launch and in two (wider tables)."""
    page, rows, columns = 16, 12, 4
    table = np.full((rows, columns + wide), -5)
    table[:, :columns] = np.arange(rows * columns).reshape(rows, columns)[:, ::-1]
    lens = np.full(rows, 3 * page + 7)
    refs = np.ones(rows * columns + 30, int)
    refs[rows * columns:] = 0
    parent = np.array([0, 1, 2, 3, 3, 4, 4, 4, 5, 5, 6, 8, 9, 9, 9])                               # rows 7, 10 and 11 end
    for row, count in ((0, 0), (1, -4), (3, 0), (4, -1), (5, 2), (6, 3), (7, 0), (9, -9), (10, -2)):
        refs[table[row, 3]] = count
    refs[table[2, 1]], refs[table[11, 0]] = 0, 0                                                  # whole pages, kept and given up
    for counts in (refs, np.where(refs < 0, refs, np.minimum(refs, 1))):
        new = np.full((len(parent), table.shape[1]), -5)
        want = fork_of_low_counts(counts, page, table, lens, parent, new)
        assert 7 in want[4]
        bufs = [guarded(x) for x in (counts, new, np.full(len(parent), -9), np.full((len(parent), 3), -9))]
        status = i32([0])
        B.et_pages_fork(bufs[0][1], page, i32(table), i32(lens), i32(parent), bufs[1][1], bufs[2][1], bufs[3][1], status)
        assert all(guards_hold(wide) for wide, _ in bufs)
        for (_, got), expected in zip(bufs, want[:4]):
            assert np.array_equal(got.cpu().numpy(), expected)
        assert status.item() == 7
        copied, fresh = want[3][want[3][:, 0] >= 0, 0], want[3][want[3][:, 0] >= 0, 1]
        assert not set(copied) & set(fresh)


# ---- et_beam_select: rows of many chunks, a block each ------------------------------------------------------------------
# From 592 rows on a block walks a whole row, 4 096 logits at a time.

def many_rows(patterns, dtype, rows=600):
    """`rows` rows on the GPU, patterns one after the other and over again."""
    import torch
    x = torch.empty((rows, len(patterns[0])), dtype=dtype, device="cuda")
    for i, y in enumerate(patterns):
        x[i::len(patterns)] = y.to(dtype)
    return x


def check_many(B, patterns, k, dtype, accurate=None):                                            # noqa: F811
    """Each row's best k, in order, and their scores against 64 bits; equal rows have equal results, bit by bit."""
    import torch
    rows, n = 600, len(patterns)
    x = many_rows(patterns, dtype, rows)
    parent, token, score, done = (t.view(rows, k) for t in B.et_beam_select(x, 1, k))
    assert not (done & (parent >= 0)).any()
    for i in range(n):
        y = x[i].double()
        # in descending order, equal ones by their tokens: sort() is stable
        order = torch.sort(y, descending=True, stable=True).indices[:k]
        live = y[order] > -math.inf
        if not math.isfinite(torch.logsumexp(y, 0).item()):
            live[:] = False
        want = torch.where(live, order, -1).int()
        want = torch.cat([want, want.new_full((k - len(want),), -1)])
        assert (token[i::n] == want).all(), i
        assert (parent[i::n] == torch.where(want >= 0, torch.arange(i, rows, n, device="cuda").unsqueeze(1), -1)).all(), i
        assert (score[i::n] == score[i]).all() and (done[i::n] == (want < 0)).all(), i
        got = (want >= 0).sum().item()
        value = y[order[:got]] - torch.logsumexp(y, 0)
        bound = 2.0 ** -20 if y.abs().max() < 2 ** 23 or accurate is None else accurate
        assert ((score[i, :got].double() - value).abs() <= bound + 2.0 ** -24 * value.abs()).all(), i
        assert (score[i, got:] == -math.inf).all()


@pytest.mark.parametrize("fp32", [True, False])
@pytest.mark.parametrize("k", [1, 20, 33, 64])
@pytest.mark.parametrize("vocab", [9 * 4096 + 55, 10 * 4096, 31 * 4096 + 4])
def test_select_of_unlucky_orders_in_long_rows(B, vocab, k, fp32):                               # noqa: F811
    """What floods the list behind the first chunk: rising logits, each chunk above the last, values that are equal across chunks' ends, a
    bar that only the next chunks' equals reach."""
    import torch
    i = torch.arange(vocab, device="cuda").float()
    gen = torch.Generator(device="cuda").manual_seed(k)
    noise = torch.randn(vocab, device="cuda", generator=gen)
    patterns = [i / 512, -i / 512, torch.full_like(i, 0.3), i * 7919 % 3, torch.div(i, 4096, rounding_mode="floor"), -torch.div(i, 4096, rounding_mode="floor"),
                torch.div(i + 2048, 4096, rounding_mode="floor"), torch.where(i % 4096 < 4096 - k, -5.0, 1.0), torch.where(i % 4096 > 4090, 2.0, noise),
                torch.where(i < 2 * 4096, i / 4096, 2.0 - 1e-4 * (i % 3)), noise + i / 20_000, torch.where(i > vocab - 20, 9.0, -9.0), noise * 1000,
                torch.where((i % 4096 // 4 % 256) < 8, 50 + i / 1000, -i / 100)]
    if not fp32:
        patterns = [y * 4 for y in patterns]
    check_many(B, patterns, k, torch.float32 if fp32 else torch.bfloat16)


@pytest.mark.parametrize("fp32", [True, False])
def test_select_of_long_rows_that_are_not_finite(B, fp32):                                       # noqa: F811
    """Banned tokens in whole chunks, infinities and NaN in the first chunk, a middle one and the last one."""
    import torch
    vocab, inf = 12 * 4096 + 7, math.inf
    i = torch.arange(vocab, device="cuda")
    y = torch.randn(vocab, device="cuda")
    patterns = [y, torch.where(i < 4096, -inf, y), torch.where(i >= 4096, -inf, y), torch.where(i // 4096 % 2 == 0, -inf, y), torch.where(i < vocab - 3, -inf, y),
                torch.full_like(y, -inf), torch.where(i % 4096 == 4095, y, -inf)]
    for at in (5, 6 * 4096 + 100, vocab - 1):
        patterns += [torch.where(i == at, math.nan, y), torch.where(i == at, inf, y), torch.where(i == at, -inf, y), torch.where(i == at, 3e38, y),
                     torch.where(i == at, -3e38, y)]
    for k in (3, 64):
        check_many(B, patterns, k, torch.float32 if fp32 else torch.bfloat16)


def sums_patterns(vocab):
    """Rows whose terms round alike: one token, or one of each thread, above equal ones that weigh as much together; rising ones; large
    offsets."""
    import torch
    i = torch.arange(vocab, device="cuda").double()
    one, first = i == vocab // 3, (i < 1024) & (i % 4 == 0)
    got = [torch.where(one, 0, -t) for t in (3.1, 7.77, 9.7, 11.1, 11.46, 12.7, 13.6, 13.75, 13.86)]
    got += [torch.where(first, 0, -t) for t in (3.3, 6.1, 8.3, 11.46)]
    got += [torch.where(one, 0.3, -t) for t in (8.05, 11.2, 13.3)] + [torch.full_like(i, c) for c in (0.1234, -77.7, 1000.1, 40_000.3, -705.2, -706.0, -3543.3)]
    got += [i * 2e-6, i * 1e-4, -i * 2e-6, 5e-8 * i + 1, torch.floor(i / 4096) * 3.9, torch.floor(i / 4096) * 0.7, torch.sin(i) * 3, torch.cos(i * i) * 9 + 700]
    got += [torch.where(one, 0, -t) + c for t in (8.3, 11.46) for c in (17.3, -511.9, 4095.3, 70_000.0)]
    return got


@pytest.mark.parametrize("vocab,fp32", [(152_064, True), (152_064, False), (40_003, True), (600_000, True), (1 << 20, True)])
def test_select_accurate_sums_of_long_rows(B, vocab, fp32):                                      # noqa: F811
    """The logarithm within the documented 2^-20 where a thread adds up the terms of 10 to 256 chunks."""
    import torch
    check_many(B, sums_patterns(vocab), 2, torch.float32 if fp32 else torch.bfloat16)


def test_select_accurate_sums_of_large_logits(B):                                                # noqa: F811
    """Beyond 2^23 logits are whole numbers at least, and the logarithm is within 2^-19."""
    import torch
    vocab = 152_064
    i = torch.arange(vocab, device="cuda").double()
    chunk = torch.floor(i / 4096)
    patterns = [2.0 ** 23 + i % 3, 2.0 ** 23 + chunk * 5, -2.0 ** 24 + 2 * chunk, torch.where(i == 99_000, 2.0 ** 23 + 12, 2.0 ** 23), 2.0 ** 23 - 30 + chunk,
                -2.0 ** 23 + chunk, 1e30 + 0 * i, torch.where(chunk > 20, 2.0 ** 23, -1e30), -3e38 + i * 1e33, torch.where(chunk < 9, -2.0 ** 25, chunk)]
    check_many(B, patterns, 5, torch.float32, accurate=2.0 ** -19)


@pytest.mark.parametrize("n_req,beams,k,vocab", [(65_535, 1, 3, 37), (2_047, 32, 16, 5), (900, 2, 64, 5_001)])
def test_select_of_the_most_rows(B, n_req, beams, k, vocab):                                     # noqa: F811
    """Against a sort of all continuations in 64 bits, where no two are near one another."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn((n_req * beams, vocab), device="cuda", generator=gen) * 3
    scores = torch.randn(n_req * beams, device="cuda", generator=gen)
    parent, token, score, done = (t.view(n_req, k) for t in B.et_beam_select(x, beams, k, scores=scores))
    total = (torch.log_softmax(x.double(), 1) + scores.double().unsqueeze(1)).view(n_req, -1)
    best, at = torch.sort(total, dim=1, descending=True, stable=True)
    n = min(k, beams * vocab)
    clear = torch.ones((n_req, n), dtype=torch.bool, device="cuda")
    gaps = best[:, :-1] - best[:, 1:] > 2.0 ** -18
    clear[:, :min(n, gaps.shape[1])] &= gaps[:, :n]
    clear[:, 1:] &= gaps[:, :n - 1]
    first = torch.arange(n_req, device="cuda").unsqueeze(1) * beams
    assert clear.float().mean() > 0.98
    assert (token[:, :n] == at[:, :n] % vocab)[clear].all() and (parent[:, :n] == first + at[:, :n] // vocab)[clear].all()
    assert ((score[:, :n].double() - best[:, :n]).abs() <= 2.0 ** -20 + 2.0 ** -24 * best[:, :n].abs()).all()
    assert (token[:, n:] == -1).all() and (score[:, n:] == -math.inf).all() and not done[:, :n].any()


def test_calls_at_the_same_time(B):                                                              # noqa: F811
    """The same calls over two states on two streams at once, with a workspace each: as one after the other."""
    import torch
    rng = np.random.default_rng(8)
    states = [random_state(rng, n, 900, 16, 9000) for n in (700, 90)]
    logits = [torch.randn((r, 20_011), device="cuda") for r in (64, 300)]

    def calls(state, x, stream):
        lens, table, refs = state
        with torch.cuda.stream(stream):
            r, t, n, status = i32(refs), i32(table), i32(lens), i32([0])
            other = i32(np.full((2 * len(lens), table.shape[1]), -1))
            parent = i32(np.arange(2 * len(lens)) // 2)
            got = []
            for _ in range(6):
                n = B.et_pages_update(r, 16, t, n, status=status, stream=stream)
                got += [n, *B.et_beam_select(x, 2, 9, stream=stream)]
            got += [*B.et_pages_fork(r, 16, t, n, parent, other, status=status, stream=stream), r, t, other, status]
        return got

    one = torch.cuda.current_stream()
    want = [calls(s, x, one) for s, x in zip(states, logits)]
    torch.cuda.synchronize()
    for _ in range(10):
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        got = [calls(s, x, stream) for s, x, stream in zip(states, logits, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
