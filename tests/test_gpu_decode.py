"""The decode step's operators (include/earlytom_decode.h) against plain implementations in 64 bits: the paged cache (append,
read), attention over it and the dense layer for few rows; then all of them together as one decode step of a model.

Tolerances count roundings: a value rounded to bf16 is off by at most 2^-8 of it, to e4m3 by 2^-4 (or half the smallest step);
fp32 sums of n terms by n * 2^-23 of the sum of magnitudes (the tensor cores may truncate where fp32 addition rounds)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

BF16, E4M3_HALF = 2.0 ** -8, 2.0 ** -4


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2605_30010_b200 import binding
    return binding


# ---- plain implementations (numpy, 64 bits) ---------------------------------------------------------------------------

def code_values():
    got = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        got[c] = (-1.0 if c & 128 else 1.0) * (math.nan if c & 127 == 127 else m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return got


CODES = code_values()


def e4m3_rows(x):
    """x [..., d] in 64 bits -> (codes as values, exponents): the smallest e with max|x| <= 448 * 2^e, then nearest, ties to even."""
    fin = np.where(np.isfinite(x), np.abs(x), 0.0)
    top = fin.max(-1)
    m, ex = np.frexp(top)
    e = np.where(top > 0, ex - 9 + (m > 0.875), -127)
    e = np.clip(e, -127, 127)
    y = np.where(np.isfinite(x), x, np.nan) * np.ldexp(1.0, -e)[..., None]
    step = np.ldexp(1.0, np.maximum(np.frexp(np.abs(np.where(np.isnan(y), 1.0, y)))[1] - 1, -6) - 3)
    return np.round(y / step) * step, e


def rotate(x, pos, theta):
    """x [rows][heads][d], pos [rows]: rotate-half."""
    half = x.shape[-1] // 2
    ang = pos[:, None].astype(np.float64) * float(theta) ** (-np.arange(half) / half)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def f64(t):
    return t.detach().double().cpu().numpy()


def bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def i32(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Cache:
    """A paged cache with every byte of it set to something, and a table of distinct pages for n_seq sequences."""

    def __init__(self, rng, n_seq, max_pages, kv_heads, page, d, e4m3, spare=3):
        import torch
        self.page, self.kv_heads, self.d, self.e4m3 = page, kv_heads, d, e4m3
        self.n_pages = n_seq * max_pages + spare
        shape = (self.n_pages, 2, kv_heads, page, d)
        x = rng.standard_normal(shape) * np.exp2(rng.integers(-3, 4, shape[:-1]))[..., None]
        if e4m3:
            v, e = e4m3_rows(x)
            self.data = torch.from_numpy(v.astype(np.float32)).cuda().to(torch.float8_e4m3fn)
            self.scale = torch.from_numpy((e + 127).astype(np.uint8)).cuda()
        else:
            self.data, self.scale = bf16(x), None
        self.table = i32(rng.permutation(self.n_pages)[:n_seq * max_pages].reshape(n_seq, max_pages))

    def bytes(self):
        import torch
        return self.data.view(torch.uint8 if self.e4m3 else torch.int16).clone(), None if self.scale is None else self.scale.clone()

    def values(self):
        import torch
        if not self.e4m3:
            return f64(self.data)
        return CODES[self.data.view(torch.uint8).cpu().numpy()] * np.ldexp(1.0, self.scale.cpu().numpy().astype(int) - 127)[..., None]

    def rows(self, s, first, n, values=None):
        """[2][kv_heads][n][d] of sequence s."""
        values = self.values() if values is None else values
        pos = np.arange(first, first + n)
        pages = self.table.cpu().numpy()[s][pos // self.page]
        return values[pages, :, :, pos % self.page].transpose(1, 2, 0, 3)


# ---- append and read --------------------------------------------------------------------------------------------------

APPENDS = [
    # rows of each sequence, start of each, heads, kv_heads, page, d, theta
    ([1], [0], 4, 2, 16, 64, 1e4),
    ([1], [7675], 28, 4, 64, 128, 1e6),
    ([1, 1, 1, 1, 1], [0, 15, 16, 31, 100], 7, 1, 16, 128, 1e6),
    ([37, 1, 0, 64, 129], [0, 63, 5, 1, 127], 6, 2, 32, 128, 5e5),
    ([200], [3], 0, 4, 128, 128, 0.0),
    ([5, 300, 17], [1000, 0, 2], 0, 3, 16, 64, 0.0),
    ([2, 3], [10, 20], 5, 5, 64, 64, 0.0),
    ([(7 * i) % 5 for i in range(150)], [(37 * i) % 91 for i in range(150)], 2, 2, 16, 64, 1e4),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_then_read(B, case, e4m3):
    import torch
    counts, starts, heads, kvh, page, d, theta = APPENDS[case]
    rng = np.random.default_rng(case)
    n_seq, rows = len(counts), sum(counts)
    max_pages = max((s + n + page - 1) // page for s, n in zip(starts, counts)) + 1
    c = Cache(rng, n_seq, max_pages, kvh, page, d, e4m3)
    data0, scale0 = c.bytes()
    pad, extra = 3, 16                                # rows behind the last sequence; columns that belong to something else
    x = rng.standard_normal((rows + pad, (heads + 2 * kvh) * d)) * np.exp2(rng.integers(-6, 7, (rows + pad, 1)))
    wide = torch.full((rows + pad, x.shape[1] + extra), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :x.shape[1]] = bf16(x)
    qkv = wide[:, :x.shape[1]]
    x = f64(qkv).reshape(rows + pad, heads + 2 * kvh, d)
    one_each = counts == [1] * n_seq
    offsets = None if one_each else i32(np.concatenate([[0], np.cumsum(counts)]))
    if one_each:
        qkv, pad = qkv[:rows], 0
    status, new_len = i32([0]), i32([-9] * n_seq)
    q_out = torch.full((rows + pad, heads * d), 7.0, dtype=torch.bfloat16, device="cuda") if theta and heads else None
    before = qkv.clone()
    B.et_kv_append(c.data, c.scale, qkv, heads, c.table, i32(starts), offsets, theta, q_out, new_len, status)
    torch.cuda.synchronize()
    assert status.item() == 0
    assert new_len.tolist() == [s + n for s, n in zip(starts, counts)]
    assert torch.equal(before, qkv)
    pos = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, counts)])
    seq = np.repeat(np.arange(n_seq), counts)
    k, v, q = x[:rows, heads:heads + kvh], x[:rows, heads + kvh:], x[:rows, :heads]
    # a turned value is off by the fp32 roundings of two products, their factors and the angle, and by its own rounding
    def slack(z):
        return 2.0 ** -20 * (np.abs(z) + np.abs(np.roll(z, d // 2, -1)))
    ks = np.zeros_like(k)
    if theta:
        ks, qs = slack(k), slack(q)
        k, q = rotate(k, pos, theta), rotate(q, pos, theta)
        if heads:
            got = f64(q_out[:rows]).reshape(q.shape)
            assert (np.abs(got - q) <= BF16 * np.abs(q) + qs).all()
            assert (q_out[rows:] == 7.0).all()
    want = np.stack([k, v], 1)                                                  # [rows][2][kvh][d]
    places = c.table.cpu().numpy()[seq, pos // page], pos % page
    got = c.values()[places[0], :, :, places[1]]
    if not e4m3:
        tol = BF16 * np.abs(want)
        tol[:, 0] += ks
        if not theta:
            assert np.array_equal(got, want)
        assert (np.abs(got - want) <= tol).all()
    else:
        exp = c.scale.cpu().numpy().astype(int)[places[0], :, :, places[1]] - 127
        vals, e = e4m3_rows(want)
        sure = slice(1, 2) if theta else slice(0, 2)                            # planes that no fp32 rounding touched
        assert np.array_equal(exp[:, sure], e[:, sure])
        assert np.array_equal(got[:, sure], (vals * np.ldexp(1.0, e)[..., None])[:, sure])
        top = np.abs(want).max(-1)
        assert (top <= 448 * np.ldexp(1.0, exp) * (1 + 2.0 ** -18)).all() and (top > 224 * np.ldexp(1.0, exp) * (1 - 2.0 ** -18)).all()
        assert (np.abs(got - want)[:, 0] <= E4M3_HALF * np.abs(want[:, 0]) + np.ldexp(2.0 ** -10, exp)[:, 0, :, None] + 2 * ks).all()
    # nothing else was written
    data1, scale1 = c.bytes()
    touched = torch.zeros((c.n_pages, page), dtype=torch.bool, device="cuda")
    touched[torch.from_numpy(places[0]).cuda().long(), torch.from_numpy(places[1]).cuda().long()] = True
    keep = ~touched[:, None, None, :].expand(c.n_pages, 2, kvh, page)
    assert torch.equal(data0[keep], data1[keep])
    if e4m3:
        assert torch.equal(scale0[keep], scale1[keep])
    # and the rows come back as they are stored
    out = torch.full((rows + pad, 2 * kvh * d + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    B.et_kv_read(c.data, c.scale, c.table, i32(starts), rows + pad, offsets, out[:, :2 * kvh * d], status)
    torch.cuda.synchronize()
    assert np.array_equal(f64(out[:rows, :2 * kvh * d]), got.reshape(rows, -1))
    assert (out[rows:] == 5.0).all() and (out[:, 2 * kvh * d:] == 5.0).all() and status.item() == 0


@pytest.mark.parametrize("d,theta,start", [(128, 1e6, 0), (128, 1e4, 900_000), (64, 5e5, 0), (64, 1e4, 77_777)])
def test_turned_keys_are_exact(B, d, theta, start):
    """A turned key on its way to e4m3 is off by two fp32 roundings (and 2^-39 of the pair that it comes from): what is stored lies
    between the conversions of the two ends of that interval, in all of two million values."""
    n, kvh, heads, page = 4000, 4 if d == 128 else 8, 1, 128
    rng = np.random.default_rng(d + start)
    first = start // page
    max_pages = (start + n + page - 1) // page
    c = Cache(rng, 1, max_pages - first, kvh, page, d, True)
    table = i32(np.concatenate([np.zeros(first), c.table.cpu().numpy()[0]])[None])
    qkv = bf16(rng.standard_normal((n, (heads + 2 * kvh) * d)))
    status = i32([0])
    B.et_kv_append(c.data, c.scale, qkv, heads, table, i32([start]), i32([0, n]), theta=theta, status=status)
    assert status.item() == 0
    x = f64(qkv).reshape(n, heads + 2 * kvh, d)[:, heads:heads + kvh]
    pos = np.arange(start, start + n)
    want = rotate(x, pos, theta)
    pages, place = table.cpu().numpy()[0][pos // page], pos % page
    got = c.values()[pages, 0, :, place]
    e = c.scale.cpu().numpy().astype(int)[pages, 0, :, place] - 127
    # the reference's angles, up to 2^20, are off by 2^-53 of them for the frequency and as much for the product: 2^-32
    slack = 2.0 ** -23 * np.abs(want) + 2.0 ** -31 * (np.abs(x) + np.abs(np.roll(x, d // 2, -1)))

    def nearest(y):
        y = y * np.ldexp(1.0, -e)[..., None]
        step = np.ldexp(1.0, np.maximum(np.frexp(np.abs(y))[1] - 1, -6) - 3)
        return np.round(y / step) * step * np.ldexp(1.0, e)[..., None]

    top = np.abs(want).max(-1)
    assert (top <= 448 * np.ldexp(1.0, e) * (1 + 2.0 ** -22)).all() and (top >= 224 * np.ldexp(1.0, e) * (1 - 2.0 ** -22)).all()
    assert ((nearest(want - slack) <= got) & (got <= nearest(want + slack))).all()


def test_append_with_one_theta_after_another(B):
    """Calls with different bases and head sizes in turn, far positions: each turns by its own angles."""
    import torch
    rng = np.random.default_rng(17)
    for d, theta, start in ((128, 1e6, 1_000_000), (64, 1e4, 5), (128, 1e4, 70_000), (64, 5e5, 2_000_000), (128, 1e6, 999_983)):
        page, kvh, heads = 128, 1, 2
        max_pages = start // page + 1
        c = Cache(rng, 1, 1, kvh, page, d, False)
        table = i32(np.zeros((1, max_pages)))
        x = bf16(rng.standard_normal((1, (heads + 2 * kvh) * d)))
        q = B.et_kv_append(c.data, None, x, heads, table, i32([start]), theta=theta)
        v = f64(x).reshape(1, heads + 2 * kvh, d)
        want = rotate(v, np.array([start]), theta)
        tol = BF16 * np.abs(want) + 2.0 ** -20 * (np.abs(v) + np.abs(np.roll(v, d // 2, -1)))
        assert (np.abs(f64(q).reshape(1, heads, d) - want[:, :heads]) <= tol[:, :heads]).all()
        assert (np.abs(f64(c.data[0, 0, 0, start % page]) - want[0, heads]) <= tol[0, heads]).all()


def test_e4m3_conversion_edges(B):
    """Ties, the border between two exponents, the smallest and largest rows, zeros, NaN and infinities."""
    import torch
    d, kvh, page = 64, 1, 16
    rng = np.random.default_rng(5)
    rows = [np.zeros(d), np.full(d, 448.0), np.full(d, 450.0), np.full(d, 447.0), np.full(d, -448.0 * 2.0 ** 30), np.full(d, 2.0 ** -133),
            np.full(d, 2.0 ** 127 * 1.75), np.linspace(-1, 1, d), np.r_[448.0, np.arange(d - 1) / 8 + 1 / 16],
            np.r_[448.0, (np.arange(d - 1) - 20) * 2.0 ** -10], np.r_[math.nan, np.ones(d - 1)], np.r_[math.inf, -math.inf, np.ones(d - 2) * 3],
            np.full(d, math.nan), np.r_[math.inf, np.zeros(d - 1)], np.r_[-0.0, np.ones(d - 1)], np.r_[1e-38, np.zeros(d - 1)]]
    x = np.stack([np.concatenate([r, rng.standard_normal(d)]) for r in rows])
    c = Cache(rng, 1, 1, kvh, page, d, True)
    qkv = bf16(x)
    x = f64(qkv).reshape(len(rows), 2, d)
    status = i32([0])
    B.et_kv_append(c.data, c.scale, qkv, 0, c.table, i32([0]), i32([0, len(rows)]), status=status)
    got = c.rows(0, 0, len(rows))[:, 0].transpose(1, 0, 2)
    vals, e = e4m3_rows(x)
    want = vals * np.ldexp(1.0, e)[..., None]
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[10, 0, 0]) and np.isnan(got[11, 0, :2]).all() and (got[11, 0, 2:] == 3).all()
    out = B.et_kv_read(c.data, c.scale, c.table, i32([0]), len(rows), i32([0, len(rows)]))
    back = f64(out).reshape(x.shape)
    assert np.array_equal(back, f64(bf16(want)), equal_nan=True) and status.item() == 0


def test_read_at_the_ends_of_bf16(B):
    """Rows read from an e4m3 cache: exact from 2^-130 on, bf16's smallest steps below, infinite from 2^128 on."""
    d, kvh, page = 64, 1, 16
    rng = np.random.default_rng(6)
    c = Cache(rng, 1, 1, kvh, page, d, True)
    codes = np.arange(256, dtype=np.uint8).reshape(1, 4, 64)                    # four rows hold every code
    scales = [0, 1, 2, 7, 120, 246, 247]                                        # bytes; 2^(b - 127)
    import torch
    for b in scales:
        c.data.view(torch.uint8)[c.table[0, 0].long(), 0, 0, :4] = torch.from_numpy(codes[0]).cuda()
        c.scale[c.table[0, 0].long(), 0, 0, :4] = b
        out = B.et_kv_read(c.data, c.scale, c.table, i32([0]), 4, i32([0, 4]))[:, :d]
        want = CODES[codes[0]] * 2.0 ** (b - 127)
        with np.errstate(over="ignore"):
            nearest = f64(bf16(want))
        assert np.array_equal(f64(out), nearest, equal_nan=True)
        exact = np.isnan(want) | ((np.abs(want) >= 2.0 ** -130) & (np.abs(want) < 2.0 ** 128)) | (want == 0)
        assert np.array_equal(f64(out)[exact], want[exact], equal_nan=True)
        assert np.isinf(f64(out)[np.abs(want) >= 2.0 ** 128]).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_rows_that_cannot_be_placed_are_skipped(B, e4m3):
    """Slots not in use, positions behind the table, pages that are not in the cache: skipped and reported, the others land."""
    import torch
    rng = np.random.default_rng(9)
    kvh, page, d, heads = 2, 16, 64, 2
    c = Cache(rng, 4, 2, kvh, page, d, e4m3)
    good = c.table.clone()
    for bad, code in ((c.n_pages, B.ET_PAGED_BAD_PAGE), (-1, B.ET_PAGED_BAD_PAGE), (None, B.ET_PAGED_CAPACITY), ("off", 0)):
        table, start = good.clone(), [3, 17, 30, 9]
        if bad is None:
            start[1] = 32
        elif bad == "off":
            start[1] = -1
        else:
            table[1, 1] = bad
        data0, scale0 = c.bytes()
        qkv, status, new_len = bf16(rng.standard_normal((4, (heads + 2 * kvh) * d))), i32([0]), i32([0] * 4)
        q = torch.full((4, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
        B.et_kv_append(c.data, c.scale, qkv, heads, table, i32(start), theta=1e4, q_out=q, new_len=new_len, status=status)
        assert status.item() == code
        assert new_len.tolist() == [4, {None: 32, "off": -1}.get(bad, 18), 31, 10]
        assert (q[1] == 7.0).all() and not (q[[0, 2, 3]] == 7.0).all(1).any()
        data1, _ = c.bytes()
        changed = {tuple(i) for i in (data0 != data1).any(-1).any(2).any(1).nonzero().tolist()}
        assert changed == {(good[s, start[s] // page].item(), start[s] % page) for s in (0, 2, 3)}
        out = torch.full((4, 2 * kvh * d), 5.0, dtype=torch.bfloat16, device="cuda")
        status.zero_()
        B.et_kv_read(c.data, c.scale, table, i32(start), 4, None, out, status)
        assert status.item() == code and (out[1] == 5.0).all()
        for s in (0, 2, 3):
            assert np.array_equal(f64(out[s]), c.rows(s, start[s], 1).reshape(-1))


def test_new_lengths_stay_within_the_table(B):
    """new_len is never more than the table's pages hold, also where a sequence started behind them; a negative start stays."""
    rng = np.random.default_rng(10)
    kvh, page, d = 1, 16, 64
    starts = [33, 32, 31, 2 ** 31 - 1, 40, -5, 2 ** 31 - 3, 0]
    counts = [1, 2, 4, 3, 0, 1, 3, 2]
    c = Cache(rng, len(starts), 2, kvh, page, d, False)
    rows = bf16(rng.standard_normal((sum(counts), 2 * kvh * d)))
    new, status = i32([-9] * len(starts)), i32([0])
    B.et_kv_append(c.data, None, rows, 0, c.table, i32(starts), i32(np.concatenate([[0], np.cumsum(counts)])), new_len=new, status=status)
    assert new.tolist() == [32, 32, 32, 32, 32, -5, 32, 2] and status.item() == B.ET_PAGED_CAPACITY
    n = len(starts)
    new.fill_(-9)
    B.et_kv_append(c.data, None, rows[:n], 0, c.table, i32(starts), new_len=new)          # one row for each
    assert new.tolist() == [32, 32, 32, 32, 32, -5, 32, 1]


@pytest.mark.parametrize("e4m3", [False, True])
def test_offsets_that_do_not_fit_write_nothing_outside(B, e4m3):
    """Offsets far below zero (a row's distance from them passes 32 bits), falling ones and ones behind the rows: nothing is placed
    where no row belongs, and new lengths count only rows that the call has."""
    import torch
    rng = np.random.default_rng(11)
    kvh, page, d, rows = 1, 16, 64, 6
    c = Cache(rng, 2, 2, kvh, page, d, e4m3)
    x = bf16(rng.standard_normal((rows, 2 * kvh * d)))
    low = -2 ** 31
    for offsets, start, placed, lengths, code in (
            ([low, low + 1, 6], [0, 3], [], [0, 9], B.ET_PAGED_CAPACITY),       # rows stand 2^31 and more behind the second offset
            ([low, 6, 6], [20, 0], [], [26, 0], B.ET_PAGED_CAPACITY),
            ([0, 6, 2], [4, 30], [(0, 4 + i) for i in range(6)], [10, 30], 0),
            ([0, 4, 2 ** 31 - 1], [1, 2], [(0, 1 + i) for i in range(4)] + [(1, 2), (1, 3)], [5, 4], 0),
            ([9, 12, 15], [1, 2], [], [1, 2], 0)):
        before, _ = c.bytes()
        new, status = i32([-9, -9]), i32([0])
        B.et_kv_append(c.data, c.scale, x, 0, c.table, i32(start), i32(offsets), new_len=new, status=status)
        after, _ = c.bytes()
        changed = {tuple(i) for i in (before != after).any(-1).any(2).any(1).nonzero().tolist()}
        assert changed == {(c.table[s, p // page].item(), p % page) for s, p in placed}
        assert new.tolist() == lengths and status.item() == code
        out = torch.full((rows, 2 * kvh * d), 5.0, dtype=torch.bfloat16, device="cuda")
        status.zero_()
        B.et_kv_read(c.data, c.scale, c.table, i32(start), rows, i32(offsets), out, status)
        assert ((out == 5.0).all(1).sum().item() == rows - len(placed)) and status.item() == code
        c.data.view(torch.uint8 if e4m3 else torch.int16).copy_(before)


# ---- attention --------------------------------------------------------------------------------------------------------

def attention_reference(q, k, v):
    """q [heads][d], k, v [kv_heads][n][d] in 64 bits: (out, lse, sum p|v|, max sum |q||k|)."""
    heads, d = q.shape
    group = heads // k.shape[0]
    k, v = np.repeat(k, group, 0), np.repeat(v, group, 0)
    s = np.einsum("hd,hnd->hn", q, k) / math.sqrt(d)
    size = (np.einsum("hd,hnd->hn", np.abs(q), np.abs(k)) / math.sqrt(d)).max(-1)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    lse = np.log(p.sum(-1)) + top[:, 0]
    p /= p.sum(-1, keepdims=True)
    return np.einsum("hn,hnd->hd", p, v), lse, np.einsum("hn,hnd->hd", p, np.abs(v)), size


def check_attention(out, lse, q, lens, cache, heads, alive=None, values=None):
    """Scores of d fp32 products are off by d * 2^-23 of the sum of magnitudes, and the exponentials by as much relatively (plus
    2^-20 for themselves and their sum); a probability rounded to 11 bits by 2^-11."""
    d = cache.d
    values = cache.values() if values is None else values
    for s, n in enumerate(lens):
        if n <= 0:
            assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
            continue
        k, v = cache.rows(s, 0, n, values)
        if alive is not None:
            k, v = k[:, alive[s][:n]], v[:, alive[s][:n]]
        want, wl, mass, size = attention_reference(q[s], k, v)
        drift = d * 2.0 ** -23 * size + 2.0 ** -20
        got = f64(out[s]).reshape(heads, d)
        tol = BF16 * np.abs(want) + (2.0 ** -11 + 2 * drift)[:, None] * mass + 1e-30
        assert (np.abs(got - want) <= tol).all(), f"sequence {s} of {n}: off by {(np.abs(got - want) / tol).max():.3g} of the tolerance"
        assert (np.abs(f64(lse[s]) - wl) <= drift + 2.0 ** -22 * np.abs(wl)).all()


def run_attention(B, q, heads, c, lens, table=None, **kw):
    import torch
    n_seq = q.shape[0]
    out = torch.full((n_seq, heads * c.d), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n_seq, heads), 9.0, dtype=torch.float32, device="cuda")
    status = i32([0])
    B.et_attention_paged(q, heads, c.data, c.scale, c.table if table is None else table, i32(lens), out=out, lse=lse, status=status, **kw)
    torch.cuda.synchronize()
    return out, lse, status.item()


ATTENTIONS = [
    # lengths, heads, kv_heads, page
    ([1], 4, 4, 16),
    ([61], 28, 4, 16),
    ([64, 65, 63, 0, 1, 2, 15, 16, 17, 31, 33, 127, 128, 129, -4], 7, 1, 16),
    ([300, 0, 1023], 10, 2, 32),
    ([513, 40], 16, 2, 64),
    ([700, 1], 9, 1, 128),
    ([257, 256], 23, 1, 64),
    ([150, 31], 80, 2, 32),
    ([5000], 28, 4, 64),
    ([4097, 3, 2000], 8, 8, 128),
    (list(range(0, 200, 3)), 4, 2, 16),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(ATTENTIONS)))
def test_attention(B, case, d, e4m3):
    lens, heads, kvh, page = ATTENTIONS[case]
    rng = np.random.default_rng(100 * case + d + e4m3)
    c = Cache(rng, len(lens), max(1, (max(lens) + page - 1) // page), kvh, page, d, e4m3)
    q = bf16(rng.standard_normal((len(lens), heads * d)) * 2)
    out, lse, status = run_attention(B, q, heads, c, lens)
    assert status == 0
    check_attention(out, lse, f64(q).reshape(len(lens), heads, d), lens, c, heads)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,kvh,page,d,longest", [(8, 8, 16, 64, 300), (28, 4, 32, 128, 400), (16, 1, 64, 128, 900), (6, 2, 16, 64, 1000), (2, 1, 32, 64, 90)])
def test_attention_many_short_sequences(B, heads, kvh, page, d, longest, e4m3):
    """Many more sequences than SMs, of very different lengths in no order, some empty: every CTA has many pieces."""
    rng = np.random.default_rng(heads * 7 + e4m3)
    n_seq = 331 if longest > 100 else 1500
    lens = [int(longest * x ** 3) for x in rng.random(n_seq)]
    lens[5:9] = [longest, 0, 1, longest]
    c = Cache(rng, n_seq, (longest + page - 1) // page, kvh, page, d, e4m3)
    q = bf16(rng.standard_normal((n_seq, heads * d)))
    out, lse, status = run_attention(B, q, heads, c, lens)
    assert status == 0
    check_attention(out, lse, f64(q).reshape(n_seq, heads, d), lens, c, heads, values=c.values())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,kvh,page,d", [(56, 8, 64, 128), (80, 8, 16, 128), (8, 8, 32, 64), (128, 8, 128, 64)])
def test_attention_long_runs(B, heads, kvh, page, d, e4m3):
    """Enough positions that every CTA goes round its ring of stages many times, pages out of order, a second sequence behind the
    long one; reference in 64 bits on the GPU."""
    import torch
    rng = np.random.default_rng(heads + e4m3)
    lens, gen = [40000, 777], torch.Generator(device="cuda").manual_seed(heads)
    max_pages = (max(lens) + page - 1) // page
    n_pages = 2 * max_pages
    table = i32(rng.permutation(n_pages).reshape(2, max_pages))
    rows = torch.randn((sum(lens), 2 * kvh * d), device="cuda", generator=gen, dtype=torch.bfloat16)
    data = torch.zeros((n_pages, 2, kvh, page, d), device="cuda", dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    scale = torch.zeros((n_pages, 2, kvh, page), device="cuda", dtype=torch.uint8) if e4m3 else None
    start, offsets = i32([0, 0]), i32([0, lens[0], sum(lens)])
    B.et_kv_append(data, scale, rows, 0, table, start, offsets)
    stored = B.et_kv_read(data, scale, table, start, sum(lens), offsets).double().view(-1, 2, kvh, d)
    q = torch.randn((2, heads * d), device="cuda", generator=gen, dtype=torch.bfloat16)
    lse = torch.empty((2, heads), device="cuda")
    for _ in range(3):
        status = i32([0])
        out = B.et_attention_paged(q, heads, data, scale, table, i32(lens), lse=lse, status=status)
        assert status.item() == 0
        for s in range(2):
            k, v = (stored[offsets[s]:offsets[s + 1], i].permute(1, 0, 2) for i in (0, 1))
            qs = q[s].double().view(kvh, heads // kvh, d)
            z = qs @ k.transpose(1, 2) / math.sqrt(d)
            size = (qs.abs() @ k.abs().transpose(1, 2)).amax(-1) / math.sqrt(d)
            p = torch.softmax(z, -1)
            want, mass = p @ v, p @ v.abs()
            drift = d * 2.0 ** -23 * size + 2.0 ** -20
            off = (out[s].double().view_as(want) - want).abs()
            # a sum of n positive weights in fp32, pieces of at most 64 of them joined: n / 64 more roundings
            tol = BF16 * want.abs() + ((2.0 ** -11 + 2 * drift).unsqueeze(-1) + lens[s] / 64 * 2.0 ** -23) * mass
            assert (off <= tol).all()
            assert ((lse[s].double().view(kvh, -1) - torch.logsumexp(z, -1)).abs() <= drift + lens[s] / 64 * 2.0 ** -23 + 2.0 ** -19).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,n,rising", [(2, 1_000_000, False), (12, 1_000_000, False), (2, 300_000, True), (12, 300_000, True)])
def test_attention_long_sums(B, heads, n, rising, e4m3):
    """As many sequences as CTAs, over the same pages, of up to a million positions each and with positive values: the tensor core cuts
    off what does not fit an accumulator, 2^-23 of it for each of the 1024 instructions (or fewer) after which it starts again from
    zero.  The values follow the keys, so that the outputs differ by more than their rounding, which vanishes in the mean over
    3 000 of them (to 1e-4, five times its spread).  rising: scores grow along the cache, by 60 nats in all."""
    import torch
    kvh, page, d, n_seq = 1, 128, 128, 148
    gen = torch.Generator(device="cuda").manual_seed(n + heads)
    pages = (n + page - 1) // page
    k = torch.randn((n, d), device="cuda", generator=gen)
    v = (3 + k + 0.5 * torch.randn((n, d), device="cuda", generator=gen)).clamp(min=0.01) * torch.exp2(torch.arange(d, device="cuda") / d)
    if rising:
        k[:, 0] = torch.linspace(-30, 30, n, device="cuda") * math.sqrt(d) / 16
    rows = torch.cat([k, v], 1).to(torch.bfloat16)
    data = torch.zeros((pages, 2, kvh, page, d), device="cuda", dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    scale = torch.zeros((pages, 2, kvh, page), device="cuda", dtype=torch.uint8) if e4m3 else None
    table = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32).view(1, -1)
    B.et_kv_append(data, scale, rows, 0, table, i32([0]), i32([0, n]))
    k, v = B.et_kv_read(data, scale, table, i32([0]), n, i32([0, n])).double().split(d, 1)
    q = torch.randn((n_seq, heads, d), device="cuda", generator=gen)
    if rising:
        q[:, :, 0] = 16.0
    q = q.to(torch.bfloat16)
    lse = torch.empty((n_seq, heads), device="cuda")
    out = B.et_attention_paged(q.view(n_seq, -1), heads, data, scale, table.expand(n_seq, -1).contiguous(), i32([n] * n_seq), lse=lse)
    mean = []
    for s in range(0, n_seq, 13):
        z = q[s].double() @ k.T / math.sqrt(d)
        size = (q[s].double().abs() @ k.abs().T).amax(-1) / math.sqrt(d)
        want = torch.softmax(z, -1) @ v
        drift = d * 2.0 ** -23 * size + 2.0 ** -20
        off = (out[s].view(heads, d).double() - want) / want
        assert (off.abs() <= BF16 + 2.0 ** -11 + 2 * drift.unsqueeze(-1)).all(), f"{off.abs().max().item():.3g}"
        assert ((lse[s].double() - torch.logsumexp(z, -1)).abs() <= drift + n / 512 * 2.0 ** -24 + 2.0 ** -19).all()
        mean.append(off)
    mean = torch.stack(mean).mean().item()
    assert abs(mean) <= 1024 * 2.0 ** -23 + 1e-4, mean


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,kvh,d", [(1, 1, 128), (14, 2, 64), (23, 1, 128)])
def test_attention_long_runs_of_uneven_sequences(B, heads, kvh, d, e4m3):
    """Runs of more tiles than a piece has, that begin and end anywhere in sequences of very different lengths: every way in which
    pieces go on from one another, inside a CTA and from one to the next; the workspace is full of NaN before.  Scores rise along
    the cache, so that the pieces' maxima differ."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(heads)
    rng = np.random.default_rng(heads + e4m3)
    page, longest = 64, 600_000
    lens = [int(x) for x in rng.integers(1, longest, 44 // kvh)]
    lens[2], lens[5], lens[8], lens[9], lens[-1] = longest, 1, 0, 130, 65_536
    pages = longest // page
    rows = torch.randn((longest, 2, kvh, d), device="cuda", generator=gen)
    rows[:, 0, :, 0] = (torch.linspace(-20, 20, longest, device="cuda") * math.sqrt(d) / 16).unsqueeze(1)
    rows[:, 1] += torch.linspace(-2, 2, longest, device="cuda").view(-1, 1, 1)
    data = torch.zeros((pages, 2, kvh, page, d), device="cuda", dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16)
    scale = torch.zeros((pages, 2, kvh, page), device="cuda", dtype=torch.uint8) if e4m3 else None
    table = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32).view(1, -1)
    B.et_kv_append(data, scale, rows.to(torch.bfloat16).view(longest, -1), 0, table, i32([0]), i32([0, longest]))
    stored = B.et_kv_read(data, scale, table, i32([0]), longest, i32([0, longest])).view(longest, 2, kvh, d)
    n_seq = len(lens)
    q = torch.randn((n_seq, kvh, heads // kvh, d), device="cuda", generator=gen)
    q[:, :, :, 0] = 16 * torch.rand((n_seq, kvh, heads // kvh), device="cuda", generator=gen)      # some flat, some steep
    q = q.to(torch.bfloat16)
    lse, status = torch.empty((n_seq, heads), device="cuda"), i32([0])
    ws = torch.full((B.ET_PAGED_WORKSPACE,), 255, dtype=torch.uint8, device="cuda")
    out = B.et_attention_paged(q.view(n_seq, -1), heads, data, scale, table.expand(n_seq, -1).contiguous(), i32(lens), lse=lse,
                               workspace=ws, status=status)
    assert status.item() == 0
    for s, n in enumerate(lens):
        got, got_lse = out[s].view(kvh, -1, d).double(), lse[s].view(kvh, -1).double()
        if n == 0:
            assert (got == 0).all() and (got_lse == -math.inf).all()
            continue
        for h in range(kvh):
            k, v, qs = stored[:n, 0, h].double(), stored[:n, 1, h].double(), q[s, h].double()
            z = qs @ k.T / math.sqrt(d)
            drift = d * 2.0 ** -23 * (qs.abs() @ k.abs().T).amax(-1) / math.sqrt(d) + 2.0 ** -20
            p = torch.softmax(z, -1)
            want, mass = p @ v, p @ v.abs()
            # 1024 instructions of the tensor core between sums in fp32, of which there are n / 512 and fewer
            tol = BF16 * want.abs() + (2.0 ** -11 + 2 * drift + 1024 * 2.0 ** -23 + n / 512 * 2.0 ** -24).unsqueeze(-1) * mass
            off = (got[h] - want).abs() / tol
            assert (off <= 1).all(), f"sequence {s} of {n}: off by {off.max().item():.3g} of the tolerance"
            assert ((got_lse[h] - torch.logsumexp(z, -1)).abs() <= drift + n / 512 * 2.0 ** -24 + 2.0 ** -19).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_peaked_and_far_apart_scores(B, e4m3):
    """Scores from one key that takes all to thousands apart, growing and falling along the cache; queries of very different
    sizes; values of very different sizes, the large ones where nothing looks."""
    rng = np.random.default_rng(77)
    n, heads, kvh, page, d = 900, 6, 2, 32, 128
    c = Cache(rng, 2, (n + page - 1) // page, kvh, page, d, e4m3)
    q = rng.standard_normal((2, heads, d))
    q *= np.array([1e-6, 0.1, 1.0, 8.0, 40.0, 1000.0])[None, :, None]
    x = np.empty((2 * n, 2, kvh, d))
    for s, sign in ((0, 1.0), (1, -1.0)):
        ramp = sign * np.linspace(-3, 3, n)[:, None, None]
        x[s * n:(s + 1) * n, 0] = rng.standard_normal((n, kvh, d)) * 0.5 + ramp * rng.standard_normal((1, kvh, d))
        x[s * n:(s + 1) * n, 1] = rng.standard_normal((n, kvh, d)) * np.exp2(rng.integers(-12, 13, (n, kvh, 1)))
    B.et_kv_append(c.data, c.scale, bf16(x.reshape(2 * n, -1)), 0, c.table, i32([0, 0]), i32([0, n, 2 * n]))
    qt = bf16(q.reshape(2, -1))
    out, lse, status = run_attention(B, qt, heads, c, [n, n - 7])
    assert status == 0
    check_attention(out, lse, f64(qt).reshape(2, heads, d), [n, n - 7], c, heads)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("heads,n", [(6, 150), (24, 150), (6, 9000), (24, 9000)])
def test_attention_large_values_in_one_dimension(B, heads, n, e4m3):
    """Live rows of values with one large dimension (and zeros beside it) among ordinary rows, at equal, higher and lower scores:
    the other dimensions, to which the large rows give nothing, have to be right on their own.  A weight has 11 bits or more down
    to 2^-21 of the largest probability, whatever the rows' scales are, and is off by 2^-32 of it at most below."""
    import torch
    kvh, page, d = 2, 32, 128
    sizes = [2.0 ** p for p in (3, 9, 15, 21, 40, 90)]
    gaps = [0.0, 8.0, -8.0]                                  # natural logarithm of a large row's weight over an ordinary one's
    cases = [(a, g) for a in sizes for g in gaps]
    rng = np.random.default_rng(heads + n)
    n_seq = len(cases)
    c = Cache(rng, n_seq, (n + page - 1) // page, kvh, page, d, e4m3)
    q = np.zeros((n_seq, heads, d))
    q[:, :, 0] = 16.0
    q[:, :, 1:] = rng.standard_normal((n_seq, heads, d - 1)) * 0.25
    x = np.empty((n_seq, n, 2, kvh, d))
    x[:, :, 0] = rng.standard_normal((n_seq, n, kvh, d)) * 0.25
    x[:, :, 1] = rng.standard_normal((n_seq, n, kvh, d))
    x[:, :, 0, :, 0] = 0.0
    for s, (size, gap) in enumerate(cases):
        at = np.arange(5, n, 47)                             # in every warp's part of a tile, now and then
        x[s, at, 0, :, 0] = gap * math.sqrt(d) / 16
        x[s, at, 1] = 0.0
        x[s, at, 1, :, 3] = 448.0 * size
    for s in range(n_seq):
        B.et_kv_append(c.data, c.scale, bf16(x[s].reshape(n, -1)), 0, c.table[s:s + 1], i32([0]), i32([0, n]))
    qt = bf16(q.reshape(n_seq, -1))
    out, lse, status = run_attention(B, qt, heads, c, [n] * n_seq)
    assert status == 0
    values, qs = c.values(), f64(qt).reshape(n_seq, heads, d)
    for s, case in enumerate(cases):
        k, v = c.rows(s, 0, n, values)
        want, wl, mass, size = attention_reference(qs[s], k, v)
        drift = d * 2.0 ** -23 * size + 2.0 ** -20
        top = np.exp((np.einsum("hd,hnd->hn", qs[s], np.repeat(k, heads // kvh, 0)) / math.sqrt(d)).max(-1) - wl)   # largest probability
        below = 2.0 ** -32 * top[:, None] * np.repeat(np.abs(v).sum(1), heads // kvh, 0)
        tol = BF16 * np.abs(want) + (2.0 ** -11 + 2 * drift + n / 64 * 2.0 ** -23)[:, None] * mass + below + 1e-30
        off = np.abs(f64(out[s]).reshape(heads, d) - want) / tol
        assert (off <= 1).all(), f"size and gap {case}: off by {off.max():.3g} of the tolerance in dimension {off.max(0).argmax()}"
        assert (np.abs(f64(lse[s]) - wl) <= drift + n / 64 * 2.0 ** -23 + 2.0 ** -22 * np.abs(wl)).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_ignores_what_stands_behind_the_length(B, e4m3):
    """NaN, infinities and the largest numbers behind a sequence's end (in its last page and on the pages after it), and NaN on
    the pages that no table names, change nothing, bit by bit."""
    import torch
    rng = np.random.default_rng(3)
    lens, heads, kvh, page, d = [1, 17, 64, 130, 0, 79], 14, 2, 32, 128
    c = Cache(rng, len(lens), 6, kvh, page, d, e4m3)
    q = bf16(rng.standard_normal((len(lens), heads * d)))
    a = run_attention(B, q, heads, c, lens)
    used = torch.zeros((c.n_pages, page), dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens):
        for p in range(n):
            used[c.table[s, p // page].item(), p % page] = True
    stale = ~used[:, None, None, :].expand(c.n_pages, 2, kvh, page)
    for fill in (0x7f, 0xff) if e4m3 else (math.nan, math.inf, -3.0e38):
        if e4m3:
            c.data.view(torch.uint8)[stale] = fill
            c.scale[stale] = 254
        else:
            c.data[stale] = fill
        b = run_attention(B, q, heads, c, lens)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and b[2] == 0


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_nan_in_a_live_place_is_seen(B, e4m3):
    import torch
    rng = np.random.default_rng(4)
    lens, heads, kvh, page, d = [100, 100], 4, 2, 16, 64
    c = Cache(rng, 2, 7, kvh, page, d, e4m3)
    c.data[c.table[1, 2].item(), 0, 1, 5, 3] = math.nan                        # a key of the second head of sequence 1
    out, lse, _ = run_attention(B, bf16(rng.standard_normal((2, heads * d))), heads, c, lens)
    out = out.view(2, kvh, 2, d)
    assert torch.isfinite(out[0].float()).all() and torch.isfinite(out[1, 0].float()).all()
    assert torch.isnan(out[1, 1].float()).all() and torch.isnan(lse[1, 2:]).all()


@pytest.mark.parametrize("heads,lens", [(6, [90, 150, 33]), (24, [90, 150, 33]), (6, [9000, 150, 4001]), (24, [9000, 150, 4001])])
def test_attention_infinite_values(B, heads, lens):
    """An infinity among a column's live values is that column's result, both signs or a NaN make it NaN, wherever they stand: at the
    largest weight, at ordinary ones, at one of 2^-80; the other columns keep their bits."""
    import torch
    kvh, page, d = 2, 32, 128
    rng = np.random.default_rng(heads + lens[0])
    c = Cache(rng, len(lens), (max(lens) + page - 1) // page, kvh, page, d, False)
    table = c.table.cpu().numpy()
    q = rng.standard_normal((len(lens), heads, d))
    q[:, :, 0] = 8.0
    c.data[:, 0, :, :, 0] = 0.0
    c.data[table[0, 40 // page], 0, :, 40 % page, 0] = 64.0                     # sequence 0: position 40 has nearly all of the weight
    for p in (50, 51):
        c.data[table[0, p // page], 0, :, p % page, 0] = -14.0                  # and these about 2^-80 of it
    qt = bf16(q.reshape(len(lens), -1))
    a = run_attention(B, qt, heads, c, lens)
    inf, nan = math.inf, math.nan
    marks = [(0, 3, 40, inf), (0, 4, 7, inf), (0, 5, 50, -inf), (0, 6, 51, inf), (0, 7, 40, -inf), (0, 8, 12, inf), (0, 8, 13, -inf), (0, 9, 40, nan),
             (0, 10, lens[0] - 1, -inf), (1, 3, 0, inf), (1, 4, 149, -inf), (1, 5, 64, inf), (1, 5, 65, inf), (1, 6, 100, nan), (2, 127, 32, -inf)]
    want = {}
    for s, dim, pos, x in marks:
        assert pos < lens[s]
        c.data[table[s, pos // page], 1, :, pos % page, dim] = x
        want[s, dim] = want.get((s, dim), 0.0) + x
    b = run_attention(B, qt, heads, c, lens)
    got, plain = b[0].view(len(lens), heads, d), a[0].view(len(lens), heads, d)
    for (s, dim), x in want.items():
        assert torch.isnan(got[s, :, dim].float()).all() if x != x else (got[s, :, dim] == x).all(), (s, dim, x, got[s, :, dim].tolist())
    keep = torch.ones_like(got, dtype=torch.bool)
    for s, dim in want:
        keep[s, :, dim] = False
    assert torch.equal(got[keep], plain[keep]) and torch.equal(a[1], b[1]) and torch.isfinite(plain.float()).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_attention_over_bad_pages_and_long_lengths(B, e4m3):
    """Pages that are not in the cache count as absent, lengths behind the table as the table's end; both are reported."""
    rng = np.random.default_rng(6)
    heads, kvh, page, d, max_pages = 7, 1, 16, 128, 9
    c = Cache(rng, 3, max_pages, kvh, page, d, e4m3)
    q = bf16(rng.standard_normal((3, heads * d)))
    table, lens = c.table.clone(), [140, 100, 60]
    table[0, 3], table[0, 8], table[2, 0] = c.n_pages, -7, 2 ** 31 - 1
    alive = [np.ones(144, dtype=bool) for _ in lens]
    alive[0][48:64] = alive[0][128:] = alive[2][:16] = False
    out, lse, status = run_attention(B, q, heads, c, lens, table)
    assert status == B.ET_PAGED_BAD_PAGE
    good = f64(q).reshape(3, heads, d)
    check_attention(out, lse, good, lens, c, heads, alive)
    out, lse, status = run_attention(B, q, heads, c, [2 ** 31 - 1, 145, 60])
    assert status == B.ET_PAGED_CAPACITY
    check_attention(out, lse, good, [144, 144, 60], c, heads)
    table[1] = -1                                                               # every page of a sequence is bad: an empty row
    out, lse, status = run_attention(B, q, heads, c, lens, table)
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all() and status == B.ET_PAGED_BAD_PAGE


def test_attention_reads_queries_from_packed_rows(B):
    import torch
    rng = np.random.default_rng(8)
    lens, heads, kvh, page, d = [90, 33, 7], 6, 2, 16, 64
    c = Cache(rng, 3, 6, kvh, page, d, False)
    packed = bf16(rng.standard_normal((3, (heads + 2 * kvh) * d)))
    a = run_attention(B, packed[:, :heads * d], heads, c, lens)
    b = run_attention(B, packed[:, :heads * d].contiguous(), heads, c, lens)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out = B.et_attention_paged(packed, heads, c.data, c.scale, c.table, i32(lens))          # no lse, no status, own workspace
    assert torch.equal(out, a[0])


def test_attention_is_reproducible_and_independent_of_its_workspace(B):
    import torch
    rng = np.random.default_rng(12)
    lens, heads, kvh, page, d = [3001, 17, 900, 0, 2500], 28, 4, 64, 128
    c = Cache(rng, 5, 47, kvh, page, d, True)
    q = bf16(rng.standard_normal((5, heads * d)))
    a = run_attention(B, q, heads, c, lens)
    for fill in (0, 255, 127):
        ws = torch.full((B.ET_PAGED_WORKSPACE,), fill, dtype=torch.uint8, device="cuda")
        b = run_attention(B, q, heads, c, lens, workspace=ws)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_in_a_graph_follows_its_inputs(B):
    """Captured once, replayed with other lengths, tables and queries; beside it, eager calls on another stream with a workspace
    of their own."""
    import torch
    rng = np.random.default_rng(13)
    n, heads, kvh, page, d = 4, 14, 2, 32, 128
    c = Cache(rng, n, 60, kvh, page, d, False)
    q, lens = bf16(rng.standard_normal((n, heads * d))), i32([5, 5, 5, 5])
    out, lse = torch.empty((n, heads * d), dtype=torch.bfloat16, device="cuda"), torch.empty((n, heads), dtype=torch.float32, device="cuda")
    ws = torch.empty(B.ET_PAGED_WORKSPACE, dtype=torch.uint8, device="cuda")
    B.et_attention_paged(q, heads, c.data, None, c.table, lens, out=out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.et_attention_paged(q, heads, c.data, None, c.table, lens, out=out, lse=lse, workspace=ws)
    other, results = torch.cuda.Stream(), []
    values = c.values()
    for now in ([1900, 0, 64, 3], [1, 1920, 700, 1700]):
        lens.copy_(i32(now))
        q.copy_(bf16(rng.standard_normal((n, heads * d))))
        torch.cuda.synchronize()
        for _ in range(3):
            graph.replay()
            with torch.cuda.stream(other):
                results.append(B.et_attention_paged(q, heads, c.data, None, c.table, lens, stream=other))
        torch.cuda.synchronize()
        check_attention(out, lse, f64(q).reshape(n, heads, d), now, c, heads, values=values)
        assert all(torch.equal(r, out) for r in results)
        results.clear()


@pytest.mark.parametrize("e4m3", [False, True])
def test_cache_beyond_32_bit_offsets(B, e4m3):
    """A cache of more than 2^32 bytes: pages at its end are written, read and attended to."""
    import torch
    kvh, page, d, heads, n = 8, 128, 128, 16, 300
    row = 2 * kvh * page * d * (1 if e4m3 else 2)
    n_pages = (1 << 32) // row + 40
    data = torch.zeros((n_pages, 2, kvh, page, d), dtype=torch.uint8 if e4m3 else torch.bfloat16, device="cuda")
    data = data.view(torch.float8_e4m3fn) if e4m3 else data
    scale = torch.zeros((n_pages, 2, kvh, page), dtype=torch.uint8, device="cuda") if e4m3 else None
    rng = np.random.default_rng(21)
    table = i32([[n_pages - 1, n_pages - 20, 1], [2, n_pages - 3, n_pages - 2]])
    x = bf16(rng.standard_normal((2 * n, 2 * kvh * d)))
    B.et_kv_append(data, scale, x, 0, table, i32([0, 0]), i32([0, n, 2 * n]))
    back = B.et_kv_read(data, scale, table, i32([0, 0]), 2 * n, i32([0, n, 2 * n]))
    if e4m3:
        vals, e = e4m3_rows(f64(x).reshape(2 * n, 2, kvh, d))
        want = (vals * np.ldexp(1.0, e)[..., None]).reshape(2 * n, -1)
    else:
        want = f64(x)
    assert np.array_equal(f64(back), want)
    small = Cache(rng, 2, 3, kvh, page, d, e4m3)                                # the same rows in a small cache give the same bits
    B.et_kv_append(small.data, small.scale, x, 0, small.table, i32([0, 0]), i32([0, n, 2 * n]))
    q = bf16(rng.standard_normal((2, heads * d)))
    a = B.et_attention_paged(q, heads, data, scale, table, i32([n, n - 9]))
    b = B.et_attention_paged(q, heads, small.data, small.scale, small.table, i32([n, n - 9]))
    assert torch.equal(a, b)


def test_attention_of_sequences_that_share_pages(B):
    """Two sequences may name the same pages (a common beginning): both read them."""
    import torch
    rng = np.random.default_rng(22)
    lens, heads, kvh, page, d = [150, 150, 96], 12, 4, 32, 128
    c = Cache(rng, 3, 5, kvh, page, d, True)
    c.table[1] = c.table[0]
    c.table[2, :3] = c.table[0, :3]
    q = bf16(rng.standard_normal((3, heads * d)))
    q[1] = q[0]
    out, lse, status = run_attention(B, q, heads, c, lens)
    assert status == 0 and torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1])
    check_attention(out, lse, f64(q).reshape(3, heads, d), lens, c, heads)


def test_calls_on_a_stream_of_their_own(B):
    """The stream argument: what the calls create belongs to that stream, and calls on two streams at once do not disturb one
    another (each with the workspace and the outputs that the calls create)."""
    import torch
    rng = np.random.default_rng(41)
    lens, heads, kvh, page, d = [700, 3, 1500], 14, 2, 32, 128
    c = Cache(rng, 3, 50, kvh, page, d, False)
    q = bf16(rng.standard_normal((3, heads * d)))
    want = B.et_attention_paged(q, heads, c.data, None, c.table, i32(lens))
    rows = B.et_kv_read(c.data, None, c.table, i32([0, 0, 0]), 100, i32([0, 50, 53, 60]))
    a, w = bf16(rng.standard_normal((20, 4096))), bf16(rng.standard_normal((5120, 4096)))
    y = B.et_linear_rows(a, w)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        s = streams[i % 2]
        got.append((B.et_attention_paged(q, heads, c.data, None, c.table, i32(lens), stream=s),
                    B.et_kv_read(c.data, None, c.table, i32([0, 0, 0]), 100, i32([0, 50, 53, 60]), stream=s), B.et_linear_rows(a, w, stream=s)))
        torch.cuda.synchronize() if i == 9 else None
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) and torch.equal(r, rows) and torch.equal(z, y) for x, r, z in got)
    assert (rows[60:] == 0).all()


def test_calls_report_their_own_errors_only(B):
    """A model that does not fit on the card is refused (an allocation fails); the decode calls after it run and say so."""
    import torch
    rng = np.random.default_rng(42)
    heads, kvh, page, d = 4, 2, 16, 64
    c = Cache(rng, 2, 2, kvh, page, d, False)
    qkv, lens, new = bf16(rng.standard_normal((2, (heads + 2 * kvh) * d))), i32([3, 17]), i32([0, 0])
    a, w = bf16(rng.standard_normal((2, 64))), bf16(rng.standard_normal((64, 64)))

    def step():
        q = B.et_kv_append(c.data, None, qkv, heads, c.table, lens, theta=1e4, new_len=new)
        return q, B.et_kv_read(c.data, None, c.table, lens, 2), B.et_attention_paged(q, heads, c.data, None, c.table, new), B.et_linear_rows(a, w)

    want = step()
    H, V = 4096, 1 << 27                                     # staging one matrix would take 2^41 bytes
    cfg = B.et_llm_config(1152, H, 1, 32, 8, 128, 4096, V, 1e-6, 1e4, 1, 256, 0)
    qkv_dim, m = (32 + 16) * 128, 4096
    count = V * H + 1152 * H + H + H * H + H + (H + H * qkv_dim + qkv_dim + 4096 * H + H + H * 2 * m + m * H) + H + H * V
    data = (B.C.c_float * 4)()                               # nothing of it is read
    for again in range(2):
        handle = B.C.c_void_p()
        weights = B.et_llm_weights(B.C.cast(data, B.C.c_void_p), count, 0)
        assert B.lib().et_llm_create(B.C.byref(cfg), B.C.byref(weights), B.C.byref(handle)) == 4       # ET_ERR_OOM
        got = step()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    x, y = torch.ones((1, 64), device="cuda"), torch.empty((1, 64), dtype=torch.bfloat16, device="cuda")
    B.lib().et_rmsnorm(x.data_ptr(), x.data_ptr(), 1e-6, y.data_ptr(), 1, 64, torch.cuda.current_stream().cuda_stream)    # takes the error with it


# ---- dense layer for few rows -----------------------------------------------------------------------------------------

def linear_reference(a, w, bias, epilogue, gelu_tanh, c0):
    """(result, what it may be off) in 64 bits."""
    y = a @ w.T + bias
    # K products summed in fp32, at least 16 at a time inside an instruction
    err = (a.shape[1] / 16 + 32) * 2.0 ** -22 * (np.abs(a) @ np.abs(w).T + np.abs(bias))
    if epilogue == 2:
        return c0 + y, err + 2.0 ** -23 * (np.abs(c0) + np.abs(y))
    if epilogue == 1:
        if gelu_tanh:
            z = 0.5 * y * (1 + np.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
        else:
            z = 0.5 * y * (1 + np.vectorize(math.erf)(y / math.sqrt(2)))
        # the slope is at most 1.13; 1 + tanh and 1 + erf are off by 2^-23 where they nearly vanish
        return z, 1.13 * err + 2.0 ** -21 * np.abs(y) + BF16 * np.abs(z)
    if epilogue == 4:
        t, e = y.reshape(y.shape[0], -1, 2, 32), err.reshape(y.shape[0], -1, 2, 32)
        g, u = t[:, :, 0].reshape(y.shape[0], -1), t[:, :, 1].reshape(y.shape[0], -1)
        eg, eu = e[:, :, 0].reshape(g.shape), e[:, :, 1].reshape(g.shape)
        s = g / (1 + np.exp(-g))
        return s * u, 1.1 * eg * (np.abs(u) + eu) + np.abs(s) * eu + (BF16 + 2.0 ** -20) * np.abs(s * u)
    return y, err + BF16 * np.abs(y)


LINEARS = [(1, 64, 64), (1, 3584, 4608), (3, 8, 5), (7, 520, 1), (8, 1000, 333), (9, 18944, 256), (16, 72, 3584), (17, 1152, 512),
           (25, 2048, 1000), (32, 3584, 768), (31, 40, 2049), (5, 18944, 3584)]


@pytest.mark.parametrize("epilogue,gelu_tanh,with_bias", [(0, 1, True), (0, 1, False), (1, 1, True), (1, 0, True), (2, 1, True), (2, 1, False), (4, 1, True), (4, 1, False)])
@pytest.mark.parametrize("M,K,N", LINEARS)
def test_linear_rows(B, M, K, N, epilogue, gelu_tanh, with_bias):
    import torch
    if epilogue == 4:
        N = max(256, N // 256 * 256)
    rng = np.random.default_rng(M * 1000 + K + N + epilogue)
    a, w = bf16(rng.standard_normal((M, K))), bf16(rng.standard_normal((N, K)) / math.sqrt(K))
    bias = rng.standard_normal(N).astype(np.float32) if with_bias else None
    outs = N // 2 if epilogue == 4 else N
    c0 = rng.standard_normal((M, outs)).astype(np.float32)
    guard = torch.full((M * outs + 64,), 3.0, dtype=torch.float32 if epilogue == 2 else torch.bfloat16, device="cuda")
    c = guard[:M * outs].view(M, outs)
    if epilogue == 2:
        c.copy_(torch.from_numpy(c0))
    B.et_linear_rows(a, w, None if bias is None else torch.from_numpy(bias).cuda(), epilogue, gelu_tanh, c=c)
    want, tol = linear_reference(f64(a), f64(w), np.zeros(N) if bias is None else bias.astype(np.float64), epilogue, gelu_tanh, c0.astype(np.float64))
    err = np.abs(f64(c) - want)
    assert (err <= tol + 1e-30).all(), f"{(err / tol).max():.3g} of the tolerance"
    assert (guard[M * outs:] == 3.0).all()


@pytest.mark.parametrize("M,K,N,chain", [(5, 18944, 3584, 4), (32, 18944, 3584, 4), (13, 18944, 1100, 4), (1, 3584, 37888, 4), (1, 3584, 4608, 16),
                                         (8, 18944, 256, 20), (1, 65536, 8, 64)])
def test_linear_rows_long_sums(B, M, K, N, chain):
    """Sums of positive products, where what the tensor core cuts off adds up: at most 2^-23 of a partial sum for each instruction of a
    chain.  With many weights a chain is one stage of four instructions; with few it is a warp's share of K, `chain` instructions long.
    Partial sums are added in fp32, whose rounding errors have no sign: in the mean over the outputs they stay below 2^-24."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(K + N + M)
    a, w = (torch.randn((n, K), device="cuda", generator=gen).abs().to(torch.bfloat16) for n in (M, N))
    c = torch.zeros((M, N), device="cuda")
    B.et_linear_rows(a, w, None, 2, c=c)
    want = a.double() @ w.double().T
    off = (c.double() - want) / want
    # worst case of the additions: one rounding for each of the K / 64 steps of a rank, and those of the ranks' and warps' sums
    assert off.abs().max().item() <= chain * 2.0 ** -23 + (K / 64 + 16) * 2.0 ** -24
    assert abs(off.mean().item()) <= chain * 2.0 ** -23 + 2.0 ** -24, off.mean().item()


@pytest.mark.parametrize("M,K,N", [(1, 1 << 20, 32), (12, 1 << 20, 64), (20, 1 << 18, 70), (31, 1 << 20, 8), (1, 1 << 24, 1), (2, 300_008, 3)])
def test_linear_rows_longest_sums(B, M, K, N):
    """Few weight rows as long as can be: chains of at most 128 instructions."""
    test_linear_rows_long_sums(B, M, K, N, 128)


@pytest.mark.parametrize("epilogue", [0, 2])
@pytest.mark.parametrize("M,K,N", [(3, 1000, 40007), (12, 136, 46001), (32, 72, 50002), (17, 1016, 12003), (32, 264, 22010)])
def test_linear_rows_in_blocks_of_fewer_rows(B, M, K, N, epilogue):
    """Blocks' rows follow from how many blocks the card holds; none of these fills whole blocks of 128."""
    test_linear_rows(B, M, K, N, epilogue, 1, True)


@pytest.mark.parametrize("M,K,N", [(2, 1024, 384), (12, 3584, 640), (30, 2048, 384)])
def test_linear_rows_from_16_byte_aligned_operands(B, M, K, N):
    """Operands that start 16 bytes behind a 32-byte border give what aligned ones give."""
    import torch
    rng = np.random.default_rng(M)
    a, w = bf16(rng.standard_normal((M, K))), bf16(rng.standard_normal((N, K)))
    x = B.et_linear_rows(a, w)
    moved = [torch.empty(z.numel() + 8, dtype=torch.bfloat16, device="cuda")[8:].view_as(z).copy_(z) for z in (a, w)]
    assert moved[0].data_ptr() % 32 == 16 and moved[1].data_ptr() % 32 == 16
    for p, q in ((moved[0], w), (a, moved[1]), moved):
        # two 16-byte loads in place of one of 32: the same operands in the same places of the same instructions
        assert torch.equal(B.et_linear_rows(p, q), x)


def test_linear_rows_rows_do_not_touch_each_other(B):
    """A NaN row stays alone, and a row gives the same bits whatever the other rows of the call hold."""
    import torch
    rng = np.random.default_rng(2)
    a, w = bf16(rng.standard_normal((13, 777 * 8))), bf16(rng.standard_normal((300, 777 * 8)))
    x = B.et_linear_rows(a, w)
    b = a.clone()
    b[5] = math.nan
    b[7:] *= 3
    y = B.et_linear_rows(b, w)
    assert torch.isnan(y[5].float()).all() and torch.equal(x[[0, 1, 2, 3, 4, 6]], y[[0, 1, 2, 3, 4, 6]])


def test_linear_rows_agrees_with_linear_bf16(B):
    """The same arguments and weight order as the wide dense layer: results within the roundings of both."""
    import torch
    rng = np.random.default_rng(3)
    for epilogue, N in ((0, 640), (1, 640), (2, 640), (4, 1024)):
        a, w = bf16(rng.standard_normal((24, 512))), bf16(rng.standard_normal((N, 512)) / math.sqrt(512))
        bias = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda()
        c = torch.zeros((24, 640), dtype=torch.float32, device="cuda") if epilogue == 2 else None
        x, _ = B.et_linear_bf16(a, w, bias, epilogue, c=None if c is None else c.clone())
        y = B.et_linear_rows(a, w, bias, epilogue, c=c)
        d = (x.float() - y.float()).abs()
        # the wide layer's GELU uses the hardware tanh (2^-11 of the argument)
        assert (d <= 2 * BF16 * x.float().abs() + (2.0 ** -10 if epilogue == 1 else 2.0 ** -16) * (1 + x.float().abs())).all()


# ---- together ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("e4m3", [False, True])
def test_decode_step_follows_the_prefill(B, e4m3):
    """A prompt is prefilled, its cache moved into pages, and the next token decoded layer by layer with the operators: logits
    agree with the prefill of the longer sequence.  Both paths keep activations in bf16 but round at different places; the bound
    is the framework's for whole bf16 models, 2e-2 of the largest logit; an e4m3 cache adds the spread of its own rounding,
    2^-4 / sqrt(3) of each key and value, averaged over many positions and layers: 0.1 of the largest logit."""
    import torch
    from synthetic.llm import LLM_SMALL, llm_views, make_llm_weights, make_prompt, make_visual_tokens
    sh = LLM_SMALL
    blob = make_llm_weights(sh, 4)
    n = 150
    ids, _ = make_prompt(sh, n + 1, 0, 4)
    vis = torch.from_numpy(make_visual_tokens(sh, 40, 4)).cuda()
    llm = B.LanguageModel(sh, blob, max_tokens=256, keep_kv_cache=True)
    want = llm.prefill(ids[:100], vis, ids[100:]).logits
    pre = llm.prefill(ids[:100], vis, ids[100:n], want_kv=True)
    total = pre.n_tokens
    W = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in llm_views(sh, blob).items()}
    def t16(x):
        return x.to(torch.bfloat16).T.contiguous()
    page, kvh, d = 32, sh.kv_heads, sh.head_dim
    rng = np.random.default_rng(1)
    x = W["embed"].to(torch.bfloat16)[int(ids[n])].float().view(1, -1).clone()
    table = i32(rng.permutation(16)[:8].reshape(1, 8))
    lens, new, status = i32([total]), i32([0]), i32([0])
    for i in range(sh.num_layers):
        w = {k[len(f"l{i}."):]: v for k, v in W.items() if k.startswith(f"l{i}.")}
        cache = torch.zeros((16, 2, kvh, page, d), dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16, device="cuda")
        scale = torch.zeros((16, 2, kvh, page), dtype=torch.uint8, device="cuda") if e4m3 else None
        B.et_kv_append(cache, scale, pre.kv_cache[i], 0, table, i32([0]), i32([0, total]), status=status)
        if not e4m3:
            assert torch.equal(B.et_kv_read(cache, scale, table, i32([0]), total, i32([0, total])), pre.kv_cache[i])
        qkv = B.et_linear_rows(B.et_rmsnorm(x, w["rms1_g"], sh.rms_eps), t16(w["wqkv"]), w["bqkv"])
        q = B.et_kv_append(cache, scale, qkv, sh.heads, table, lens, theta=sh.rope_theta, new_len=new, status=status)
        att = B.et_attention_paged(q, sh.heads, cache, scale, table, new, status=status)
        B.et_linear_rows(att, t16(w["wo"]), None, 2, c=x)
        h = B.et_rmsnorm(x, w["rms2_g"], sh.rms_eps)
        m = sh.mlp_dim
        gate, up = t16(w["wgu"])[:m], t16(w["wgu"])[m:]
        pad = -m % 128                                  # whole tiles of 256 weight rows; the padding's outputs are dropped
        gate, up = (torch.cat([z, torch.zeros((pad, z.shape[1]), dtype=z.dtype, device="cuda")]) for z in (gate, up))
        tiled = torch.stack([gate.view(-1, 32, gate.shape[1]), up.view(-1, 32, up.shape[1])], 1).reshape(-1, gate.shape[1])
        act = B.et_linear_rows(h, tiled.contiguous(), None, 4)[:, :m].contiguous()
        B.et_linear_rows(act, t16(w["wd"]), None, 2, c=x)
    logits = torch.zeros((1, sh.vocab), dtype=torch.float32, device="cuda")
    B.et_linear_rows(B.et_rmsnorm(x, W["final_g"], sh.rms_eps), t16(W["lm_head"]), None, 2, c=logits)
    assert status.item() == 0 and new.item() == total + 1
    off = (logits[0] - want).abs().max().item() / want.abs().max().item()
    assert off <= (0.1 if e4m3 else 2e-2), off


def test_decode_operators_in_one_graph(B):
    """Three tokens decoded by one captured step (append, attention) whose lengths advance on the device, on a side stream,
    against the same steps run one by one."""
    import torch
    rng = np.random.default_rng(31)
    n, heads, kvh, page, d = 3, 6, 2, 16, 64
    lens0 = [14, 0, 33]

    def fresh():
        return Cache(np.random.default_rng(32), n, 4, kvh, page, d, True)

    qkvs = [bf16(rng.standard_normal((n, (heads + 2 * kvh) * d))) for _ in range(3)]
    a, want, lens = fresh(), [], i32(lens0)
    for qkv in qkvs:
        new = torch.empty_like(lens)
        q = B.et_kv_append(a.data, a.scale, qkv, heads, a.table, lens, theta=1e4, new_len=new)
        want.append(B.et_attention_paged(q, heads, a.data, a.scale, a.table, new))
        lens = new
    b, stream = fresh(), torch.cuda.Stream()
    lens, new, qkv = i32(lens0), i32([0] * n), qkvs[0].clone()
    q = torch.empty((n, heads * d), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(B.ET_PAGED_WORKSPACE, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()

    def step():
        B.et_kv_append(b.data, b.scale, qkv, heads, b.table, lens, theta=1e4, q_out=q, new_len=new)
        B.et_attention_paged(q, heads, b.data, b.scale, b.table, new, out=out, workspace=ws)
        lens.copy_(new)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for x, y in zip(qkvs, want):
        qkv.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, y)
    assert torch.equal(b.bytes()[0], a.bytes()[0]) and torch.equal(b.scale, a.scale)


@pytest.mark.parametrize("e4m3", [False, True])
def test_steps_one_behind_the_other_without_waiting(B, e4m3):
    """Sixty decode steps (dense layer, append, attention, dense layer), each reading what the step before has just written --
    lengths, cache rows, activations -- enqueued without a wait, against the same steps with a wait behind every call: the
    same bits.  (The kernels are set up while the ones before them still run.)"""
    import torch
    n, heads, kvh, page, d, hidden = 5, 6, 2, 16, 64, 512
    rng = np.random.default_rng(51)
    wqkv = bf16(rng.standard_normal(((heads + 2 * kvh) * d, hidden)) / math.sqrt(hidden))
    wo = bf16(rng.standard_normal((hidden, heads * d)) / math.sqrt(heads * d))
    x0 = bf16(rng.standard_normal((n, hidden)))

    def run(wait):
        c = Cache(np.random.default_rng(52), n, 6, kvh, page, d, e4m3)
        both = i32([13, 0, 30, 5, 31] + [0] * n)                               # lengths, in turn in two halves of one line
        lens = [both[:n], both[n:]]
        qkv = torch.empty((n, (heads + 2 * kvh) * d), dtype=torch.bfloat16, device="cuda")
        q = torch.empty((n, heads * d), dtype=torch.bfloat16, device="cuda")
        att, x, ws = torch.empty_like(q), x0.clone(), torch.empty(B.ET_PAGED_WORKSPACE, dtype=torch.uint8, device="cuda")
        out = torch.empty((60, n, hidden), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        done = torch.cuda.synchronize if wait else (lambda: None)
        for i in range(60):
            B.et_linear_rows(x, wqkv, c=qkv)
            done()
            B.et_kv_append(c.data, c.scale, qkv, heads, c.table, lens[i % 2], theta=1e4, q_out=q, new_len=lens[1 - i % 2])
            done()
            B.et_attention_paged(q, heads, c.data, c.scale, c.table, lens[1 - i % 2], out=att, workspace=ws)
            done()
            x = B.et_linear_rows(att, wo, epilogue=1, c=out[i])
            done()
        torch.cuda.synchronize()
        return out, both.tolist()

    a, la = run(True)
    for _ in range(3):
        b, lb = run(False)
        assert torch.equal(a, b) and la == lb
    assert la[:n] == [73, 60, 90, 65, 91]
