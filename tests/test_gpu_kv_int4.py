"""The cache of 4 bits (ET_KV_INT4): rows going in and coming back, and attention over it, against plain implementations in 64 bits.

A block of 32 values has the scale s = the smallest bf16 not below max|x| / 7 and codes 8 + x / s, rounded to nearest with ties to
even.  Codes and scales have to be the definition's exactly, turned keys' among them where no value is nearer to a border than the
64-bit angle tells.  Tolerances of what is computed count roundings: half a step of bf16 is 2^-8 of the value, d products in fp32
are off by d * 2^-23 of the sum of their magnitudes (the tensor cores may truncate), a weight of 16 bits by 2^-16."""
import math

import numpy as np
import pytest

from tests.test_gpu_decode import attention_reference, bf16, f64, i32, rotate

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8


@pytest.fixture(scope="module")
def B():
    import torch
    assert torch.cuda.is_available()
    from paper_2605_30010_b200 import binding
    return binding


def next_bf16_up(x):
    """The smallest bf16 that is not below x >= 0 (64 bits)."""
    m, e = np.frexp(x)
    e = np.maximum(e, -125)                                   # subnormals: steps of 2^-133
    return np.where(x > 0, np.ldexp(np.ceil(np.ldexp(x, 8 - e)), e - 8), 0.0)


def quantise(x):
    """x [..., d] in 64 bits -> (whole numbers -7 .. 7, scales [..., d / 32]; NaN and zeros for a block that is not finite)."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    fine = (np.abs(y) <= np.finfo(np.float32).max).all(-1)
    y = np.where(fine[..., None], y, 0.0)
    s = next_bf16_up(np.abs(y).max(-1) / 7)
    n = np.where(s[..., None] > 0, np.rint(y / np.where(s > 0, s, 1.0)[..., None]), 0.0)
    return n.reshape(x.shape), np.where(fine, s, np.nan)


class Cache4:
    """A paged cache of 4 bits with every byte of it set to something, and a table of distinct pages for n_seq sequences."""

    def __init__(self, rng, n_seq, max_pages, kv_heads, page, d, spare=3):
        import torch
        self.page, self.kv_heads, self.d = page, kv_heads, d
        self.n_pages = n_seq * max_pages + spare
        shape = (self.n_pages, 2, kv_heads, page, d)
        x = rng.standard_normal(shape) * np.exp2(rng.integers(-3, 4, shape[:-1]))[..., None]
        self.put(*quantise(x))
        self.table = i32(rng.permutation(self.n_pages)[:n_seq * max_pages].reshape(n_seq, max_pages))

    def put(self, n, s):
        import torch
        c = (n + 8).astype(np.uint8)
        self.data = torch.from_numpy(np.ascontiguousarray(c[..., ::2] | (c[..., 1::2] << 4))).cuda()
        self.scale = bf16(s)

    def codes(self):
        b = self.data.cpu().numpy().astype(int)
        return np.stack([b & 15, b >> 4], -1).reshape(*b.shape[:-1], -1) - 8

    def values(self):
        return self.codes() * np.repeat(f64(self.scale), 32, -1)

    def rows(self, s, first, n, values=None):
        """[2][kv_heads][n][d] of sequence s."""
        values = self.values() if values is None else values
        pos = np.arange(first, first + n)
        pages = self.table.cpu().numpy()[s][pos // self.page]
        return values[pages, :, :, pos % self.page].transpose(1, 2, 0, 3)


STORES = [
    # rows of each sequence, start of each, heads, kv_heads, page, d, theta
    ([1], [0], 4, 2, 16, 64, 1e4),
    ([1], [7675], 28, 4, 64, 128, 1e6),
    ([1, 1, 1, 1, 1], [0, 15, 16, 31, 100], 7, 1, 16, 128, 1e6),
    ([37, 1, 0, 64, 129], [0, 63, 5, 1, 127], 6, 2, 32, 128, 5e5),
    ([200], [3], 0, 4, 128, 128, 0.0),
    ([5, 300, 17], [1000, 0, 2], 0, 3, 16, 64, 0.0),
    ([2, 3], [10, 20], 5, 5, 64, 64, 0.0),
    ([700, 411], [9_000, 4], 2, 4, 128, 128, 1e4),
    ([(7 * i) % 5 for i in range(150)], [(37 * i) % 91 for i in range(150)], 2, 2, 16, 64, 1e4),
]


@pytest.mark.parametrize("case", range(len(STORES)))
def test_rows_go_in_and_come_back(B, case):
    import torch
    counts, starts, heads, kvh, page, d, theta = STORES[case]
    rng = np.random.default_rng(case)
    n_seq, rows = len(counts), sum(counts)
    c = Cache4(rng, n_seq, max((s + n + page - 1) // page for s, n in zip(starts, counts)) + 1, kvh, page, d)
    data0, scale0 = c.data.clone(), c.scale.clone()
    pad = 0 if counts == [1] * n_seq else 3                   # rows behind the last sequence
    x = rng.standard_normal((rows + pad, (heads + 2 * kvh) * d)) * np.exp2(rng.integers(-6, 7, (rows + pad, 1)))
    wide = torch.full((rows + pad, x.shape[1] + 16), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :x.shape[1]] = bf16(x)
    qkv = wide[:, :x.shape[1]]
    x = f64(qkv).reshape(rows + pad, heads + 2 * kvh, d)
    offsets = i32(np.concatenate([[0], np.cumsum(counts)])) if pad else None
    status, new_len = i32([0]), i32([-9] * n_seq)
    q_out = torch.full((rows + pad, heads * d), 7.0, dtype=torch.bfloat16, device="cuda") if theta and heads else None
    B.et_kv_append(c.data, c.scale, qkv, heads, c.table, i32(starts), offsets, theta, q_out, new_len, status)
    torch.cuda.synchronize()
    assert status.item() == 0 and new_len.tolist() == [s + n for s, n in zip(starts, counts)]
    pos = np.concatenate([np.arange(s, s + n) for s, n in zip(starts, counts)])
    seq = np.repeat(np.arange(n_seq), counts)
    k, v, q = x[:rows, heads:heads + kvh], x[:rows, heads + kvh:], x[:rows, :heads]
    if theta:
        slack = 2.0 ** -20 * (np.abs(q) + np.abs(np.roll(q, d // 2, -1)))
        k, q = rotate(k, pos, theta), rotate(q, pos, theta)
        if heads:
            assert (np.abs(f64(q_out[:rows]).reshape(q.shape) - q) <= BF16 * np.abs(q) + slack).all() and (q_out[rows:] == 7.0).all()
    n, s = quantise(np.stack([k, v], 1))
    places = c.table.cpu().numpy()[seq, pos // page], pos % page
    got_n, got_s = c.codes()[places[0], :, :, places[1]], f64(c.scale)[places[0], :, :, places[1]]
    # the reference's own angle, a product in 64 bits, is off by 2^-52 of up to 10^6: two values in 10^9 may lie that near to a border
    sure = slice(1, 2) if theta else slice(0, 2)
    assert np.array_equal(got_s[:, sure], s[:, sure]) and np.array_equal(got_n[:, sure], n[:, sure])
    assert (got_s != s).sum() + (got_n != n).sum() <= (n.size * 1e-7 > 1)
    keep = torch.ones((c.n_pages, page), dtype=torch.bool, device="cuda")
    keep[torch.from_numpy(places[0]).cuda().long(), torch.from_numpy(places[1]).cuda().long()] = False
    keep = keep[:, None, None].expand(c.n_pages, 2, kvh, page)
    assert torch.equal(data0[keep], c.data[keep]) and torch.equal(scale0.view(torch.int16)[keep], c.scale.view(torch.int16)[keep])
    out = torch.full((rows + pad, 2 * kvh * d + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    B.et_kv_read(c.data, c.scale, c.table, i32(starts), rows + pad, offsets, out[:, :2 * kvh * d], status)
    want = torch.from_numpy(got_n * np.repeat(got_s, 32, -1)).to(torch.bfloat16).reshape(rows, -1)
    assert torch.equal(out[:rows, :2 * kvh * d].cpu(), want)
    assert (out[rows:] == 5.0).all() and (out[:, 2 * kvh * d:] == 5.0).all() and status.item() == 0


@pytest.mark.parametrize("d,theta,start", [(128, 1e6, 0), (128, 1e4, 900_000), (64, 5e5, 2 ** 30 - 4001), (64, 1e4, 77_777)])
def test_codes_of_turned_keys(B, d, theta, start):
    """Codes and scales are those of keys turned in extended precision; a key that is nearer to a border between two codes than the
    frequencies' 2^-56 of a turn times the position, or 2^-50, leaves may lie on either side."""
    import torch
    rng = np.random.default_rng(start % 1000 + d)
    kvh, page, n = 2, 128, 4000
    first, last = start // page, (start + n - 1) // page
    table = torch.full((1, last + 1), -1, dtype=torch.int32, device="cuda")
    table[0, first:] = i32(rng.permutation(last + 1 - first))
    data = torch.zeros((last + 1 - first, 2, kvh, page, d // 2), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((last + 1 - first, 2, kvh, page, d // 32), dtype=torch.bfloat16, device="cuda")
    x = bf16(rng.standard_normal((n, 2 * kvh * d)) * np.exp2(rng.integers(-6, 7, (n, 1))))
    B.et_kv_append(data, scale, torch.cat([x[:, :d], x], 1), 1, table, i32([start]), i32([0, n]), theta)
    half = d // 2
    ang = np.arange(start, start + n).astype(np.longdouble)[:, None, None] * np.longdouble(theta) ** (-np.arange(half).astype(np.longdouble) / half)
    c, s = np.cos(ang), np.sin(ang)
    k = f64(x).reshape(n, 2, kvh, d)[:, 0].astype(np.longdouble)
    k = np.concatenate([k[..., :half] * c - k[..., half:] * s, k[..., half:] * c + k[..., :half] * s], -1)
    pos = np.arange(start, start + n)
    places = table.cpu().numpy()[0][pos // page], pos % page
    b = data.cpu().numpy()[places[0], 0, :, places[1]].astype(int)
    codes, scales = np.stack([b & 15, b >> 4], -1).reshape(n, kvh, d) - 8, f64(scale)[places[0], 0, :, places[1]]
    want, size = quantise(k.astype(np.float64))
    slack = (2.0 ** -50 + start * 2.0 ** -54) * np.abs(k).reshape(n, kvh, -1, 32).max(-1)
    assert (np.abs(scales - size) <= np.where(scales == size, 0, 2 * slack + 2.0 ** -7 * size * (np.abs(7 * np.minimum(scales, size) - np.abs(k).reshape(n, kvh, -1, 32).max(-1)) <= 7 * slack))).all()
    y = np.abs(k.astype(np.float64) - codes * np.repeat(scales, 32, -1))
    assert (y <= np.repeat(scales / 2 + 2 * slack, 32, -1)).all()
    assert (codes != want).sum() <= 2 + start * 2.0 ** -53 * 100 * codes.size


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rotated", [False, True])
def test_conversion_edges(B, d, rotated):
    """Ties, borders, blocks of zeros, the ends of bf16, values that are not finite; turned at position 0, where a key is itself."""
    import torch
    blocks = []
    for top in (7.0, 1.0, 3.0, 447.0, 2.0 ** -133, 3 * 2.0 ** -133, 2.0 ** -130, 2.0 ** -126, 1.9921875 * 2.0 ** -120, 2.0 ** 127 * 1.9921875, 2.0 ** 120, 0.0):
        s = float(next_bf16_up(np.float64(top / 7)))
        blocks.append([top] + [s * (i / 2 - 7) for i in range(29)] + [0.0, -0.0])    # every level and every border
        blocks.append([-top] + [top * (i + 1) / 32 for i in range(31)])
    for odd in (math.nan, math.inf, -math.inf):
        blocks.append([1.0] * 31 + [odd])
        blocks.append([odd] + [0.0] * 31)
    blocks.append([0.0] * 31 + [-0.0])
    while len(blocks) % (d // 32):
        blocks.append([1.0] * 32)
    x = bf16(np.clip(np.nan_to_num(np.array(blocks), nan=12345.0, posinf=1e300, neginf=-1e300), -3.3895e38, 3.3895e38))
    for i, b in enumerate(blocks):
        for j, y in enumerate(b):
            if not math.isfinite(y):
                x[i, j] = y
    rows = x.numel() // d
    x = x.view(rows, d)
    c = Cache4(np.random.default_rng(1), rows, 1, 1, 16, d)
    qkv = torch.cat([torch.ones((rows, 2 * d), dtype=torch.bfloat16, device="cuda"), x, x.flip(0)], 1)      # two heads of queries
    B.et_kv_append(c.data, c.scale, qkv if rotated else qkv[:, 2 * d:].contiguous(), 2 if rotated else 0, c.table, i32([0] * rows),
                   theta=1e4 if rotated else 0.0)
    # (position 0 turns by nothing, but a product with zero makes a NaN of an infinity's partner in the other half)
    n, s = quantise(np.stack([f64(x), f64(x.flip(0))], 1)[:, :, None])
    places = c.table.cpu().numpy()[:, 0], np.zeros(rows, int)
    got_n, got_s = c.codes()[places[0], :, :, places[1]], f64(c.scale)[places[0], :, :, places[1]]
    if rotated:
        both = np.isfinite(s).all(-1, keepdims=True)[:, :1] & np.ones_like(s[:, :1], bool)
        near = both | ~np.isfinite(got_s[:, :1])
        assert near.all()                                                          # keys: only a block next to one that is not finite differs
        n[:, :1], got_n[:, :1] = n[:, :1] * np.repeat(both, 32, -1), got_n[:, :1] * np.repeat(both, 32, -1)
        s[:, :1], got_s[:, :1] = np.where(both, s[:, :1], 0), np.where(both, got_s[:, :1], 0)
    assert np.array_equal(got_s, s, equal_nan=True) and np.array_equal(got_n, n)
    back = B.et_kv_read(c.data, c.scale, c.table, i32([0] * rows), rows)
    want = torch.from_numpy(c.values()[places[0], :, :, places[1]]).to(torch.bfloat16).view(rows, -1)
    assert torch.equal(torch.nan_to_num(back.cpu(), 3.0, 4.0, 5.0), torch.nan_to_num(want, 3.0, 4.0, 5.0))


def test_turned_keys_at_the_end_of_fp32(B):
    """Keys whose turned values lie between 2^128 (1 - 2^-21), which fp32 still holds, and 2^128: a NaN for a scale, never an infinity."""
    rng = np.random.default_rng(9)
    pos = rng.integers(0, 4096, 1 << 25)
    x, y = (np.ldexp((128 + rng.integers(0, 128, pos.size)).astype(np.float64), 120 - rng.integers(0, 2, pos.size)) for _ in range(2))
    turned = np.abs(x * np.cos(pos) - y * np.sin(pos))
    hit = np.flatnonzero((turned >= 2.0 ** 128 * (1 - 2.0 ** -21)) & (turned < 2.0 ** 128))
    below = np.flatnonzero((turned < 2.0 ** 128 * (1 - 2.0 ** -20)) & (turned > 2.0 ** 128 * (1 - 2.0 ** -17)))[:len(hit)]
    assert len(hit) >= 3
    rows = np.concatenate([hit, below])
    k = np.zeros((len(rows), 2, 64))
    k[:, 0, 0], k[:, 0, 32] = x[rows], y[rows]                # the first frequency is one radian a position
    c = Cache4(rng, len(rows), 4096 // 128, 1, 128, 64)
    B.et_kv_append(c.data, c.scale, bf16(k.reshape(len(rows), 128)), 0, c.table, i32(pos[rows]), theta=1e4)
    page = c.table.cpu().numpy()[np.arange(len(rows)), pos[rows] // 128]
    got = f64(c.scale)[page, 0, 0, pos[rows] % 128]
    _, want = quantise(rotate(k[:, :1], pos[rows], 1e4)[:, 0])
    assert np.isnan(got[:len(hit), 0]).all() and not np.isinf(got).any()
    assert np.array_equal(got[len(hit):], want[len(hit):], equal_nan=True)


def check_attention(out, lse, q, lens, c, heads, alive=None):
    d, values = c.d, c.values()
    for s, n in enumerate(lens):
        if n <= 0:
            assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
            continue
        k, v = c.rows(s, 0, n, values)
        if alive is not None:
            k, v = k[:, alive[s][:n]], v[:, alive[s][:n]]
        want, wl, mass, size = attention_reference(q[s], k, v)
        drift = d * 2.0 ** -23 * size + 2.0 ** -20
        got = f64(out[s]).reshape(heads, d)
        tol = BF16 * np.abs(want) + (2.0 ** -16 + n * 2.0 ** -23 + 2 * drift)[:, None] * mass + 1e-30
        assert (np.abs(got - want) <= tol).all(), f"sequence {s} of {n}: off by {(np.abs(got - want) / tol).max():.3g} of the tolerance"
        assert (np.abs(f64(lse[s]) - wl) <= drift + 2.0 ** -22 * np.abs(wl)).all()


def run_attention(B, q, heads, c, lens, table=None, **kw):
    import torch
    n_seq = len(lens)
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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", range(len(ATTENTIONS)))
def test_attention(B, case, d):
    lens, heads, kvh, page = ATTENTIONS[case]
    rng = np.random.default_rng(100 * case + d)
    c = Cache4(rng, len(lens), max(1, (max(lens) + page - 1) // page), kvh, page, d)
    q = bf16(rng.standard_normal((len(lens), heads * d)) * 2)
    out, lse, status = run_attention(B, q, heads, c, lens)
    assert status == 0
    check_attention(out, lse, f64(q).reshape(len(lens), heads, d), lens, c, heads)


@pytest.mark.parametrize("heads,kvh,page,d,longest", [(8, 8, 16, 64, 300), (28, 4, 32, 128, 400), (16, 1, 64, 128, 900), (6, 2, 16, 64, 1000), (2, 1, 32, 64, 90)])
def test_attention_many_short_sequences(B, heads, kvh, page, d, longest):
    rng = np.random.default_rng(heads * 7)
    n_seq = 331 if longest > 100 else 1500
    lens = [int(longest * x ** 3) for x in rng.random(n_seq)]
    lens[5:9] = [longest, 0, 1, longest]
    c = Cache4(rng, n_seq, (longest + page - 1) // page, kvh, page, d)
    q = bf16(rng.standard_normal((n_seq, heads * d)))
    out, lse, status = run_attention(B, q, heads, c, lens)
    assert status == 0
    check_attention(out, lse, f64(q).reshape(n_seq, heads, d), lens, c, heads)


@pytest.mark.parametrize("heads,kvh,page,d", [(56, 8, 64, 128), (80, 8, 16, 128), (8, 8, 32, 64), (128, 8, 128, 64)])
def test_attention_long_runs(B, heads, kvh, page, d):
    """Enough positions that every CTA goes round its ring many times; one sequence, then one next to a short one."""
    rng = np.random.default_rng(heads + d)
    for lens in ([40_000], [12_345, 70]):
        c = Cache4(rng, len(lens), (max(lens) + page - 1) // page, kvh, page, d)
        q = bf16(rng.standard_normal((len(lens), heads * d)))
        out, lse, status = run_attention(B, q, heads, c, lens)
        assert status == 0
        check_attention(out, lse, f64(q).reshape(len(lens), heads, d), lens, c, heads)


def test_attention_peaked_and_far_apart_scores(B):
    """Scores from one key that takes all to thousands apart, growing and falling along the cache; values of very different sizes, the
    large ones where nothing looks, scales at both ends of bf16."""
    rng = np.random.default_rng(77)
    n, heads, kvh, page, d = 900, 6, 2, 32, 128
    c = Cache4(rng, 2, (n + page - 1) // page, kvh, page, d)
    k = rng.standard_normal((2, kvh, n, d))
    k[0, :, :, 0] += np.linspace(-300, 300, n)
    k[1, :, :, 0] += np.linspace(300, -300, n)
    v = rng.standard_normal((2, kvh, n, d)) * np.exp2(rng.integers(-100, 1, (2, kvh, n, 1)))
    v[0, :, :450] *= 2.0 ** 100
    v[:, :, :, :32] *= 2.0 ** -20
    x = bf16(np.stack([k, v], 1).transpose(0, 3, 1, 2, 4).reshape(2 * n, -1))
    B.et_kv_append(c.data, c.scale, x, 0, c.table, i32([0, 0]), i32([0, n, 2 * n]))
    q = rng.standard_normal((2, heads, d)) * np.exp2(np.arange(heads) * 3.0 - 9)[None, :, None]
    q = bf16(q.reshape(2, -1))
    out, lse, status = run_attention(B, q, heads, c, [n, n])
    assert status == 0
    check_attention(out, lse, f64(q).reshape(2, heads, d), [n, n], c, heads)


def test_attention_ignores_what_stands_behind_the_length(B):
    """Codes of every kind and scales of NaN and infinity behind the lengths, in the same tiles and pages."""
    import torch
    rng = np.random.default_rng(5)
    lens, heads, kvh, page, d = [61, 130, 1, 64, 17], 7, 1, 32, 128
    c = Cache4(rng, len(lens), 6, kvh, page, d)
    q = bf16(rng.standard_normal((len(lens), heads * d)))
    a = run_attention(B, q, heads, c, lens)
    for s, n in enumerate(lens):
        for pos in range(n, 6 * page):
            p = c.table[s, pos // page].item()
            c.data[p, :, :, pos % page] = (7 * pos) % 256
            c.scale[p, :, :, pos % page] = [math.nan, math.inf, -math.inf, 3e38][pos % 4]
    b = run_attention(B, q, heads, c, lens)
    assert a[2] == b[2] == 0 and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_nan_in_a_live_place_is_seen(B):
    rng = np.random.default_rng(6)
    lens, heads, kvh, page, d = [70, 200], 8, 2, 16, 64
    c = Cache4(rng, 2, 13, kvh, page, d)
    q = bf16(rng.standard_normal((2, heads * d)))
    want, _, _ = run_attention(B, q, heads, c, lens)
    p, t = c.table[1, 150 // page].item(), 150 % page
    c.scale[p, 1, 1, t, 0] = math.nan                          # the first 32 dimensions of the second head's value
    out, lse, _ = run_attention(B, q, heads, c, lens)
    seen = out.view(2, heads, d).isnan()
    assert seen[1, 4:, :32].all() and seen.sum().item() == 4 * 32 and not lse.isnan().any()
    assert (out.view(2, heads, d)[~seen] == want.view(2, heads, d)[~seen]).all()
    c.scale[p, 0, 1, t, 1] = math.nan
    out, lse, _ = run_attention(B, q, heads, c, lens)
    assert lse.isnan()[1, 4:].all() and lse.isnan().sum().item() == 4 and out.view(2, heads, d)[1, 4:].isnan().all()


def test_attention_over_bad_pages_and_long_lengths(B):
    rng = np.random.default_rng(8)
    heads, kvh, page, d = 6, 2, 16, 64
    c = Cache4(rng, 3, 5, kvh, page, d)
    q = bf16(rng.standard_normal((3, heads * d)))
    table = c.table.clone()
    table[0, 1], table[0, 3], table[1, 0] = -1, c.n_pages, 2 ** 31 - 1
    lens = [75, 16, 5 * page + 3]
    out, lse, status = run_attention(B, q, heads, c, lens, table)
    assert status == B.ET_PAGED_BAD_PAGE
    pos = np.arange(5 * page)
    alive = [(pos // page != 1) & (pos // page != 3), pos < 0, pos >= 0]
    check_attention(out[::2], lse[::2], f64(q).reshape(3, heads, d)[::2], [75, 80], Rows(c, [0, 2]), heads, alive=alive[::2])
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    _, _, status = run_attention(B, q, heads, c, lens)
    assert status == B.ET_PAGED_CAPACITY


class Rows:
    """Some of a cache's sequences."""

    def __init__(self, c, which):
        self.c, self.which, self.d = c, which, c.d

    def values(self):
        return self.c.values()

    def rows(self, s, first, n, values=None):
        return self.c.rows(self.which[s], first, n, values)


@pytest.mark.parametrize("heads,n", [(2, 400_000), (12, 400_000)])
def test_attention_long_sums(B, heads, n):
    """As many sequences as CTAs over the same pages, with positive values: what the tensor core cuts off stays within 1024
    instructions' worth (2^-23 of the sum each), in the mean as well (1e-4 is five times the spread of the outputs' roundings)."""
    import torch
    kvh, page, d, n_seq = 1, 128, 128, 148
    gen = torch.Generator(device="cuda").manual_seed(n + heads)
    pages = n // page
    k = torch.randn((n, d), device="cuda", generator=gen)
    v = (3 + k + 0.5 * torch.randn((n, d), device="cuda", generator=gen)).clamp(min=0.01) * torch.exp2(torch.arange(d, device="cuda") / d)
    data = torch.zeros((pages, 2, kvh, page, d // 2), device="cuda", dtype=torch.uint8)
    scale = torch.zeros((pages, 2, kvh, page, d // 32), device="cuda", dtype=torch.bfloat16)
    table = torch.randperm(pages, device="cuda", generator=gen).to(torch.int32).view(1, -1)
    B.et_kv_append(data, scale, torch.cat([k, v], 1).to(torch.bfloat16), 0, table, i32([0]), i32([0, n]))
    codes = torch.stack([data & 15, data >> 4], -1).view(pages, 2, kvh, page, d).double() - 8
    stored = (codes * scale.double().repeat_interleave(32, -1))[table[0].long()].permute(1, 0, 2, 3, 4).reshape(2, n, d)
    del codes
    k, v = stored
    q = torch.randn((n_seq, heads, d), device="cuda", generator=gen).to(torch.bfloat16)
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


def test_cache_beyond_32_bit_offsets(B):
    """Rows, scales and attention at the far end of a cache of 4.5 GB."""
    import torch
    kvh, page, d = 8, 128, 128
    n_pages = (1 << 32) // (2 * kvh * page * d // 2) + 40
    data = torch.zeros((n_pages, 2, kvh, page, d // 2), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((n_pages, 2, kvh, page, d // 32), dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(3)
    n = 300
    table = i32([[n_pages - 1, 2, n_pages - 7]])
    x = bf16(rng.standard_normal((n, 2 * kvh * d)))
    B.et_kv_append(data, scale, x, 0, table, i32([0]), i32([0, n]))
    back = B.et_kv_read(data, scale, table, i32([0]), n, i32([0, n]))
    q = bf16(rng.standard_normal((1, kvh * d)))
    out = B.et_attention_paged(q, kvh, data, scale, table, i32([n]))
    num, s = quantise(f64(x).reshape(n, 2, kvh, d))
    v = num * np.repeat(s, 32, -1)
    assert torch.equal(back.cpu(), torch.from_numpy(v).to(torch.bfloat16).view(n, -1))
    want, _, mass, size = attention_reference(f64(q).reshape(kvh, d), *v.transpose(1, 2, 0, 3))
    drift = d * 2.0 ** -23 * size + 2.0 ** -20
    assert (np.abs(f64(out).reshape(kvh, d) - want) <= BF16 * np.abs(want) + (2.0 ** -16 + n * 2.0 ** -23 + 2 * drift)[:, None] * mass).all()


def test_attention_is_reproducible_and_independent_of_its_workspace(B):
    import torch
    rng = np.random.default_rng(9)
    lens, heads, kvh, page, d = [3000, 5, 700], 28, 4, 64, 128
    c = Cache4(rng, 3, 47, kvh, page, d)
    q = bf16(rng.standard_normal((3, heads * d)))
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((B.ET_PAGED_WORKSPACE,), fill, dtype=torch.uint8, device="cuda")
        out, lse, _ = run_attention(B, q, heads, c, lens, workspace=ws)
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_rows_that_cannot_be_placed_are_skipped(B):
    """Slots not in use, positions behind the table, pages that are not in the cache, offsets that do not fit: skipped and reported, the
    others land, nothing else is written."""
    import torch
    rng = np.random.default_rng(9)
    kvh, page, d, heads = 2, 16, 64, 2
    c = Cache4(rng, 4, 2, kvh, page, d)
    good = c.table.clone()
    for bad, code in ((c.n_pages, B.ET_PAGED_BAD_PAGE), (-1, B.ET_PAGED_BAD_PAGE), (None, B.ET_PAGED_CAPACITY), ("off", 0)):
        table, start = good.clone(), [3, 17, 30, 9]
        if bad is None:
            start[1] = 32
        elif bad == "off":
            start[1] = -1
        else:
            table[1, 1] = bad
        data0, scale0 = c.data.clone(), c.scale.view(torch.int16).clone()
        qkv, status, new_len = bf16(rng.standard_normal((4, (heads + 2 * kvh) * d))), i32([0]), i32([0] * 4)
        q = torch.full((4, heads * d), 7.0, dtype=torch.bfloat16, device="cuda")
        B.et_kv_append(c.data, c.scale, qkv, heads, table, i32(start), theta=1e4, q_out=q, new_len=new_len, status=status)
        assert status.item() == code and new_len.tolist() == [4, {None: 32, "off": -1}.get(bad, 18), 31, 10]
        assert (q[1] == 7.0).all() and not (q[[0, 2, 3]] == 7.0).all(1).any()
        where = {(good[s, start[s] // page].item(), start[s] % page) for s in (0, 2, 3)}
        for a, b in ((data0, c.data), (scale0, c.scale.view(torch.int16))):
            assert {tuple(i) for i in (a != b).any(-1).any(2).any(1).nonzero().tolist()} == where
        out = torch.full((4, 2 * kvh * d), 5.0, dtype=torch.bfloat16, device="cuda")
        status.zero_()
        B.et_kv_read(c.data, c.scale, table, i32(start), 4, None, out, status)
        assert status.item() == code and (out[1] == 5.0).all()
        for s in (0, 2, 3):
            assert torch.equal(out[s].cpu(), torch.from_numpy(c.rows(s, start[s], 1).reshape(-1)).to(torch.bfloat16))
    c = Cache4(rng, 2, 2, kvh, page, d)
    x, low = bf16(rng.standard_normal((6, 2 * kvh * d))), -2 ** 31
    for offsets, start, placed, lengths, code in (
            ([low, low + 1, 6], [0, 3], [], [0, 9], B.ET_PAGED_CAPACITY), ([low, 6, 6], [20, 0], [], [26, 0], B.ET_PAGED_CAPACITY),
            ([0, 6, 2], [4, 26], [(0, 4 + i) for i in range(6)], [10, 26], 0), ([9, 12, 15], [1, 2], [], [1, 2], 0)):
        before, new, status = c.data.clone(), i32([-9, -9]), i32([0])
        B.et_kv_append(c.data, c.scale, x, 0, c.table, i32(start), i32(offsets), new_len=new, status=status)
        changed = {tuple(i) for i in (before != c.data).any(-1).any(2).any(1).nonzero().tolist()}
        assert changed == {(c.table[s, p // page].item(), p % page) for s, p in placed} and new.tolist() == lengths and status.item() == code
        c.data.copy_(before)


@pytest.mark.parametrize("rows,heads,kvh", [(1, 40, 3), (2, 3, 16), (5, 0, 1), (90, 28, 4), (1500, 7, 1), (4000, 1, 5)])
def test_a_row_by_one_warp_or_by_several(B, rows, heads, kvh):
    """Few rows are split over warps, many dealt several to a warp; the last row of a batch stands alone in its block."""
    import torch
    rng = np.random.default_rng(rows)
    d, page = 64, 16
    pages = (rows + 7 + page - 1) // page
    c = Cache4(rng, 1, pages, kvh, page, d)
    qkv = bf16(rng.standard_normal((rows, (heads + 2 * kvh) * d)))
    q = B.et_kv_append(c.data, c.scale, qkv, heads, c.table, i32([7]), i32([0, rows]), theta=1e4)
    x = f64(qkv).reshape(rows, heads + 2 * kvh, d)
    pos = np.arange(7, 7 + rows)
    n, s = quantise(np.stack([rotate(x[:, heads:heads + kvh], pos, 1e4), x[:, heads + kvh:]], 1))
    places = c.table.cpu().numpy()[0][pos // page], pos % page
    assert np.array_equal(c.codes()[places[0], :, :, places[1]], n) and np.array_equal(f64(c.scale)[places[0], :, :, places[1]], s)
    if heads:
        want = rotate(x[:, :heads], pos, 1e4)
        slack = 2.0 ** -20 * (np.abs(x[:, :heads]) + np.abs(np.roll(x[:, :heads], d // 2, -1)))
        assert (np.abs(f64(q).reshape(want.shape) - want) <= BF16 * np.abs(want) + slack).all()


def test_decode_step_follows_the_prefill(B):
    """A prompt is prefilled, its cache moved into pages of 4 bits, and the next token decoded layer by layer: against the same step
    over pages of bf16 that hold what the 4-bit pages read back as.  The two differ by the roundings of that reading (2^-8 of a
    value) and of the activations between; the bound is the framework's for whole bf16 models, 2e-2 of the largest logit."""
    import torch
    from synthetic.llm import LLM_SMALL, llm_views, make_llm_weights, make_prompt
    sh = LLM_SMALL
    blob = make_llm_weights(sh, 4)
    ids, _ = make_prompt(sh, 151, 0, 4)
    llm = B.LanguageModel(sh, blob, max_tokens=256, keep_kv_cache=True)
    pre = llm.prefill(ids[:100], None, ids[100:150], want_kv=True)
    total, page, kvh, d, m = pre.n_tokens, 32, sh.kv_heads, sh.head_dim, sh.mlp_dim
    W = {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in llm_views(sh, blob).items()}
    t16 = lambda x: x.to(torch.bfloat16).T.contiguous()                                           # noqa: E731
    table = i32(np.random.default_rng(1).permutation(16)[:8].reshape(1, 8))
    logits = []
    for four in (True, False):
        x = W["embed"].to(torch.bfloat16)[int(ids[150])].float().view(1, -1).clone()
        lens, new, status = i32([total]), i32([0]), i32([0])
        for i in range(sh.num_layers):
            w = {k[len(f"l{i}."):]: v for k, v in W.items() if k.startswith(f"l{i}.")}
            data = torch.zeros((16, 2, kvh, page, d // 2), dtype=torch.uint8, device="cuda")
            scale = torch.zeros((16, 2, kvh, page, d // 32), dtype=torch.bfloat16, device="cuda")
            B.et_kv_append(data, scale, pre.kv_cache[i], 0, table, i32([0]), i32([0, total]), status=status)
            if not four:
                rows = B.et_kv_read(data, scale, table, i32([0]), total, i32([0, total]), status=status)
                data, scale = torch.zeros((16, 2, kvh, page, d), dtype=torch.bfloat16, device="cuda"), None
                B.et_kv_append(data, None, rows, 0, table, i32([0]), i32([0, total]), status=status)
            qkv = B.et_linear_rows(B.et_rmsnorm(x, w["rms1_g"], sh.rms_eps), t16(w["wqkv"]), w["bqkv"])
            if not four:                                          # the new token's row is quantised as well
                one, s1 = torch.zeros((1, 2, kvh, 16, d // 2), dtype=torch.uint8, device="cuda"), torch.zeros((1, 2, kvh, 16, d // 32), dtype=torch.bfloat16, device="cuda")
                far = i32([[0] * (total // 16 + 1)])
                q = B.et_kv_append(one, s1, qkv, sh.heads, far, lens, theta=sh.rope_theta, new_len=new, status=status)
                B.et_kv_append(data, None, B.et_kv_read(one, s1, far, lens, 1), 0, table, lens, status=status)
            else:
                q = B.et_kv_append(data, scale, qkv, sh.heads, table, lens, theta=sh.rope_theta, new_len=new, status=status)
            att = B.et_attention_paged(q, sh.heads, data, scale, table, new, status=status)
            B.et_linear_rows(att, t16(w["wo"]), None, 2, c=x)
            h = B.et_rmsnorm(x, w["rms2_g"], sh.rms_eps)
            gu = torch.zeros((1, 2 * m), dtype=torch.float32, device="cuda")
            B.et_linear_rows(h, t16(w["wgu"]), None, 2, c=gu)
            act = (gu[:, :m] / (1 + torch.exp(-gu[:, :m])) * gu[:, m:]).to(torch.bfloat16)
            B.et_linear_rows(act.contiguous(), t16(w["wd"]), None, 2, c=x)
        out = torch.zeros((1, sh.vocab), dtype=torch.float32, device="cuda")
        B.et_linear_rows(B.et_rmsnorm(x, W["final_g"], sh.rms_eps), t16(W["lm_head"]), None, 2, c=out)
        assert status.item() == 0 and new.item() == total + 1
        logits.append(out[0])
    off = (logits[0] - logits[1]).abs().max().item() / logits[1].abs().max().item()
    assert off <= 2e-2, off
