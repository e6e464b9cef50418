"""Attention over the cache of 4 bits (ET_KV_INT4) at the ends of its queries' range, against the 64-bit reference of test_gpu_kv_int4.py
and its tolerances."""
import numpy as np
import pytest

from tests.test_gpu_decode import bf16, f64, i32
from tests.test_gpu_kv_int4 import B, Cache4, check_attention, run_attention                      # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kvh,d", [(6, 2, 128), (6, 2, 64), (7, 1, 128), (14, 1, 128), (23, 1, 64)])
def test_attention_of_queries_up_to_the_end_of_their_type(B, heads, kvh, d):                      # noqa: F811
    """Queries of up to 2^127 with keys as small as that: the scores are ordinary ones.  Heads of ordinary queries beside them are not
    touched by it."""
    import torch
    rng = np.random.default_rng(heads + d)
    lens, page = [300, 65, 1, 640], 16
    c = Cache4(rng, len(lens), 40, kvh, page, d)
    rows = np.concatenate([[0], np.cumsum(lens)])
    k = rng.standard_normal((rows[-1], kvh, d)) * 2.0 ** -122
    x = bf16(np.stack([k, rng.standard_normal(k.shape)], 1).reshape(rows[-1], -1))
    B.et_kv_append(c.data, c.scale, x, 0, c.table, i32([0] * len(lens)), i32(rows))
    powers = np.array([121, 126, 0, 120, 118, 123, 100, 125, 122, 119, 0, 124, 60, -60])[np.arange(heads) % 14]
    q = np.clip(rng.standard_normal((len(lens), heads, d)), -3, 3)
    far = bf16((q * 2.0 ** powers[:, None]).reshape(len(lens), -1))
    assert f64(far).max() < np.inf and np.abs(f64(far)).max() > 2.0 ** 126
    out, lse, status = run_attention(B, far, heads, c, lens)
    assert status == 0
    check_attention(out, lse, f64(far).reshape(len(lens), heads, d), lens, c, heads)
    near = powers < 110
    plain = bf16((q * 2.0 ** np.where(near, powers, 1)[:, None]).reshape(len(lens), -1))
    out0, lse0, _ = run_attention(B, plain, heads, c, lens)
    keep = torch.from_numpy(near).cuda()
    assert torch.equal(out.view(-1, heads, d)[:, keep], out0.view(-1, heads, d)[:, keep]) and torch.equal(lse[:, keep], lse0[:, keep])
