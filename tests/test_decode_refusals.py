"""What the decode step's entry points refuse, before anything is launched.  The addresses below are made up, so this
runs only where there is no GPU that a call could reach if it were not refused."""
import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where no GPU can be reached")

INVALID, SHAPE, CAPACITY = 1, 2, 3
P = 1 << 20            # some 16-byte aligned address


@pytest.fixture(scope="module")
def B():
    from paper_2605_30010_b200 import build
    build.build()
    from paper_2605_30010_b200 import binding
    return binding


def call(B, name, base, order, **change):
    cache = dict(data=P, scale=None, n_pages=8, kv_heads=2, page_size=16, head_dim=64, format=0)
    cache.update({k[6:]: v for k, v in change.items() if k.startswith("cache_")})
    args = dict(base, **{k: v for k, v in change.items() if not k.startswith("cache_")})
    c = B.et_kv_cache(*[cache[k] for k in ("data", "scale", "n_pages", "kv_heads", "page_size", "head_dim", "format")])
    return getattr(B.lib(), name)(B.C.byref(c), *[args[k] for k in order])


APPEND = dict(qkv=P, stride=(4 + 4) * 64, rows=3, heads=4, table=P, n_seq=3, max_pages=4, offsets=None, start=P, theta=1e4, q_out=P,
              new_len=None, status=None, stream=None)
READ = dict(out=P, stride=4 * 64, rows=3, table=P, n_seq=3, max_pages=4, offsets=None, start=P, status=None, stream=None)
ATTEND = dict(q=P, stride=4 * 64, out=P, lse=None, n_seq=3, heads=4, table=P, max_pages=4, lens=P, ws=P, ws_bytes=4 << 20, status=None,
              stream=None)

CACHE = [(dict(cache_data=None), INVALID), (dict(cache_data=P + 8), INVALID), (dict(cache_format=2), INVALID), (dict(cache_format=1), INVALID),
         (dict(cache_scale=P), INVALID), (dict(cache_format=1, cache_scale=P + 4), INVALID), (dict(cache_n_pages=0), SHAPE),
         (dict(cache_head_dim=96), SHAPE), (dict(cache_head_dim=256), SHAPE), (dict(cache_page_size=8), SHAPE), (dict(cache_page_size=48), SHAPE),
         (dict(cache_page_size=256), SHAPE), (dict(cache_kv_heads=0), SHAPE), (dict(cache_n_pages=1 << 25), CAPACITY),
         (dict(cache_n_pages=2 ** 31 - 1, cache_kv_heads=2 ** 31 - 1), CAPACITY),
         (dict(table=None), INVALID), (dict(n_seq=0, rows=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 27), CAPACITY)]


@pytest.mark.parametrize("change,want", CACHE + [
    (dict(qkv=None), INVALID), (dict(qkv=P + 2), INVALID), (dict(start=None), INVALID), (dict(rows=0), SHAPE), (dict(rows=4), SHAPE),
    (dict(rows=-1, offsets=P), SHAPE), (dict(theta=1.0), INVALID), (dict(theta=-2.0), INVALID), (dict(theta=float("nan")), INVALID),
    (dict(theta=float("inf")), INVALID), (dict(q_out=None), INVALID), (dict(theta=0.0), INVALID), (dict(q_out=P + 8), INVALID),
    (dict(heads=-1), SHAPE), (dict(heads=0), INVALID), (dict(heads=0, q_out=None, stride=4 * 64 - 8), SHAPE), (dict(stride=8 * 64 + 4), SHAPE),
    (dict(stride=8 * 64 - 8), SHAPE), (dict(new_len=P), INVALID), (dict(heads=2 ** 31 - 1), SHAPE)])
def test_append_refuses(B, change, want):
    assert call(B, "et_kv_append", APPEND, list(APPEND), **change) == want


@pytest.mark.parametrize("change,want", CACHE + [
    (dict(out=None), INVALID), (dict(out=P + 4), INVALID), (dict(start=None), INVALID), (dict(rows=2), SHAPE), (dict(stride=4 * 64 - 8), SHAPE),
    (dict(stride=4 * 64 + 1), SHAPE), (dict(rows=0, offsets=P), SHAPE)])
def test_read_refuses(B, change, want):
    assert call(B, "et_kv_read", READ, list(READ), **change) == want


@pytest.mark.parametrize("change,want", [(c, w) for c, w in CACHE if "rows" not in c] + [
    (dict(n_seq=0), SHAPE), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(lens=None), INVALID), (dict(ws=None), INVALID),
    (dict(q=P + 2), INVALID), (dict(out=P + 2), INVALID), (dict(ws=P + 8), INVALID), (dict(heads=0), SHAPE), (dict(heads=5), SHAPE),
    (dict(stride=4 * 64 - 8), SHAPE), (dict(stride=4 * 64 + 2), SHAPE), (dict(ws_bytes=(4 << 20) - 1), CAPACITY), (dict(n_seq=1 << 23), CAPACITY)])
def test_attention_refuses(B, change, want):
    assert call(B, "et_attention_paged", ATTEND, list(ATTEND), **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(a=None), INVALID), (dict(w=None), INVALID), (dict(c=None), INVALID), (dict(a=P + 2), INVALID), (dict(w=P + 8), INVALID),
    (dict(c=P + 4), INVALID), (dict(epilogue=3), INVALID), (dict(epilogue=5), INVALID), (dict(epilogue=-1), INVALID), (dict(M=0), SHAPE),
    (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=12), SHAPE), (dict(epilogue=4, N=128), SHAPE), (dict(M=33), CAPACITY),
    (dict(N=(1 << 24) + 8), CAPACITY), (dict(K=(1 << 24) + 8), CAPACITY)])
def test_linear_rows_refuses(B, change, want):
    base = dict(a=P, w=P, bias=None, c=P, M=4, N=64, K=64, epilogue=0, gelu=1, status=None, stream=None)
    args = dict(base, **change)
    assert B.lib().et_linear_rows(*[args[k] for k in base]) == want


def test_null_cache_is_refused(B):
    assert B.lib().et_kv_append(None, *APPEND.values()) == INVALID
    assert B.lib().et_kv_read(None, *READ.values()) == INVALID
    assert B.lib().et_attention_paged(None, *ATTEND.values()) == INVALID


def test_struct_matches_the_header(B, tmp_path):
    import ctypes
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include "earlytom_decode.h"\nint main(){printf("%zu %u %d %d\\n",sizeof(et_kv_cache),'
                   'ET_PAGED_WORKSPACE,ET_PAGED_CAPACITY,ET_PAGED_BAD_PAGE);return 0;}\n')
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sz")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "sz")]).split()]
    assert B._KV_CACHE.size == ctypes.sizeof(B.et_kv_cache)
    fields = (1 << 40, 2 << 40, 3, 4, 5, 6, 1)
    assert B._KV_CACHE.pack(*fields)[:36] == bytes(B.et_kv_cache(*fields))[:36]
    assert got == [ctypes.sizeof(B.et_kv_cache), B.ET_PAGED_WORKSPACE, B.ET_PAGED_CAPACITY, B.ET_PAGED_BAD_PAGE]


def test_python_calls_refuse_what_they_cannot_pass_on(B):
    """Types, shapes and strides of the tensors, and tensors that are not on the GPU."""
    import torch
    bf = torch.bfloat16
    cache = torch.zeros((4, 2, 2, 16, 64), dtype=bf)
    table, lens = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros((3, 256), dtype=bf)
    bad = [lambda: B.et_attention_paged(q, 4, cache.float(), None, table, lens),
           lambda: B.et_attention_paged(q, 4, cache, torch.zeros(4, 2, 2, 16, dtype=torch.uint8), table, lens),
           lambda: B.et_attention_paged(q, 4, cache.view(torch.int16).to(torch.float8_e4m3fn), None, table, lens),
           lambda: B.et_attention_paged(q, 4, cache.transpose(2, 3), None, table, lens),
           lambda: B.et_attention_paged(q, 4, cache, None, table.long(), lens),
           lambda: B.et_attention_paged(q[:, :100], 4, cache, None, table, lens),
           lambda: B.et_kv_read(cache, None, table.T, lens, 3)]
    for f in bad:
        with pytest.raises(B.EarlyTomError) as e:
            f()
        assert e.value.status == INVALID


def test_python_calls_refuse_shapes_with_the_binding_s_error(B):
    """Tensors of another number of dimensions and negative counts are refused like everything else, not by an error of torch's."""
    bf = torch.bfloat16
    cache = torch.zeros((4, 2, 2, 16, 64), dtype=bf)
    table, lens = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    q, a, w = torch.zeros((3, 256), dtype=bf), torch.zeros((2, 64), dtype=bf), torch.zeros((64, 64), dtype=bf)
    bad = [lambda: B.et_linear_rows(a[0], w), lambda: B.et_linear_rows(a, w[0]), lambda: B.et_linear_rows(a[None], w),
           lambda: B.et_linear_rows(a.sum(), w), lambda: B.et_attention_paged(q.sum(), 4, cache, None, table, lens),
           lambda: B.et_attention_paged(q, -1, cache, None, table, lens), lambda: B.et_attention_paged(q[None], 4, cache, None, table, lens),
           lambda: B.et_kv_append(cache, None, q.sum(), 0, table, lens), lambda: B.et_kv_append(cache, None, q, -1, table, lens, theta=1e4),
           lambda: B.et_kv_read(cache, None, table, lens, -1), lambda: B.et_kv_read(cache, None, table, lens, 3, out=q.sum()),
           lambda: B.et_kv_read(cache, None, table, lens, 3, out=q[:, 0])]
    for i, f in enumerate(bad):
        with pytest.raises(B.EarlyTomError) as e:
            f()
        assert e.value.status == INVALID, i
