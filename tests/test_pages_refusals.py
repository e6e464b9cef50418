"""What the calls of include/earlytom_pages.h and of the 4-bit cache refuse, before anything is launched.  The addresses below are made
up, so this runs only where there is no GPU that a call could reach if it were not refused."""
import os
import subprocess

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


UPDATE = dict(refs=P, n_pages=100, page=16, table=2 * P, n_seq=3, max_pages=4, lens=3 * P, keep=None, add=None, new_len=4 * P, offsets=None,
              slots=None, rows=0, ws=P, bytes=1 << 20, status=None, stream=None)
FORK = dict(refs=P, n_pages=100, page=16, table=2 * P, n_old=3, max_pages=4, lens=3 * P, parent=4 * P, n_new=5, new_table=5 * P, new_len=6 * P,
            copies=7 * P, ws=P, bytes=1 << 20, status=None, stream=None)
SELECT = dict(logits=P, fp32=0, stride=1000, n_req=2, beams=3, vocab=1000, scores=None, done=None, eos=-1, k=4, parent=P, token=P, new_scores=P,
              new_done=None, ws=P, bytes=1 << 20, stream=None)
SIZES = [(dict(refs=None), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(new_len=None), INVALID), (dict(ws=None), INVALID),
         (dict(ws=P + 8), INVALID), (dict(n_pages=0), SHAPE), (dict(page=8), SHAPE), (dict(page=48), SHAPE), (dict(page=256), SHAPE),
         (dict(max_pages=0), SHAPE), (dict(n_pages=1 << 27), CAPACITY), (dict(max_pages=(1 << 26) + 1), CAPACITY)]


@pytest.mark.parametrize("change,want", SIZES + [
    (dict(n_seq=0), SHAPE), (dict(n_seq=65537), CAPACITY), (dict(n_seq=60000, max_pages=40000), CAPACITY), (dict(rows=5), SHAPE),
    (dict(rows=-1), SHAPE), (dict(rows=(1 << 30) + 1, slots=P), CAPACITY), (dict(bytes=423), CAPACITY), (dict(keep=4 * P), INVALID),
    (dict(add=4 * P), INVALID)])
def test_update_refuses(B, change, want):
    assert B.lib().et_pages_update(*dict(UPDATE, **change).values()) == want


@pytest.mark.parametrize("change,want", SIZES + [
    (dict(parent=None), INVALID), (dict(new_table=None), INVALID), (dict(copies=None), INVALID), (dict(new_table=2 * P), INVALID),
    (dict(new_len=3 * P), INVALID), (dict(new_len=4 * P), INVALID), (dict(n_old=0), SHAPE), (dict(n_new=0), SHAPE), (dict(n_old=16385), CAPACITY),
    (dict(n_new=16385), CAPACITY), (dict(n_new=16384, max_pages=1 << 17), CAPACITY), (dict(bytes=479), CAPACITY)])
def test_fork_refuses(B, change, want):
    assert B.lib().et_pages_fork(*dict(FORK, **change).values()) == want


@pytest.mark.parametrize("change,want", [
    (dict(logits=None), INVALID), (dict(logits=P + 1), INVALID), (dict(logits=P + 2, fp32=1), INVALID), (dict(parent=None), INVALID),
    (dict(token=None), INVALID), (dict(new_scores=None), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID), (dict(scores=P), INVALID),
    (dict(done=P, new_done=P, eos=1), INVALID), (dict(n_req=0), SHAPE), (dict(beams=0), SHAPE), (dict(vocab=0), SHAPE), (dict(k=0), SHAPE),
    (dict(stride=999), SHAPE), (dict(eos=1000), SHAPE), (dict(eos=-2), SHAPE), (dict(done=P), SHAPE), (dict(beams=33), CAPACITY),
    (dict(k=65), CAPACITY), (dict(vocab=(1 << 20) + 1, stride=1 << 21), CAPACITY), (dict(n_req=30000), CAPACITY),
    (dict(bytes=6 * (8 * 4 + 16) - 1), CAPACITY)])
def test_select_refuses(B, change, want):
    assert B.lib().et_beam_select(*dict(SELECT, **change).values()) == want


def cache_of(B, **change):
    c = dict(data=P, scale=P, n_pages=8, kv_heads=2, page_size=16, head_dim=64, format=2)
    c.update(change)
    return B.et_kv_cache(*c.values())


def test_copy_refuses(B):
    def call(cache, copies=P, n=3):
        return B.lib().et_kv_copy(B.C.byref(cache) if cache else None, copies, n, None, None)
    assert call(None) == INVALID and call(cache_of(B), None) == INVALID
    assert call(cache_of(B), P, 0) == SHAPE and call(cache_of(B), P, -1) == SHAPE and call(cache_of(B), P, (1 << 24) + 1) == CAPACITY
    assert call(cache_of(B, scale=None)) == INVALID and call(cache_of(B, format=0)) == INVALID and call(cache_of(B, format=3)) == INVALID
    assert call(cache_of(B, head_dim=96)) == SHAPE and call(cache_of(B, n_pages=1 << 25)) == CAPACITY


def test_cache_of_4_bits_needs_its_scales(B):
    for change, want in ((dict(scale=None), INVALID), (dict(scale=P + 8), INVALID), (dict(head_dim=32), SHAPE), (dict(data=P + 4), INVALID)):
        c = B.C.byref(cache_of(B, **change))
        assert B.lib().et_kv_append(c, P, 512, 3, 4, P, 3, 4, None, P, 1e4, P, None, None, None) == want
        assert B.lib().et_kv_read(c, P, 256, 3, P, 3, 4, None, P, None, None) == want
        assert B.lib().et_attention_paged(c, P, 256, P, None, 3, 4, P, 4, P, P, 4 << 20, None, None) == want


def test_workspaces_and_codes_match_the_header(B, tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include "earlytom_pages.h"\nint main(){printf("%llu %llu %llu %d %d %d %d %d\\n",'
                   'ET_PAGES_WORKSPACE(1001,7),ET_FORK_WORKSPACE(1001,7),ET_BEAM_WORKSPACE(6,12289,5),ET_PAGED_NO_PAGE,ET_PAGED_BAD_COUNT,'
                   'ET_PAGED_BAD_ROW,ET_KV_INT4,ET_BEAM_CHUNK);return 0;}\n')
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "sz")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "sz")]).split()]
    assert got == [B.ET_PAGES_WORKSPACE(1001, 7), B.ET_FORK_WORKSPACE(1001, 7), B.ET_BEAM_WORKSPACE(6, 12289, 5), B.ET_PAGED_NO_PAGE,
                   B.ET_PAGED_BAD_COUNT, B.ET_PAGED_BAD_ROW, B.ET_KV_INT4, B.ET_BEAM_CHUNK]


def test_python_calls_refuse_what_they_cannot_pass_on(B):
    """Types, shapes and strides of the tensors, and tensors that are not on the GPU."""
    i = torch.int32
    refs, table, lens = torch.zeros(8, dtype=i), torch.zeros((3, 2), dtype=i), torch.zeros(3, dtype=i)
    x = torch.zeros((6, 40))
    four, scale = torch.zeros((4, 2, 2, 16, 32), dtype=torch.uint8), torch.zeros((4, 2, 2, 16, 2), dtype=torch.bfloat16)
    copies, q = torch.zeros((2, 3), dtype=i), torch.zeros((3, 256), dtype=torch.bfloat16)
    update = lambda refs=refs, table=table, lens=lens, **kw: B.et_pages_update(refs, 16, table, lens, **kw)                       # noqa: E731
    fork = lambda refs=refs, table=table, lens=lens, parent=lens, new=table.clone(), **kw: B.et_pages_fork(refs, 16, table, lens, parent, new, **kw)  # noqa: E731
    bad = [lambda: update(), lambda: update(refs=refs.long()), lambda: update(refs=refs[::2]), lambda: update(refs=refs.view(2, 4)),
           lambda: update(table=table.T), lambda: update(lens=lens[:2]), lambda: update(keep=lens.long()), lambda: update(add=lens[:1]),
           lambda: update(new_len=lens.float()), lambda: update(row_offsets=lens), lambda: update(slots=table), lambda: update(status=lens),
           lambda: update(workspace=torch.zeros((9, 9), dtype=torch.uint8)[:, ::2]),
           lambda: fork(), lambda: fork(new=torch.zeros((3, 3), dtype=i)), lambda: fork(parent=lens[:2]), lambda: fork(copies=lens),
           lambda: fork(new_len=lens.long()), lambda: fork(new=table.T),
           lambda: B.et_kv_copy(four, scale, copies), lambda: B.et_kv_copy(four, scale, copies.long()), lambda: B.et_kv_copy(four, scale, copies[:, :2]),
           lambda: B.et_kv_copy(four, None, copies), lambda: B.et_kv_copy(four, scale.float(), copies), lambda: B.et_kv_copy(four, scale[..., :1], copies),
           lambda: B.et_kv_copy(four, scale[:3], copies), lambda: B.et_kv_copy(four.view(torch.int8), scale, copies),
           lambda: B.et_kv_append(four, scale[..., 0], q, 0, table, lens), lambda: B.et_kv_read(four, scale.view(torch.float16), table, lens, 3),
           lambda: B.et_attention_paged(q, 4, four, scale.permute(0, 1, 2, 4, 3), table, lens),
           lambda: B.et_beam_select(x, 3, 4), lambda: B.et_beam_select(x.double(), 3, 4), lambda: B.et_beam_select(x[0], 3, 4), lambda: B.et_beam_select(x.T, 5, 4),
           lambda: B.et_beam_select(x, 4, 4), lambda: B.et_beam_select(x, 0, 4), lambda: B.et_beam_select(x, 3, 0),
           lambda: B.et_beam_select(x, 3, 4, scores=torch.zeros(5)), lambda: B.et_beam_select(x, 3, 4, done=torch.zeros(6)),
           lambda: B.et_beam_select(x, 3, 4, parent=torch.zeros(6, dtype=i)), lambda: B.et_beam_select(x, 3, 4, token=torch.zeros(8, dtype=torch.int64)),
           lambda: B.et_beam_select(x, 3, 4, new_scores=torch.zeros(8, dtype=torch.float64)), lambda: B.et_beam_select(x.sum(), 3, 4)]
    for n, f in enumerate(bad):
        with pytest.raises(B.EarlyTomError) as e:
            f()
        assert e.value.status == INVALID, n
