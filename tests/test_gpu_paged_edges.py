"""The paged cache's calls at the edges of what they allow: see also test_gpu_paged.py, whose definitions they are compared with."""
import math

import pytest
import torch

from test_gpu_paged import BF16, F16, F32, TYPES, attention_case, attention_reference, check_attention, half_step, ints, pkg, pool  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- fewer keys than new rows: the first rows sit in front of position 0

@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("nq,nkv,D,new,lens", [
    (8, 8, 128, [600], [100]),                                       # one query head to a kv head: row tiles longer than a unit of keys
    (8, 8, 128, [300, 1, 1500, 40], [100, 700, 1373, 0]),
    (8, 8, 64, [512, 700], [312, 1]),
    (4, 2, 128, [700, 130], [300, 129]),
    (15, 5, 64, [300, 90], [33, 80]),
    (16, 1, 128, [70], [3]),
])
def test_pieces_with_fewer_keys_than_rows(pkg, qt, kv, nq, nkv, D, new, lens):
    c = attention_case(21, [max(0, m - n) for m, n in zip(lens, new)], new, nq, nkv, D, qt, kv, 16, "hnd", pad=2)
    c["lens"] = lens
    for max_new in (0, max(new)):
        got = check_attention(pkg, c, max_new=max_new)
        for b, n in enumerate(new):
            t0 = c["start"][b]
            assert (got[t0:t0 + max(0, n - lens[b])] == 0).all()
        assert (got[-2:] == 5.0).all()


@pytest.mark.parametrize("nq,nkv", [(8, 8), (8, 2)])
def test_a_refused_piece_of_a_prompt(pkg, nq, nkv):
    """The plan refuses a piece and keeps its rows and its old length: its rows mean nothing, those of the others are as without it."""
    D, page, new = 128, 16, [5, 600, 3]
    c = attention_case(22, [200, 90, 40], new, nq, nkv, D, BF16, BF16, page, "nhd")
    n_pages = c["kc"].shape[0]
    table = c["table"].clone()
    table[0, -(-200 // page):] = -1
    table[1, -(-90 // page):] = -1
    table[2, -(-40 // page):] = -1
    held = set(table[table >= 0].tolist())
    free = [p for p in range(n_pages) if p not in held]
    # room for the first and the last, not for the piece: the last asks for none beside the first's one
    stack = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
    stack[:1] = ints(free[:1])
    lens = [200, 90, 40]
    plan = pkg.paged_plan(ints(lens), ints(new), table, stack, ints([1]), page, sum(new))
    assert plan.granted.tolist() == [5, 0, 3] and plan.lens.tolist() == [205, 90, 43] and plan.row_start.tolist() == [0, 5, 605, 608]
    rows = torch.arange(n_pages * page, device="cuda")
    for t in (c["kc"], c["vc"]):                                     # (every page holds something: no NaN from the test's own filling)
        t[rows // page, :, rows % page] = torch.randn(n_pages * page, nkv, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    c["lens"], c["start"], c["table"] = plan.lens.tolist(), plan.row_start.tolist(), table
    got = check_attention(pkg, c, finite=False)
    assert torch.isfinite(got).all()
