"""The paged cache's calls at the edges of what they allow: see also test_gpu_paged.py, whose definitions they are compared with."""
import math

import pytest
import torch

from test_gpu_paged import BF16, F16, F32, TYPES, attention_case, attention_reference, check_attention, half_step, ints, pkg, plan_case, plan_reference, \
    pool  # noqa: F401

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


# ---- NaN stays

def check_nan(pkg, c, rows_heads, max_new=0):
    """NaN in all of these (row, query head) and nowhere else."""
    got = check_attention(pkg, c, max_new=max_new, finite=False)
    want = torch.zeros(got.shape[:2], dtype=torch.bool, device="cuda")
    for t, h in rows_heads:
        want[t, h] = True
    assert torch.equal(torch.isnan(got).all(-1), want) and torch.equal(torch.isnan(got).any(-1), want)


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("nq,nkv,D,cached,new,max_new", [
    (8, 2, 128, [0, 5], [1, 2], 0),                    # one key
    (8, 2, 128, [40, 5], [2, 1], 2),                   # an item in one piece or a few
    (16, 2, 64, [4000], [3], 3),                       # in many
    (8, 2, 128, [70, 3], [200, 60], 0),                # pieces of prompts
    (8, 8, 64, [1, 3], [130, 300], 0),
    (4, 1, 128, [9000], [100], 0),                     # ... an item cut into many pieces
])
def test_a_query_with_a_nan(pkg, qt, kv, nq, nkv, D, cached, new, max_new):
    c = attention_case(31, cached, new, nq, nkv, D, qt, kv, 16, "hnd")
    T = sum(new)
    at = sorted({(0, 0), (T - 1, nq - 1), (T // 2, 1)})
    for n, (t, h) in enumerate(at):
        c["q"][t, h, 7 * n % D] = math.nan
    check_nan(pkg, c, at, max_new)


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cached,new", [([0], [1]), ([16], [1]), ([8], [1]), ([32], [1]), ([64], [1]), ([128], [1]), ([1023], [2]), ([4095, 64], [1, 1]),
                                        ([128], [90]), ([0], [70]), ([8999], [100])])
def test_a_nan_key_alone_in_its_tile(pkg, qt, kv, D, cached, new):
    """The last key of the first new row's sight has a NaN: that row and those behind it see it, wherever a tile or a piece begins."""
    c = attention_case(32, cached, new, 8, 2, D, qt, kv, 16, "hnd")
    for b, n in enumerate(cached):
        c["kc"][c["table"][b, n // 16].long(), 1, n % 16, 3] = math.nan
    rows = [(c["start"][b] + r, h) for b in range(len(new)) for r in range(new[b]) for h in range(4, 8)]
    check_nan(pkg, c, rows)


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("cached,new", [([700, 3], [1, 2]), ([6000], [3]), ([30], [40]), ([6000], [60])])
def test_keys_that_are_all_nan(pkg, qt, kv, cached, new):
    """Every score of a row is NaN, in all its pieces; the other requests' and heads' rows are as ever."""
    c = attention_case(33, cached, new, 8, 2, 128, qt, kv, 16, "nhd")
    pages = c["table"][0][c["table"][0] >= 0].long()
    c["kc"][pages, 0] = math.nan
    check_nan(pkg, c, [(t, h) for t in range(new[0]) for h in range(4)])


# ---- what the kernels of a call find in scratch, and of the launches in front of it

@pytest.mark.parametrize("fill", [0, 255, "entered"])
@pytest.mark.parametrize("qt,kv", [(BF16, BF16), (F16, F16), (F32, F16)])
def test_scratch_may_hold_anything(pkg, qt, kv, fill):
    """Zeros, ones, and the word (everywhere) that the chunk kernel leaves for the row kernel behind it."""
    c = attention_case(41, [900, 4, 3000], [200, 1, 3], 8, 2, 128, qt, kv, 16, "hnd")
    args = c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"]
    scratch = torch.empty(pkg.PAGED_ATTENTION_SCRATCH_BYTES // 4, dtype=torch.int32, device="cuda")
    scratch.fill_({0: 0, 255: -1, "entered": 0x9d1c6b35 - (1 << 32)}[fill])
    want = check_attention(pkg, c)
    for _ in range(3):
        assert torch.equal(pkg.paged_attention(*args, scratch=scratch, out=c["out"].clone()), want)


@pytest.mark.parametrize("graph", [False, True])
def test_rows_behind_a_piece_read_the_step_in_front(pkg, graph):
    """Single rows beside a piece of a prompt: the kernel of the rows starts under that of the pieces, behind plan and append launches
    that changed lengths, table and cache just now.  Step after step against the same call on a quiet device."""
    B, nq, nkv, D, page, width = 9, 8, 2, 128, 8, 40
    g = torch.Generator(device="cuda").manual_seed(42)
    n_pages, n_rows = B * width, 100
    lens, n_free = ints([0] * B), ints([n_pages])
    n_new = ints([1] * (B - 1) + [60])
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=g, device="cuda").int()
    kc, vc = pool(n_pages, nkv, page, D, BF16, "nhd")
    q, k, v = (torch.zeros(n_rows, h, D, dtype=BF16, device="cuda") for h in (nq, nkv, nkv))
    plan = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, n_rows, n_rows, B)] + [lens, n_free]
    q_rot, out = torch.zeros_like(q), torch.zeros_like(q)
    scratch = torch.empty(pkg.PAGED_ATTENTION_SCRATCH_BYTES, dtype=torch.uint8, device="cuda")

    def step():
        p = pkg.paged_plan(lens, n_new, table, free, n_free, page, n_rows, out=plan)
        pkg.paged_append(q, k, v, p.position, p.slot, kc, vc, rope_theta=1e4, q_out=q_rot)
        pkg.paged_attention(q_rot, p.row_start, p.lens, table, kc, vc, scratch=scratch, out=out)
    replay = step
    if graph:
        n_new.zero_()
        step()
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        replay = captured.replay
    for i in range(40):
        todo = [1] * (B - 1) + [60]
        if i % 4 == 3:
            todo = [-1] * B                                          # everything ends; pages go round
        n_new.copy_(ints(todo))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        out.fill_(3.0)
        replay()
        torch.cuda.synchronize()
        quiet = pkg.paged_attention(q_rot, plan[0], lens, table, kc, vc, out=torch.full_like(out, 3.0))
        assert torch.equal(out, quiet), i
        assert plan[3].tolist() == [max(0, n) for n in todo]


# ---- rows that are worked out from the definition

@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("cached,new,D", [([9000], [100], 128), ([9000], [100], 64), ([4000, 100], [1, 3], 128), ([500, 40, 8], [300, 70, 90], 128)])
def test_the_same_bits_with_infinities(pkg, qt, kv, cached, new, D):
    """An infinity in one dimension of V, seen by some rows and not by others, in items cut into pieces: the same call gives the same bits."""
    c = attention_case(51, cached, new, 8, 2, D, qt, kv, 16, "hnd")
    for n in (cached[0] // 2, cached[0] + new[0] // 2):
        c["vc"][c["table"][0, n // 16].long(), :, n % 16, 5 + n % 7] = math.inf
    first = check_attention(pkg, c, finite=False)
    assert (first[: new[0]].isinf().any(-1)).all()
    args = c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"]
    for _ in range(8):
        assert torch.equal(torch.nan_to_num(pkg.paged_attention(*args, out=c["out"].clone())), torch.nan_to_num(first))


@pytest.mark.parametrize("qt,kv", [(BF16, BF16), (F16, F16)])
def test_infinities_in_shares_of_many_items(pkg, qt, kv):
    """More items than blocks, most of them whole: those of some requests hold an infinity that a part of their rows see."""
    B, page = 150, 16
    new = [33 + 13 * b % 60 for b in range(B)]
    cached = [29 * b % 300 for b in range(B)]
    c = attention_case(52, cached, new, 8, 4, 64, qt, kv, page, "nhd", pad=3)
    at = [b for b in range(B) if b % 11 == 4]
    for b in at:
        n = cached[b] + new[b] // 2
        c["vc"][c["table"][b, n // page].long(), 1, n % page, 9] = -math.inf
    got = check_attention(pkg, c, finite=False)
    want = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    for b in at:
        want[c["start"][b] + new[b] // 2:c["start"][b + 1], 2:4, 9] = True
    assert torch.equal(got == -math.inf, want) and torch.isfinite(got[~want]).all()


# ---- append

@pytest.mark.parametrize("act", [F32, BF16, F16])
@pytest.mark.parametrize("T,D", [(3, 64), (2100, 128)])
def test_no_rotation_leaves_values_alone(pkg, act, T, D):
    """rope_theta 0 and no norm: queries and keys as they are, infinities and NaN in one half without influence on the other."""
    g = torch.Generator(device="cuda").manual_seed(61)
    q, k, v = (torch.randn(T, h, D, generator=g, device="cuda").to(act) for h in (4, 2, 2))
    for t in (q, k):
        t[0, 0, 3], t[1, 1, D // 2 + 5], t[2, 0, 1], t[T - 1, 1, D - 1] = math.inf, -math.inf, math.nan, math.inf
    kc, vc = pool(T, 2, 1, D, act, "hnd")
    at = torch.arange(T, device="cuda").int()
    got = pkg.paged_append(q, k, v, at + 1000, at, kc, vc, rope_theta=0.0)
    for x, y in ((got, q), (kc[:, :, 0], k), (vc[:, :, 0], v)):
        assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(torch.nan_to_num(x, nan=7.0), torch.nan_to_num(y, nan=7.0))


# ---- the forms that max_new chooses between

@pytest.mark.parametrize("qt", [BF16, F16])
@pytest.mark.parametrize("nq,nkv,D,cached,new", [(8, 2, 128, [700, 30], [300, 9]), (8, 8, 64, [0, 2500], [49, 120]), (16, 1, 128, [90], [3])])
def test_what_max_new_may_change(pkg, qt, nq, nkv, D, cached, new):
    """max_new 1: probabilities in two parts, each off by half a step of its own (a step of the first part squared: 2^-16, 2^-22).  Unknown:
    once rounded in the larger requests, half a step of sum p |v| further.  Both: the result's own rounding, and 2e-5 of sum p |v| as everywhere."""
    c = attention_case(71, cached, new, nq, nkv, D, qt, qt, 16, "hnd")
    ref, size = attention_reference(c["q"], c["start"], c["lens"], c["table"], c["kc"], c["vc"], c["out"])
    args = c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"]
    fine, coarse = (pkg.paged_attention(*args, max_new=m) for m in (1, 0))
    h = half_step(qt)
    # fp16: parts below 2^-24 of a probability of 2^8 or more, for as many keys as there are; results below 2^-14
    base = (2e-5 + h * h) * size + 1e-6 + (max(c["lens"]) * 2.0 ** -33 * c["vc"].nan_to_num(0).abs().max() + 2.0 ** -25 if qt == F16 else 0)
    assert ((fine.double() - ref).abs() <= h * ref.abs() + base).all()
    assert ((coarse.double() - ref).abs() <= h * (ref.abs() + size) + base).all()
    for m, want in ((1, fine), (0, coarse), (max(new), coarse)):
        assert torch.equal(pkg.paged_attention(*args, max_new=m), want)


# ---- both sides of every border between launch shapes

@pytest.mark.parametrize("B,page,width,most_new,n_rows,ended", [
    (7, 16, 20, 60, 512, 0.2), (7, 16, 20, 60, 513, 0.2),                   # a block of 128 threads, of 512
    (128, 16, 8, 3, 500, 0.1), (129, 16, 8, 3, 500, 0.1),
    (512, 16, 8, 1, 1000, 0.1), (513, 16, 8, 1, 1000, 0.1),                 # of 512, of 1024
    (7, 16, 20, 100, 1024, 0.2), (7, 16, 20, 100, 1025, 0.2),               # a block, a cluster
    (1024, 16, 8, 0, 1024, 0.1), (1025, 16, 8, 0, 1024, 0.1),
    (60, 32, 30, 400, 16384, 0.1), (60, 32, 30, 400, 16385, 0.1),           # rows by the same launch, by a second one
])
def test_plan_at_the_borders(pkg, B, page, width, most_new, n_rows, ended):
    for seed in range(2):
        lens, n_new, table, stack, n_pages, rows = plan_case(seed, B, page, width, most_new, 0, seed == 1, ended, seed == 1)
        want = plan_reference(lens, n_new, table, stack, n_pages, page, n_rows)          # (rows behind the last request's, or too few of them)
        free = torch.full((n_pages,), -9, dtype=torch.int32, device="cuda")
        free[:len(stack)] = ints(stack)
        t = ints(table)
        p = pkg.paged_plan(ints(lens), ints(n_new), t, free, ints([len(stack)]), page, n_rows)
        for name, got, ref in zip(p._fields, p, want):
            assert got.tolist() == list(ref), (seed, name)
        assert t.tolist() == want[-1], seed


@pytest.mark.parametrize("T", [1, 2, 166, 167, 200, 222, 223, 250, 285, 286, 333, 334, 400, 401, 500, 501, 666, 667, 1000, 1001, 2000, 2001])
@pytest.mark.parametrize("nq,nkv,D,act", [(32, 8, 128, BF16), (4, 2, 64, F32), (5, 1, 64, F16), (0, 1, 128, F32)])
def test_append_parts_of_a_row(pkg, nq, nkv, D, act, T):
    """Rows cut into 2000 / T parts: every part's vectors once, whatever the number of parts; as the rows one by one give them."""
    g = torch.Generator(device="cuda").manual_seed(T)
    q, k, v = (torch.randn(T, h, D, generator=g, device="cuda").to(act) if h else None for h in (nq, nkv, nkv))
    pos = torch.randint(0, 1 << 16, (T,), generator=g, device="cuda").int()
    slot = torch.randperm(T, generator=g, device="cuda").int()
    norm = 1 + 0.1 * torch.randn(D, generator=g, device="cuda")
    kc, vc = pool(T, nkv, 1, D, act, "hnd", fill=9.0)
    got = pkg.paged_append(q, k, v, pos, slot, kc, vc, q_norm=norm, k_norm=norm, rope_theta=1e6)
    some = sorted({0, T // 3, T - 1})
    for t in some:
        one = slice(t, t + 1)
        k1, v1 = pool(T, nkv, 1, D, act, "hnd")
        q1 = pkg.paged_append(None if q is None else q[one], k[one], v[one], pos[one], slot[one], k1, v1, q_norm=norm, k_norm=norm, rope_theta=1e6)
        at = slot[t].long()
        assert torch.equal(kc[at], k1[at]) and torch.equal(vc[at], v1[at]) and (q is None or torch.equal(got[t], q1[0]))
    assert torch.equal(vc[slot.long(), :, 0], v) and not (kc == 9.0).all(-1).any()


# ---- calls that the header allows

@pytest.mark.parametrize("qt,kv", TYPES)
def test_rows_in_front_of_the_first_request(pkg, qt, kv):
    """row_start need not begin at 0: rows of no request, in front and behind, stay as they were."""
    c = attention_case(81, [100, 0, 900], [70, 3, 1], 8, 2, 128, qt, kv, 16, "hnd", pad=9)
    c["start"] = [s + 5 for s in c["start"]]
    got = check_attention(pkg, c)
    assert (got[:5] == 5.0).all() and (got[c["start"][-1]:] == 5.0).all()


@pytest.mark.parametrize("qt,kv", TYPES)
def test_requests_that_share_pages(pkg, qt, kv):
    """A prompt's common pages in several tables, twice in one; other lengths behind them."""
    c = attention_case(82, [96, 30, 64, 5], [40, 2, 1, 3], 8, 2, 64, qt, kv, 16, "nhd")
    first = c["table"][0, :6].clone()
    c["table"][1, :1] = first[0]
    c["table"][2, :4] = first[:4]
    c["table"][0, 5] = first[0]
    c["table"][3, 0] = first[2]
    check_attention(pkg, c)


@pytest.mark.parametrize("qt,kv", [(F32, F16), (BF16, BF16)])
def test_the_most_requests(pkg, qt, kv):
    B = 8192
    cached = [7 * b % 40 for b in range(B)]
    new = [b % 3 for b in range(B)]
    new[5000], new[8191] = 80, 40
    # keys and values at once: a page to 64 positions, requests one after the other
    g = torch.Generator(device="cuda").manual_seed(83)
    page, nq, nkv, D = 64, 2, 1, 64
    lens = [a + n for a, n in zip(cached, new)]
    held = torch.tensor([-(-n // page) for n in lens])
    width = int(held.max())
    table = torch.full((B, width), -1, dtype=torch.int32)
    col = torch.arange(width)[None] < held[:, None]
    table[col] = torch.randperm(int(held.sum()), generator=torch.Generator().manual_seed(1)).int()
    kc, vc = (torch.randn(int(held.sum()), nkv, page, D, generator=g, device="cuda").to(kv) for _ in range(2))
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    q = torch.randn(start[-1], nq, D, generator=g, device="cuda").to(qt)
    args = ints(start), ints(lens), table.cuda(), kc, vc
    got = pkg.paged_attention(q, *args)
    # every request by itself
    for b in (1, 2, 31, 32, 4097, 4999, 5000, 5002, 8190, 8191):
        if new[b]:
            one = pkg.paged_attention(q[start[b]:start[b + 1]], ints([0, new[b]]), ints([lens[b]]), args[2][b:b + 1], kc, vc)
            assert (got[start[b]:start[b + 1]].float() - one.float()).abs().max() <= 4 * half_step(qt) * one.float().abs().max() + 1e-5
    dense = {n: [b for b in range(B) if new[b] == 1 and lens[b] == n] for n in (1, 20, 40)}
    for n, some in dense.items():
        at = args[2][some, 0].long()
        p = torch.softmax(torch.einsum("bhd,bkd->bhk", q[[start[b] for b in some]].double(), kc[at, 0, :n].double()) / 8.0, -1)
        ref = torch.einsum("bhk,bkd->bhd", p, vc[at, 0, :n].double())
        assert ((got[[start[b] for b in some]].double() - ref).abs() <= 2 * half_step(qt) * vc.float().abs().max() + 2e-5).all()


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("nq,nkv,D,page,cached,new", [
    (64, 64, 64, 16, [40, 3], [50, 1]),                              # many kv heads
    (7, 7, 128, 2, [10, 90], [34, 3]),                               # pages smaller than a copy
    (8, 8, 128, 32, [0, 333], [700, 41]),                            # one query head to a kv head, several row tiles
    (16, 16, 64, 4096, [900], [260]),                                # a page for all
    (48, 3, 64, 8, [17], [33]),
])
def test_other_head_counts(pkg, qt, kv, nq, nkv, D, page, cached, new):
    c = attention_case(84, cached, new, nq, nkv, D, qt, kv, page, "hnd", pad=1)
    for max_new in (0, 1):
        check_attention(pkg, c, max_new=max_new)


def test_two_graphs_take_turns_on_one_scratch(pkg):
    cases = [attention_case(85, [900, 4], [200, 1], 8, 2, 128, BF16, BF16, 16, "hnd"), attention_case(86, [0, 1300, 60], [90, 1, 40], 8, 8, 64, F16, F16, 32, "nhd")]
    want = [check_attention(pkg, c) for c in cases]
    args = [(c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"]) for c in cases]
    scratch = torch.empty(pkg.PAGED_ATTENTION_SCRATCH_BYTES, dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(c["out"]) for c in cases]
    graphs = []
    for a, o in zip(args, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(3):
                pkg.paged_attention(*a, scratch=scratch, out=o)
        graphs.append(g)
    for _ in range(10):
        for g, o in zip(graphs, outs):
            o.fill_(5.0)
            g.replay()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


_FIRST_CALL = """
import torch
import paper_2510_11958_b200 as pkg
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
q, k, v = (torch.randn(120, h, 64, device="cuda").bfloat16() for h in (4, 2, 2))
kc, vc = (torch.zeros(10, 2, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
lens, n_new, table, free, n_free = ints([0, 0]), ints([119, 1]), ints([[-1] * 8] * 2), torch.arange(10, device="cuda").int(), ints([10])
torch.cuda.synchronize()
def step():
    p = pkg.paged_plan(lens, n_new, table, free, n_free, 16, 120)
    r = pkg.paged_append(q, k, v, p.position, p.slot, kc, vc, rope_theta=1e4)
    return p, r, pkg.paged_attention(r, p.row_start, p.lens, table, kc, vc)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    p, r, out = step()
g.replay()
torch.cuda.synchronize()
assert p.lens.tolist() == [119, 1] and torch.isfinite(out).all()
first = out.clone()
free.copy_(torch.arange(10, device="cuda").int())
p, r, out = step()
assert torch.equal(out, first)
print("fine")
"""


def test_the_first_calls_of_a_process_are_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_CALL], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr


# ---- a decode cycle with cyclical refilling: two plans over two tables

@pytest.mark.parametrize("kv", [BF16, F16])
def test_refill_cycles_over_two_plans(pkg, kv):
    """Lower layers get all tokens of the cycle before at once, upper layers a token a pass: their lengths differ inside a cycle, so that each
    kind has a plan, a table and a pool of its own.  Requests with prompts and cycles of their own; every pass against dense histories in fp64."""
    g = torch.Generator(device="cuda").manual_seed(91)
    B, nq, nkv, D, page, width = 4, 8, 2, 64, 8, 12
    tau, prompt = [3, 1, 4, 2], [40, 1, 17, 8]

    class Stack:
        def __init__(self, n_pages):
            self.lens, self.n_free = ints([0] * B), ints([n_pages])
            self.table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
            self.free = torch.randperm(n_pages, generator=g, device="cuda").int()
            self.kc, self.vc = pool(n_pages, nkv, page, D, kv, "nhd", fill=float("nan"))
            self.past = [[torch.zeros(0, nkv, D, dtype=kv, device="cuda") for _ in range(2)] for _ in range(B)]

        def step(self, new):
            """New rows of every request through one layer: plan, append (no rotation: the history is what was given), attention."""
            T = sum(new)
            q, k, v = (torch.randn(T, h, D, generator=g, device="cuda").to(kv) for h in (nq, nkv, nkv))
            p = pkg.paged_plan(self.lens, ints(new), self.table, self.free, self.n_free, page, T)
            assert p.granted.tolist() == new
            q = pkg.paged_append(q, k, v, p.position, p.slot, self.kc, self.vc)
            out = pkg.paged_attention(q, p.row_start, p.lens, self.table, self.kc, self.vc, max_new=max(new))
            self.lens, self.n_free = p.lens, p.n_free
            at = 0
            for b, n in enumerate(new):
                rows = slice(at, at + n)
                at += n
                self.past[b] = [torch.cat([old, x[rows]]) for old, x in zip(self.past[b], (k, v))]
                kb, vb = (x.double().repeat_interleave(nq // nkv, 1) for x in self.past[b])
                s = torch.einsum("rhd,khd->hrk", q[rows].double(), kb) / math.sqrt(D)
                w = torch.softmax(s + torch.full_like(s, -math.inf).triu(len(kb) - n + 1), -1)
                ref, size = torch.einsum("hrk,khd->rhd", w, vb), torch.einsum("hrk,khd->rhd", w, vb.abs())
                # probabilities and result rounded once each, as in the other tests
                assert ((out[rows].double() - ref).abs() <= half_step(kv) * (size + ref.abs()) + 2e-5 * size + 1e-5).all()
                assert p.lens[b].item() == len(kb)
    lower, upper = Stack(B * width), Stack(B * width)
    pending, done = list(prompt), [0] * B                             # tokens that the lower layers have not seen; passes of the cycle at hand
    for n in range(9):
        full = [done[b] % tau[b] == 0 for b in range(B)]
        lower.step([pending[b] if full[b] else 0 for b in range(B)]) if any(full) else None
        upper.step([prompt[b] if n == 0 else 1 for b in range(B)])    # the whole prompt in the first pass, then the newest token
        pending = [1 if full[b] else pending[b] + 1 for b in range(B)]
        done = [d + 1 for d in done]
        for b in range(B):
            assert upper.lens[b].item() - lower.lens[b].item() == (done[b] - 1) % tau[b]
