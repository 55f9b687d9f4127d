"""The paged cache's calls (dmtd_paged_plan, dmtd_paged_append, dmtd_paged_attention) against their definitions: integers by
a loop over requests, numbers in fp64."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def pkg():
    import paper_2510_11958_b200 as pkg
    pkg.load_library()
    return pkg


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- plan

def plan_reference(lens, n_new, table, stack, n_pages, page, n_rows):
    """The rules of include/dmtd.h, one request after the other."""
    lens, table, stack, width = list(lens), [list(r) for r in table], list(stack), len(table[0])
    for b, n in enumerate(n_new):
        if n < 0:
            stack += [p for p in table[b][:-(-max(0, lens[b]) // page)] if 0 <= p < n_pages]
            lens[b] = 0
    start, granted, position, slot, asked, have = [0], [], [], [], 0, len(stack)
    for b, n in enumerate(n_new):
        ended, n, lens[b] = n < 0, max(0, n), max(0, lens[b])
        held, need = -(-lens[b] // page), -(-(lens[b] + n) // page)
        ok = not ended and need <= width and lens[b] + n <= width * page and start[-1] + n <= n_rows
        if ok:
            asked += need - held
            ok = need == held or asked <= have
        if ok:
            table[b][held:need] = [stack.pop() for _ in range(need - held)]
        for r in range(min(n, n_rows - start[-1])):
            at = lens[b] + r
            here = ok and 0 <= table[b][at // page] < n_pages
            position.append(at if here else 0)
            slot.append(table[b][at // page] * page + at % page if here else -1)
        start.append(min(n_rows, start[-1] + n))
        granted.append(n if ok else 0)
        lens[b] += granted[-1]
    position += [0] * (n_rows - len(position))
    slot += [-1] * (n_rows - len(slot))
    return start, position, slot, granted, lens, [len(stack)], table


def plan_case(seed, B, page, width, most_new, pad, short, ended, holes):
    rng = random.Random(seed)
    lens = [rng.choice([0, rng.randint(0, width * page), rng.randint(0, page)]) for _ in range(B)]
    n_new = [-1 if rng.random() < ended else rng.choice([0, 1, 1, rng.randint(0, most_new)]) for _ in range(B)]
    held = [-(-n // page) for n in lens]
    wanted = sum(max(0, -(-(c + max(0, n)) // page) - h) for c, n, h in zip(lens, n_new, held))
    spare = wanted // 2 if short else wanted + 3
    n_pages = max(1, sum(held) + spare)
    ids = rng.sample(range(n_pages), sum(held) + spare)
    table = [[ids.pop() for _ in range(h)] + [-5] * (width - h) for h in held]
    if holes:
        for row, h in zip(table, held):
            for i in range(h):
                if rng.random() < 0.2:
                    row[i] = rng.choice([-1, n_pages, 1 << 30])
    return lens, n_new, table, ids, n_pages, sum(max(0, n) for n in n_new) + pad


@pytest.mark.parametrize("B,page,width,most_new,pad,short,ended,holes", [
    (1, 16, 1, 1, 0, False, 0.0, False),
    (3, 1, 9, 4, 0, False, 0.0, False),               # a page to a position
    (8, 16, 40, 1, 2, False, 0.0, False),
    (37, 8, 30, 60, 5, False, 0.2, False),
    (37, 8, 30, 60, 5, True, 0.2, True),              # too few pages, and page ids that are none
    (700, 32, 12, 40, 0, True, 0.3, False),           # a cluster: more than 4096 rows
    (1024, 16, 20, 3, 0, False, 0.1, False),          # the last size of one block's one round
    (1025, 16, 20, 3, 1, False, 0.0, False),
    (8192, 4, 16, 9, 100, True, 0.05, True),          # the most requests
    (3000, 16, 20, 40, 7, True, 0.1, True),           # more than 16384 rows: a second launch writes them
])
def test_plan(pkg, B, page, width, most_new, pad, short, ended, holes):
    for seed in range(3):
        lens, n_new, table, stack, n_pages, n_rows = plan_case(seed, B, page, width, most_new, pad, short, ended, holes)
        want = plan_reference(lens, n_new, table, stack, n_pages, page, n_rows)
        free = torch.full((n_pages,), -9, dtype=torch.int32, device="cuda")
        free[:len(stack)] = ints(stack)
        t, n_free, L = ints(table), ints([len(stack)]), ints(lens)
        out = [torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (B + 1, n_rows, n_rows, B)] + [L, n_free]      # in place
        p = pkg.paged_plan(L, ints(n_new), t, free, n_free, page, n_rows, out=out)
        for name, got, ref in zip(p._fields, p, want):
            assert got.tolist() == list(ref), (seed, name)
        assert t.tolist() == want[-1], seed


def test_plan_cuts_off_what_does_not_fit(pkg):
    """Rows beyond n_rows, lengths beyond the table row or below zero, sums beyond 2^31, more free pages than the pool has."""
    page, n_pages = 4, 50
    table = torch.full((5, 3), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(5)
    p = pkg.paged_plan(ints([2, -7, 100, 4, 4]), ints([3, 2, 0, 2 ** 31 - 1, 2 ** 31 - 1]), table, torch.arange(49, -1, -1, device="cuda").int(),
                       ints([1000]), page, 7)
    assert p.row_start.tolist() == [0, 3, 5, 5, 7, 7]
    assert p.granted.tolist() == [3, 2, 0, 0, 0] and p.lens.tolist() == [5, 2, 12, 4, 4]
    # page ids 0, 1, ... from the end of the stack: request 0 gets one page more, request 1 its first
    assert table[0].tolist() == [0, 0, -1] and table[1].tolist() == [1, -1, -1] and p.n_free.item() == 48
    assert p.slot.tolist() == [2, 3, 0, 4, 5, -1, -1] and p.position.tolist() == [2, 3, 4, 0, 1, 0, 0]


def test_plan_without_requests(pkg):
    p = pkg.paged_plan(ints([]), ints([]), torch.zeros(0, 3, dtype=torch.int32, device="cuda"), ints([4, 5, 6]), ints([2]), 16, 3)
    assert p.row_start.tolist() == [0] and p.slot.tolist() == [-1] * 3 and p.position.tolist() == [0] * 3 and p.n_free.item() == 2


# ---- append

def pool(n_pages, nkv, page, D, dtype, layout, fill=0.0):
    """k and v [n_pages, nkv, page, D] in one of several orders in memory."""
    if layout == "hnd":
        a = torch.full((2, n_pages, nkv, page, D), fill, dtype=dtype, device="cuda")
        return a[0], a[1]
    if layout == "nhd":
        a = torch.full((2, n_pages, page, nkv, D), fill, dtype=dtype, device="cuda")
        return a[0].transpose(1, 2), a[1].transpose(1, 2)
    a = torch.full((n_pages, page, nkv, 2, D + 16), fill, dtype=dtype, device="cuda")        # K and V in turn, padded rows
    return a[..., 0, :D].transpose(1, 2), a[..., 1, :D].transpose(1, 2)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("T,nq,nkv,D,act,kv,page,layout,norm,theta", [
    (1, 4, 2, 64, F32, F32, 16, "hnd", True, 1e6),
    (1, 32, 8, 128, BF16, BF16, 1, "nhd", True, 1e6),
    (7, 32, 8, 128, F32, F16, 64, "hnd", True, 1e6),
    (33, 6, 2, 128, F16, F16, 16, "mix", False, 1e4),
    (129, 16, 8, 64, BF16, F32, 8, "mix", True, 0.0),
    (599, 4, 2, 64, F16, BF16, 32, "hnd", True, 1e6),
    (600, 4, 2, 64, F32, BF16, 32, "nhd", True, 1e6),        # the first size of the many-row form
    (1003, 8, 2, 128, BF16, F16, 16, "nhd", False, 0.0),
    (902, 0, 3, 128, F32, F32, 4, "hnd", True, 5e5),         # keys and values only
])
def test_append(pkg, T, nq, nkv, D, act, kv, page, layout, norm, theta):
    g = torch.Generator(device="cuda").manual_seed(T)
    n_pages = -(-(T + 9) // page)
    room = torch.randn(T, (nq + 2 * nkv) * D + 16, generator=g, device="cuda").mul_(3).to(act)
    q, k, v = (t.unflatten(1, (-1, D)) if t.shape[1] else None for t in room[:, :-16].split([nq * D, nkv * D, nkv * D], 1))
    position = torch.randint(0, 1 << 20, (T,), generator=g, device="cuda").int()
    position[0] = 2 ** 31 - 1
    slot = torch.randperm(n_pages * page, generator=g, device="cuda")[:T].int()
    skip = torch.arange(T, device="cuda") % 5 == 3
    slot[skip] = torch.where(torch.arange(int(skip.sum()), device="cuda") % 2 == 0, -1, n_pages * page).int()
    w = [1 + 0.2 * torch.randn(D, generator=g, device="cuda") if norm else None for _ in range(2)]
    kc, vc = pool(n_pages, nkv, page, D, kv, layout, fill=7.0)
    out = None if q is None else torch.full((T, nq, D), 9.0, dtype=act, device="cuda")
    got = pkg.paged_append(q, k, v, position, slot, kc, vc, q_norm=w[0], k_norm=w[1], eps=1e-5, rope_theta=theta, q_out=out)

    def ref(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * w.double()
        if not theta:
            return x
        a = position.double()[:, None, None] * torch.tensor([theta ** (-2 * i / D) for i in range(D // 2)], dtype=torch.float64, device="cuda")
        x0, x1 = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([x0 * a.cos() - x1 * a.sin(), x1 * a.cos() + x0 * a.sin()], -1)

    keep = ~skip

    def check(got, want, dtype):
        # fp32: the norm's sum, root and two products 4e-7 of the pair's size; the angle's fraction of a turn is rounded to
        # 2^-25, 2e-7 radians; cosine and sine 1e-7.  The 64-bit angle: a turn's fraction is off by 2^31 * 2^-52.  Then one rounding.
        size = want.abs().amax(-1, keepdim=True)
        assert ((got.double() - want).abs() <= half_step(dtype) * want.abs() + 2e-6 * size + 1e-7).all()

    if q is not None:
        check(got[keep], ref(q, w[0])[keep], act)
        assert (got[skip] == 9.0).all()
    want_k, want_v = (torch.full((n_pages, nkv, page, D), 7.0, dtype=torch.float64, device="cuda") for _ in range(2))
    s = slot[keep].long()
    want_k[s // page, :, s % page] = ref(k, w[1])[keep]
    want_v[s // page, :, s % page] = v[keep].double()
    check(kc, want_k, kv)
    assert ((vc.double() - want_v).abs() <= half_step(kv) * want_v.abs() + (2 ** -25 if kv == F16 else 0)).all()


def test_append_in_place(pkg):
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(20, h, 128, generator=g, device="cuda") for h in (8, 2, 2))
    kc, vc = pool(2, 2, 16, 128, F32, "hnd")
    pos = torch.arange(20, device="cuda").int()
    want = pkg.paged_append(q, k, v, pos, pos, kc, vc, rope_theta=1e4)
    assert pkg.paged_append(q, k, v, pos, pos, kc, vc, rope_theta=1e4, q_out=q) is q and torch.equal(q, want)


# ---- attention

def attention_reference(q, row_start, lens, table, kc, vc, out):
    """fp64; out: what rows of no request hold.  Also sum p |v| / sum p, which bounds what roundings of the probabilities move."""
    nq, D, nkv, page = q.shape[1], q.shape[2], kc.shape[1], kc.shape[2]
    ref, size = out.double().clone(), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(lens):
        t0, t1 = row_start[b], row_start[b + 1]
        if t1 == t0:
            continue
        ids = table[b].long()
        good = ((ids >= 0) & (ids < kc.shape[0])).repeat_interleave(page)[:length]
        ids = ids.clamp(0, kc.shape[0] - 1)
        k, v = (c[ids].transpose(1, 2).reshape(-1, nkv, D)[:length].double() for c in (kc, vc))
        last = length - (t1 - t0) + torch.arange(t1 - t0, device="cuda")
        seen = good[None] & (torch.arange(length, device="cuda")[None] <= last[:, None])
        for h in range(nkv):
            g = slice(h * (nq // nkv), (h + 1) * (nq // nkv))
            s = torch.einsum("rgd,kd->grk", q[t0:t1, g].double(), k[:, h]) / math.sqrt(D)
            s = torch.where(seen, s, -math.inf)
            m = s.amax(-1, keepdim=True) if length else s.new_zeros(s.shape[:2] + (1,))
            p = torch.where(seen & (s != -math.inf), torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
            total = p.sum(-1, keepdim=True)
            p = torch.where(total == 0, 0.0, p / total)
            any_row = seen.any(0)                                     # what no row sees has no influence
            vh = torch.where(any_row[:, None], v[:, h], 0.0)
            if torch.isfinite(vh).all():
                ref[t0:t1, g] = torch.einsum("grk,kd->rgd", p, vh)
                size[t0:t1, g] = torch.einsum("grk,kd->rgd", p, vh.abs())
            else:                                                     # row by row: keys that a row does not see are not multiplied
                for r in range(t1 - t0):
                    on = seen[r]
                    ref[t0 + r, g] = p[:, r, on] @ vh[on]
                    size[t0 + r, g] = p[:, r, on] @ vh[on].abs()
    return ref, size


def attention_case(seed, cached, new, nq, nkv, D, qt, kv, page, layout, pad=0, stale=float("nan"), q_room=0, scale=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens = [c + n for c, n in zip(cached, new)]
    held = [-(-n // page) for n in lens]
    n_pages = sum(held) + 2
    ids = torch.randperm(n_pages, generator=g, device="cuda").int()
    width = max(max(held), 1) + 1
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    kc, vc = pool(n_pages, nkv, page, D, kv, layout, fill=stale)     # rows behind the last key hold something else
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
        rows = torch.arange(lens[b], device="cuda")
        for c in (kc, vc):
            c[table[b].long()[rows // page], :, rows % page] = torch.randn(lens[b], nkv, D, generator=g, device="cuda").to(kv)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    T = start[-1] + pad
    q = (scale * torch.randn(T, nq * D + q_room, generator=g, device="cuda")).to(qt)[:, :nq * D].unflatten(1, (nq, D))
    out = torch.full((T, nq, D), 5.0, dtype=qt, device="cuda")
    return dict(q=q, start=start, lens=lens, table=table, kc=kc, vc=vc, out=out)


def check_attention(pkg, c, max_new=0, finite=True):
    ref, size = attention_reference(c["q"], c["start"], c["lens"], c["table"], c["kc"], c["vc"], c["out"])
    got = pkg.paged_attention(c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"], max_new=max_new, out=c["out"].clone())
    qt, kv, D = c["q"].dtype, c["kc"].dtype, c["q"].shape[2]
    n = max(c["lens"] + [1])
    v_max = torch.nan_to_num(c["vc"].float(), 0, 0, 0).abs().max().item()
    # fp32: scores of size up to 16 to 2^-20 of it (the parts of q and the sums), the exponential's argument to as much: 2e-5 of
    # sum p |v|.  16-bit queries: the probabilities are rounded once (half a step of sum p |v|; fp16 below 2^-14 of the tile's
    # largest to 2^-25, keys as many as there are), the result once.
    tol = 2e-5 * size + 1e-6 * v_max
    if qt != F32:
        tol = tol + half_step(qt) * (size + ref.abs()) + (n * 2.0 ** -25 * v_max + 2.0 ** -25 if qt == F16 else 0)
    bad = ~((got.double() - ref).abs() <= tol)
    bad &= ~(torch.isnan(ref) & torch.isnan(got.double())) & ~(ref == got.double())
    assert not bad.any(), (int(bad.sum()), (got.double() - ref)[bad].abs().max().item(), bad.nonzero()[0].tolist())
    if finite:
        assert torch.isfinite(got).all()
    return got


TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("nq,nkv,D,page,layout,cached,new", [
    (4, 2, 64, 16, "hnd", [0], [1]),                                     # one key
    (32, 8, 128, 16, "nhd", [999], [1]),
    (8, 2, 128, 1, "mix", [37, 0, 5], [1, 3, 0]),                        # a page to a position; a request that waits
    (8, 8, 128, 4, "hnd", [63, 64, 65, 15, 16, 17, 0], [1, 1, 1, 1, 1, 1, 1]),
    (16, 1, 128, 32, "nhd", [4100], [1]),                                # one item, many pieces
    (32, 8, 128, 64, "hnd", [700, 20, 333, 0, 129], [3, 3, 1, 3, 2]),    # refill rows
    (6, 2, 64, 8, "mix", [70, 300], [5, 11]),                            # three heads to a group
    (8, 2, 128, 16, "hnd", [0, 100, 250], [130, 33, 17]),                # pieces of prompts
    (16, 8, 64, 128, "nhd", [0, 640], [257, 1]),
    (32, 2, 128, 16, "hnd", [40, 0, 9], [1, 70, 2]),                     # 16 heads to a group
    (32, 8, 128, 16, "hnd", [3000], [700]),                              # items cut where one half of their rows sees no more keys
    (16, 8, 64, 64, "nhd", [1500, 2100, 0], [300, 211, 190]),
])
def test_attention(pkg, qt, kv, nq, nkv, D, page, layout, cached, new):
    c = attention_case(1, cached, new, nq, nkv, D, qt, kv, page, layout, pad=3, q_room=16)
    a = check_attention(pkg, c)
    check_attention(pkg, c, max_new=max(new))
    assert (a[-3:] == 5.0).all()
    # the same call gives the same bits
    assert torch.equal(a, check_attention(pkg, c))


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("seed", range(4))
def test_attention_drawn(pkg, qt, kv, seed):
    rng = random.Random(seed * 10 + TYPES.index((qt, kv)))
    for _ in range(3):
        B = rng.choice([1, 2, 9, 40])
        nq, nkv = rng.choice([(4, 2), (8, 8), (32, 8), (15, 5), (16, 2)])
        cached = [rng.choice([0, rng.randint(0, 40), rng.randint(0, 1500)]) for _ in range(B)]
        new = [rng.choice([0, 1, 1, 2, rng.randint(1, 20)]) for _ in range(B)]
        if rng.random() < 0.5:
            new[rng.randrange(B)] = rng.randint(100, 400)
        c = attention_case(seed, cached, new, nq, nkv, rng.choice([64, 128]), qt, kv, rng.choice([1, 2, 16, 64, 512]), rng.choice(["hnd", "nhd", "mix"]),
                           pad=rng.choice([0, 2]))
        check_attention(pkg, c, max_new=rng.choice([0, max(new), 1]))          # (a wrong max_new costs time, not results)


@pytest.mark.parametrize("qt,kv", TYPES)
def test_pages_outside_the_pool_take_their_keys_out(pkg, qt, kv):
    c = attention_case(2, [200, 50, 90, 700], [2, 1, 30, 4], 8, 2, 128, qt, kv, 16, "hnd")
    n_pages = c["kc"].shape[0]
    c["table"][0, 3:6] = -1                                              # a window has left these behind
    c["table"][0, 0] = n_pages
    c["table"][1, :] = -1                                                # none left: zeros
    c["table"][2, 1] = 2 ** 31 - 1
    c["table"][3, :] = -2 ** 31
    got = check_attention(pkg, c)
    assert (got[2] == 0).all() and (got[-4:] == 0).all()


@pytest.mark.parametrize("qt,kv", TYPES)
def test_rows_that_see_no_key(pkg, qt, kv):
    """Fewer keys than rows: the first rows sit in front of position 0.  And offsets, lengths that do not fit the buffers."""
    c = attention_case(3, [0, 0, 30], [6, 3, 2], 8, 2, 128, qt, kv, 4, "nhd")
    c["lens"] = [4, 0, 32]
    got = check_attention(pkg, c)
    assert (got[:2] == 0).all() and (got[6:9] == 0).all() and not (got[2:6] == 0).all()
    n = c["table"].shape[1] * 4
    cut = dict(c, lens=[4, 0, n])
    want = pkg.paged_attention(c["q"], ints(c["start"]), ints(cut["lens"]), c["table"], c["kc"], c["vc"], out=c["out"].clone())
    wild = pkg.paged_attention(c["q"], ints([-5] + c["start"][1:-1] + [2 ** 31 - 1]), ints([4, -3, 2 ** 31 - 1]), c["table"], c["kc"], c["vc"],
                               out=c["out"].clone())
    assert torch.equal(want, wild)


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("new", [3, 40, 200])
def test_values_that_a_row_does_not_see(pkg, qt, kv, new):
    """Infinities and NaN in keys and values of later positions of the same chunk."""
    c = attention_case(4, [70, 5], [new, 1], 8, 2, 128, qt, kv, 16, "hnd")
    for row, c_k, c_v in ((new - 1, float("nan"), float("nan")), (new // 2, 1.0, float("inf")), (new // 3, -1.0, float("-inf"))):
        at = 70 + row
        page, i = c["table"][0, at // 16].long(), at % 16
        c["kc"][page, :, i] = c_k
        c["vc"][page, :, i, 3:60] = c_v
    got = check_attention(pkg, c, finite=False)
    assert torch.isfinite(got[:new // 3]).all() and torch.isfinite(got[new]).all()
    assert torch.isnan(got[new - 1]).any()


@pytest.mark.parametrize("qt,kv", TYPES)
@pytest.mark.parametrize("cached,new", [([200, 900, 17], [1, 1, 1]), ([100, 3000, 40], [2, 1, 40])])
def test_infinities_in_sight(pkg, qt, kv, cached, new):
    """An infinite value gives infinite results, a score of minus infinity takes its key out: in tiles of one row as in others."""
    c = attention_case(14, cached, new, 8, 2, 128, qt, kv, 16, "hnd")
    c["q"][:, :, 0] = c["q"][:, :, 0].abs() + 0.25
    for b in range(3):
        page = c["table"][b, 0].long()
        c["vc"][page, :, 5, 3:60] = math.inf
        c["vc"][page, :, 5, 60:70] = -math.inf
        c["kc"][page, :, 9, 0] = -math.inf
    got = check_attention(pkg, c, finite=False)
    assert (got[:, :, 3:60] == math.inf).all() and (got[:, :, 60:70] == -math.inf).all()
    assert torch.isfinite(got[:, :, :3]).all() and torch.isfinite(got[:, :, 70:]).all()


@pytest.mark.parametrize("qt,kv", TYPES)
def test_scores_far_apart(pkg, qt, kv):
    """One key outweighs all others by far, early or late; equal scores; large ones."""
    c = attention_case(5, [300, 300, 300, 0], [1, 4, 20, 64], 8, 2, 64, qt, kv, 16, "nhd", scale=1.0)
    c["q"][:, :, 0] = 8.0
    for b, at in ((0, 3), (1, 299), (2, 150)):
        c["kc"][c["table"][b, at // 16].long(), :, at % 16, 0] = 60.0      # 60 above the rest
    c["kc"][c["table"][3, 0].long(), :, :, :] = 0.0
    check_attention(pkg, c)


@pytest.mark.parametrize("kv", [F32, BF16, F16])
@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e4, 3e5])
def test_queries_of_any_size(pkg, kv, size):
    """fp32 queries far outside fp16's range (and its precision): scores stay moderate through small or large keys."""
    new = 9
    c = attention_case(11, [200], [new], 8, 2, 64, F32, kv, 16, "hnd")
    c["q"] *= size / 1.5
    c["q"][4:, :, 5:] = 0.0
    if size > 1:
        c["kc"][:] = (c["kc"].float() * min(1.0, 4.0 / size)).to(kv)
    ref, spread = attention_reference(c["q"], c["start"], c["lens"], c["table"], c["kc"], c["vc"], c["out"])
    got = pkg.paged_attention(c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"])
    # (no further than the other tests: the parts are relative to the row's largest value)
    assert ((got.double() - ref).abs() <= 2e-5 * spread + 1e-5).all()


@pytest.mark.parametrize("nkv,pages,pad", [(2, None, 8), (2, None, 64 * 16 * 3), (1, None, 8), (2, 1, 8), (1, 1, 0)])
def test_pages_apart(pkg, nkv, pages, pad):
    """Pages with room between them, a whole number of heads or not; one kv head, one page."""
    page, D = (16, 64) if pages is None else (512, 64)
    cached, new = ([300, 5], [150, 70]) if pages is None else ([200], [150])
    c = attention_case(18, cached, new, 4, nkv, D, BF16, BF16, page, "hnd")
    if pages == 1:                                                       # the pool is the request's only page
        at = c["table"][0, 0].long()
        c["kc"], c["vc"], c["table"] = c["kc"][at:at + 1], c["vc"][at:at + 1], torch.zeros_like(c["table"])
        c["table"][:, 1:] = -1
    for name in ("kc", "vc"):
        t = c[name]
        apart = torch.full((t.shape[0], nkv * page * D + pad), float("nan"), dtype=BF16, device="cuda")
        c[name] = apart[:, :nkv * page * D].unflatten(1, (nkv, page, D))
        c[name].copy_(t)
    check_attention(pkg, c)


@pytest.mark.parametrize("qt,kv", [(F32, F16), (BF16, BF16)])
@pytest.mark.parametrize("B", [257, 700])
def test_more_requests_than_are_kept(pkg, qt, kv, B):
    """Batches whose requests do not fit shared memory; pieces of prompts far behind the first requests."""
    rng = random.Random(B)
    cached = [rng.choice([0, rng.randint(0, 30), rng.randint(0, 200)]) for _ in range(B)]
    new = [rng.choice([0, 1, 1, 2]) for _ in range(B)]
    for b in (B - 1, B // 2, 70):
        new[b] = 90
    c = attention_case(12, cached, new, 4, 2, 64, qt, kv, 16, "hnd", pad=1)
    check_attention(pkg, c)


def test_tables_of_the_largest_kind(pkg):
    """A request near the end of the plan's and the attention's ranges: positions around 2^20 in a sparse table."""
    page, n = 1024, 1 << 20
    kc, vc = pool(3, 1, page, 64, BF16, "hnd")
    g = torch.Generator(device="cuda").manual_seed(13)
    for t in (kc, vc):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    table = torch.full((1, n // page), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, 700], table[0, -1] = 2, 0, 1               # all others have been dropped
    for new in (1, 200):
        q = torch.randn(new, 2, 64, generator=g, device="cuda").to(BF16)
        c = dict(q=q, start=[0, new], lens=[n], table=table, kc=kc, vc=vc, out=torch.zeros_like(q))
        check_attention(pkg, c)


@pytest.mark.parametrize("kv", [BF16, F32])
def test_offsets_beyond_32_bits(pkg, kv):
    """A pool of more than 2^32 bytes and 2^31 values, keys at both ends."""
    nkv, page, D = 8, 128, 128
    per_page = nkv * page * D
    n_pages = (2 ** 31 + 2 ** 28) // per_page
    kc, vc = (torch.empty(n_pages, nkv, page, D, dtype=kv, device="cuda") for _ in range(2))
    ids = [0, n_pages - 1, n_pages // 2, n_pages - 2]
    g = torch.Generator(device="cuda").manual_seed(6)
    for t in (kc, vc):
        for i in ids:
            t[i] = torch.randn(nkv, page, D, generator=g, device="cuda").to(kv)
    table = ints([ids])
    for new in (1, 150):
        q = torch.randn(new, 32, D, generator=g, device="cuda").to(kv)
        lens, start = [500], [0, new]
        got = pkg.paged_attention(q, ints(start), ints(lens), table, kc, vc)
        small = pkg.paged_attention(q, ints(start), ints(lens), ints([[0, 1, 2, 3]]), kc[ids], vc[ids])
        assert torch.equal(got, small)
    k, v = (torch.randn(3, nkv, D, generator=g, device="cuda").to(kv) for _ in range(2))
    slot = ints([0, n_pages * page - 1, n_pages * page // 2 + 5])
    pkg.paged_append(None, k, v, ints([0, 0, 0]), slot, kc, vc)
    s = slot.long()
    assert torch.equal(kc[s // page, :, s % page], k) and torch.equal(vc[s // page, :, s % page], v)


# ---- a run of all three, as a server makes it

@pytest.mark.parametrize("D,nq,nkv,act,kv", [(128, 8, 2, F32, F16), (64, 4, 2, F32, F32), (128, 8, 2, BF16, BF16)])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_a_server(pkg, D, nq, nkv, act, kv, graph):
    """Requests come, refill, wait and end over 12 steps; every step's attention against a dense history in fp64.  With `graph`
    one captured step serves all of them: lengths, tables and the pool live on the device."""
    rng = random.Random(17)
    g = torch.Generator(device="cuda").manual_seed(7)
    B, page, width, n_pages, n_rows = 5, 8, 12, 14, 64
    lens, n_new = ints([0] * B), ints([0] * B)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    free, n_free = torch.arange(n_pages, device="cuda").int(), ints([n_pages])
    kc, vc = pool(n_pages, nkv, page, D, kv, "nhd", fill=float("nan"))
    norm = [1 + 0.1 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
    qkv = torch.zeros(n_rows, (nq + 2 * nkv) * D, dtype=act, device="cuda")
    q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([nq * D, nkv * D, nkv * D], 1))
    plan = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B + 1, n_rows, n_rows, B)] + [lens, n_free]
    q_rot, out = torch.zeros(n_rows, nq, D, dtype=act, device="cuda"), torch.zeros(n_rows, nq, D, dtype=act, device="cuda")
    scratch = torch.empty(48 << 20, dtype=torch.uint8, device="cuda")

    def step():
        p = pkg.paged_plan(lens, n_new, table, free, n_free, page, n_rows, out=plan)
        pkg.paged_append(q, k, v, p.position, p.slot, kc, vc, q_norm=norm[0], k_norm=norm[1], rope_theta=1e4, q_out=q_rot)
        pkg.paged_attention(q_rot, p.row_start, p.lens, table, kc, vc, scratch=scratch, out=out)

    replay = step
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()                                           # (nothing new: changes nothing)
        torch.cuda.current_stream().wait_stream(side)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        replay = captured.replay
    history = [[] for _ in range(B)]
    refused = 0
    for i in range(12):
        todo = [rng.choice([0, 1, 3, 3, rng.randint(1, 25)]) for _ in range(B)]
        for b in range(B):
            if history[b] and rng.random() < 0.15:
                todo[b] = -1
        while sum(max(0, n) for n in todo) > n_rows:
            todo[todo.index(max(todo))] //= 2
        n_new.copy_(ints(todo))
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda").to(act))
        out.fill_(3.0)
        replay()
        start, granted = plan[0].tolist(), plan[3].tolist()
        for b in range(B):
            if todo[b] < 0:
                history[b] = []
            n, t0 = granted[b], start[b]
            refused += max(0, todo[b]) - n
            history[b] += list(range(n))
            assert lens[b].item() == len(history[b])
        held = sum(-(-len(h) // page) for h in history)
        assert n_free.item() == n_pages - held
        live = [p for b, h in enumerate(history) for p in table[b, :-(-len(h) // page)].tolist()]
        assert sorted(live + free[:n_free.item()].tolist()) == list(range(n_pages))      # every page once
        # rows of refused requests do not count
        ok = [granted[b] == max(0, todo[b]) for b in range(B)]
        c = dict(q=q_rot, start=start, lens=lens.tolist(), table=table, kc=kc, vc=vc, out=torch.full_like(out, 3.0))
        rows = torch.zeros(n_rows, dtype=torch.bool, device="cuda")
        for b in range(B):
            rows[start[b]:start[b + 1]] = ok[b]
        rows[start[-1]:] = True
        ref, size = attention_reference(c["q"], start, c["lens"], table, kc, vc, c["out"])
        u = 2e-5 if act == F32 else 2e-5 + half_step(act)
        tol = u * size + (half_step(act) * ref.abs() if act != F32 else 0) + 1e-5
        assert ((out.double() - ref).abs() <= tol)[rows].all(), i
    assert refused > 0                                       # the pool ran short on the way


def test_on_another_stream(pkg):
    c = attention_case(8, [500, 3], [2, 60], 8, 2, 128, BF16, BF16, 16, "hnd")
    want = check_attention(pkg, c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = pkg.paged_attention(c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"], out=c["out"].clone())
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def _three_cases():
    return [attention_case(15, [900, 4], [200, 1], 8, 2, 128, BF16, BF16, 16, "hnd"), attention_case(16, [2500, 80, 7], [1, 3, 2], 16, 2, 64, F32, F16, 4, "nhd"),
            attention_case(17, [0, 1300, 60], [90, 1, 40], 8, 8, 64, F16, F16, 32, "mix")]


def _args(c):
    return c["q"], ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"]


@pytest.mark.parametrize("graph", [False, True])
def test_calls_in_a_row_share_scratch(pkg, graph):
    """Each call's first kernel starts under the last one's end: partial results of the call in front must be read by then."""
    cases = _three_cases()
    args, want = [_args(c) for c in cases], [check_attention(pkg, c) for c in cases]
    scratch = torch.empty(pkg.PAGED_ATTENTION_SCRATCH_BYTES, dtype=torch.uint8, device="cuda")
    order = [random.Random(1).randrange(3) for _ in range(40)]
    outs = [cases[i]["out"].clone() for i in order]

    def calls():
        for i, out in zip(order, outs):
            pkg.paged_attention(*args[i], scratch=scratch, out=out)
    if graph:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls()
        for _ in range(3):
            g.replay()
    else:
        calls()
    for i, out in zip(order, outs):
        assert torch.equal(out, want[i])


def test_two_streams_at_once(pkg):
    """Calls with scratch of their own run side by side."""
    cases = _three_cases()
    args, want = [_args(c) for c in cases], [check_attention(pkg, c) for c in cases]
    outs = [[c["out"].clone() for _ in range(30)] for c in cases]
    scratch = [torch.empty(pkg.PAGED_ATTENTION_SCRATCH_BYTES, dtype=torch.uint8, device="cuda") for _ in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for n in range(30):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                pkg.paged_attention(*args[i], scratch=scratch[i], out=outs[i][n])
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(x, w) for x in o)


def test_against_the_contiguous_cache(pkg):
    """Equal lengths: what dmtd_attention_decode gives for the same keys in one piece."""
    B, R, nq, nkv, D, n, page = 3, 3, 8, 2, 128, 400, 16
    c = attention_case(9, [n - R] * B, [R] * B, nq, nkv, D, F32, F16, page, "hnd")
    k, v = (torch.stack([t[c["table"][b, :n // page].long()].transpose(0, 1).reshape(nkv, n, D) for b in range(B)]).contiguous()
            for t in (c["kc"], c["vc"]))
    want = pkg.attention_decode(c["q"].reshape(B, R, nq, D).contiguous(), k, v, n - R)
    got = check_attention(pkg, c).view(B, R, nq, D)
    # that call rounds queries and probabilities to fp16
    assert (got - want).abs().max() <= 4 * 2.0 ** -12 * max(1.0, want.abs().max().item())


def test_tensors_of_the_wrong_kind_are_refused(pkg):
    c = attention_case(10, [20], [2], 8, 2, 64, BF16, BF16, 16, "hnd")
    start, lens, table, kc, vc, q = ints(c["start"]), ints(c["lens"]), c["table"], c["kc"], c["vc"], c["q"]
    for args in ((q.double(), start, lens, table, kc, vc), (q, start.long(), lens, table, kc, vc), (q, start, lens, table[0], kc, vc),
                 (q, start[:1], lens, table, kc, vc), (q, start, lens, table, kc, vc[:1]), (q, start, lens, table, kc, vc.float()),
                 (q.transpose(0, 1), start, lens, table, kc, vc), (q[..., :32], start, lens, table, kc, vc),
                 (q, start, lens, torch.zeros(2, 4, dtype=torch.int32, device="cuda").t()[:1], kc, vc)):
        with pytest.raises(ValueError):
            pkg.paged_attention(*args)
    with pytest.raises(ValueError):
        pkg.paged_attention(q, start, lens, table, kc, vc, out=torch.empty(2, 8, 64, device="cuda"))
    with pytest.raises(pkg.DmtdError) as e:
        pkg.paged_attention(q, start, lens, table, kc, vc, scratch=torch.empty(1 << 20, device="cuda"))
    assert "scratch" in str(e.value)
    k = torch.zeros(2, 2, 64, device="cuda")
    pos = ints([0, 1])
    for args, kw in (((None, k, k.half(), pos, pos, kc, vc), {}), ((None, k, k, pos.long(), pos, kc, vc), {}), ((None, k[:, :1], k[:, :1], pos, pos, kc, vc), {}),
                     ((None, k, k, pos, pos, kc, vc), {"k_norm": torch.ones(32, device="cuda")}),
                     ((k, k, k, pos, pos, kc, vc), {"q_out": k.half()}), ((None, k, k, pos[:1], pos, kc, vc), {})):
        with pytest.raises(ValueError):
            pkg.paged_append(*args, **kw)
    i = ints([0, 0])
    with pytest.raises(ValueError):
        pkg.paged_plan(i, ints([0]), table.repeat(2, 1), i, ints([1]), 16, 4)
    with pytest.raises(ValueError):
        pkg.paged_plan(i, i, table.repeat(2, 1), i, ints([1]), 16, 4, out=[i] * 6)
