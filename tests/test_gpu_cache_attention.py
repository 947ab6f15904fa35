"""Attention over the paged cache against its plain form in 64 bits."""
import random

import pytest
import torch

import _cache_ref as plain
from paper_2607_27744_b200 import binding as rocs

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def build(dtype, counts, lens, Hkv, G, dh, page, seed=0, order="tokens", std=1.5, spare=3):
    """A pool with the slots' pages in random places and NaN in every row that nobody holds."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    R = len(lens)
    n_pages = sum(-(-l // page) for l in lens) + spare
    width = max(1, max(-(-l // page) for l in lens)) + 1
    if order == "tokens":
        K, V = (torch.randn((n_pages, page, Hkv, dh), generator=g, device="cuda").to(dtype) for _ in range(2))
    elif order == "heads":   # [n_pages, H_kv, page, dh] in memory
        K, V = (torch.randn((n_pages, Hkv, page, dh), generator=g, device="cuda").to(dtype).transpose(1, 2) for _ in range(2))
    else:                    # keys and values of a page side by side
        both = torch.randn((n_pages, 2, page, Hkv, dh), generator=g, device="cuda").to(dtype)
        K, V = both[:, 0], both[:, 1]
    ids = list(range(n_pages))
    rng.shuffle(ids)
    slots = list(range(R + 2))
    rng.shuffle(slots)
    slots = slots[:R]
    table = torch.full((R + 2, width), -7, dtype=torch.int32)
    ln = torch.zeros(R + 2, dtype=torch.int32)
    held = torch.zeros((n_pages, page), dtype=torch.bool)
    for r, L in enumerate(lens):
        ln[slots[r]] = L
        for p in range(-(-L // page)):
            id = ids.pop()
            table[slots[r], p] = id
            held[id, :min(page, L - p * page)] = True
    K[~held.cuda()] = float("nan")
    V[~held.cuda()] = float("nan")
    off = [0]
    for c in counts:
        off.append(off[-1] + c)
    Q = (torch.randn((off[-1], Hkv * G, dh), generator=g, device="cuda") * std).to(dtype)
    offsets = torch.tensor(off, dtype=torch.int32)
    return {"K": K, "V": V, "table": table.cuda(), "lens": ln.cuda(), "slots": torch.tensor(slots, dtype=torch.int32).cuda(),
            "offsets": off, "plan": rocs.plan_create(offsets.cuda(), offsets), "Q": Q, "page": page}


def bound(dtype, O, A, S, L, dh):
    """How far a result may be off, element by element.  A: sum p |v|, S: the largest sum |q||k| scale of the row.
    fp32: a score is a sum of dh products (dh half steps of S), times a rounded scale, through tanh, exp and a distance
    (16 more); a probability is off by twice that relatively (its own and the sum's); the sums over L keys add L half steps.
    bf16: the same, plus half a step of each probability as the product's operand, and of the result."""
    e = 2.0 ** -24
    off = A * (2 * e * ((dh + 16) * S + 16) + (L + 16) * e)
    if dtype is BF16:
        off = off + 2.0 ** -8 * A + 2.0 ** -8 * (O.abs() + off)
    return off + 1e-30


def check(case, out=None, tol=1.0, **how):
    dtype = case["K"].dtype
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    got = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], out=out, **how)
    O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist(),
                              **{k: v for k, v in how.items() if k != "scale" or v > 0})
    L = int(case["lens"].max())
    off = (got.double() - O).abs()
    most = bound(dtype, O, A, S, L, case["K"].shape[-1])
    rocs.last_device_status()
    assert torch.isfinite(got).all(), "non-finite values"
    assert bool((off <= most).all()), f"off by {float((off / most).max()):.3f} of the bound"
    return got


def slopes(H):
    return 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hkv,G,dh,page", [(2, 1, 64, 16), (1, 8, 128, 64), (2, 4, 64, 32), (3, 5, 32, 24), (1, 3, 128, 128), (2, 2, 80, 7),
                                           (1, 1, 256, 16), (1, 17, 64, 8), (1, 40, 32, 16), (2, 2, 128, 256)])
def test_one_event_per_request(dtype, Hkv, G, dh, page):
    lens = [1, 2, page, page + 1, 31, 33, 64, 65, 300, 1025, 0]
    check(build(dtype, [1] * len(lens), lens, Hkv, G, dh, page, seed=page))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hkv,G,dh,page", [(2, 1, 64, 16), (1, 4, 128, 64), (2, 3, 64, 32), (1, 2, 32, 24), (1, 1, 128, 128), (1, 2, 96, 10),
                                           (2, 8, 128, 16)])
def test_chunks_of_any_length(dtype, Hkv, G, dh, page):
    counts = [1, 0, 5, 17, 64, 3, 129, 200, 2]
    lens = [1, 50, 5, 400, 64, 0, 130, 777, 1]   # the sixth: rows of a slot that holds nothing; the last: more rows than keys
    check(build(dtype, counts, lens, Hkv, G, dh, page, seed=1))


@pytest.mark.parametrize("dtype,dh,n,L", [(BF16, 128, 700, 700), (BF16, 64, 1300, 1500), (F32, 64, 150, 400), (BF16, 128, 300, 5000)])
def test_whole_histories(dtype, dh, n, L):
    check(build(dtype, [n, 1, n // 3], [L, L // 2, L // 3], 1, 2, dh, 32, seed=2))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("counts,lens,Hkv,G,dh,page", [([300, 1, 0, 40, 129], [500, 64, 10, 0, 129], 2, 1, 64, 64),
                                                       ([100, 260], [333, 50], 1, 2, 128, 16), ([7, 90], [90, 2], 2, 2, 32, 8)])
def test_candidates_see_everything(dtype, counts, lens, Hkv, G, dh, page):
    check(build(dtype, counts, lens, Hkv, G, dh, page, seed=3), causal=False)


# capped scores, distances, documents, prefixes, alone and together; rows that see nothing among them
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh,G", [(64, 1), (128, 4), (48, 2)])
@pytest.mark.parametrize("cap,bias,doc,pre,causal", [(5.0, False, 0, 0, True), (0.0, True, 0, 0, True), (0.0, False, 37, 0, True),
                                                     (0.0, False, 0, 90, True), (2.0, True, 100, 60, True), (0.0, True, 9, 0, False),
                                                     (30.0, True, 0, 0, False)])
@pytest.mark.parametrize("counts", [[1, 1, 2, 1, 1], [70, 300, 3, 150, 1]])
def test_scores_and_masks(dtype, dh, G, cap, bias, doc, pre, causal, counts):
    lens = [200, 450, 77, 150, 600]
    case = build(dtype, counts, lens, 2, G, dh, 16, seed=4)
    how = {"causal": causal, "cap": cap}
    H = 2 * G
    if bias:
        how["slopes"] = slopes(H)
    if doc:
        begin = []
        for n, L in zip(counts, lens):
            begin += [(L - n + t) // doc * doc for t in range(n)]
        begin = torch.tensor(begin, dtype=torch.int32)
        begin[::7] = 100000            # sees nothing
        begin[3::11] = -5              # as 0
        how["begin"] = begin.cuda()
    if pre:
        how["prefix"] = torch.tensor([pre, 0, 1000, -3, pre // 2], dtype=torch.int32).cuda()
    got = check(case, **how)
    if doc:
        assert torch.all(got[how["begin"] >= 100000] == 0)


@pytest.mark.parametrize("order", ["heads", "both"])
@pytest.mark.parametrize("dtype,dh,counts", [(BF16, 64, [1, 1, 1]), (BF16, 128, [200, 3, 64]), (F32, 64, [20, 1, 5])])
def test_orders_of_the_pages_and_strided_rows(order, dtype, dh, counts):
    lens = [300, 64, 190]
    case = build(dtype, counts, lens, 2, 2, dh, 32, seed=5, order=order)
    N, H = case["Q"].shape[:2]
    wide = torch.randn((N, H + 4, dh), device="cuda").to(dtype)   # queries as a slice of a fused projection
    wide[:, 2:2 + H] = case["Q"]
    case["Q"] = wide[:, 2:2 + H]
    room = torch.full((N + 2, H + 1, dh + 8), 9.0, device="cuda", dtype=dtype)
    check(case, out=room[1:N + 1, 1:, :dh])
    assert torch.all(room[0] == 9) and torch.all(room[N + 1] == 9) and torch.all(room[:, 0] == 9) and torch.all(room[:, :, dh:] == 9)


@pytest.mark.parametrize("dtype,dh,counts", [(BF16, 64, [1, 1, 1]), (BF16, 128, [200, 3, 64]), (BF16, 64, [70, 33, 300]), (F32, 64, [20, 1, 5])])
@pytest.mark.parametrize("over", ["rows", "heads", "both"])
def test_queries_broadcast(dtype, dh, counts, over):
    case = build(dtype, counts, [700, 100, 513], 2, 2, dh, 16, seed=21)
    Q = case["Q"]
    part = Q[:1 if over != "heads" else None, :1 if over != "rows" else None]
    case["Q"] = part.expand_as(Q)
    check(case)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,dh,counts", [(BF16, 64, [3, 1, 16]), (BF16, 128, [130, 40, 300]), (BF16, 64, [70, 300, 20]), (F32, 64, [30, 1, 9]),
                                             (BF16, 32, [40, 9, 30])])
def test_keys_that_a_row_does_not_see_may_hold_anything(value, dtype, dh, counts):
    lens = [400, 350, 500]
    case = build(dtype, counts, lens, 2, 2, dh, 16, seed=6)
    # the last event of every request is broken: all earlier rows are as if it were not there
    for r, L in enumerate(lens):
        s = int(case["slots"][r])
        id, at = int(case["table"][s, (L - 1) // 16]), (L - 1) % 16
        case["K"][id, at] = value
        case["V"][id, at] = value
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    got = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"])
    O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist())
    last = torch.zeros(got.shape[0], dtype=torch.bool)
    last[[o - 1 for o in case["offsets"][1:]]] = True
    assert torch.isfinite(got[~last.cuda()]).all()
    rows = (~last).cuda()
    clean_S = torch.nan_to_num(S, nan=0.0, posinf=0.0, neginf=0.0)[rows]
    most = bound(dtype, O[rows], A[rows], clean_S + 30.0, 500, dh)
    assert bool(((got[rows].double() - O[rows]).abs() <= most).all())
    assert not torch.isfinite(got[last.cuda()]).all()


@pytest.mark.parametrize("dtype,dh,counts", [(BF16, 64, [1, 1, 1]), (BF16, 128, [200, 3, 64]), (F32, 64, [20, 1, 5]), (BF16, 64, [200, 3, 64])])
def test_pages_and_slots_outside_the_pool(dtype, dh, counts):
    lens = [300, 64, 190]
    case = build(dtype, counts, lens, 2, 2, dh, 16, seed=7)
    s = case["slots"].tolist()
    case["table"][s[0], 2] = -1
    case["table"][s[0], 5] = case["K"].shape[0]
    case["table"][s[2], 0] = 2 ** 31 - 1
    case["slots"][1] = 1000
    got = check(case)
    a, b = case["offsets"][1:3]
    assert torch.all(got[a:b] == 0)
    case["slots"][1] = -1
    case["lens"][s[0]] = 2 ** 31 - 1          # as much as the table's row
    case["lens"][s[2]] = -4                   # as nothing
    case["table"][s[0], -(-300 // 16):] = -1  # pages of zeros
    id = int(case["table"][s[0], 300 // 16])
    assert id == -1 or 300 % 16 != 0
    last = int(case["table"][s[0], 18])
    case["K"][last, 12:] = 0
    case["V"][last, 12:] = 0
    check(case, causal=False)


@pytest.mark.parametrize("dtype,dh,L,n,G", [(BF16, 128, 70000, 1, 8), (BF16, 64, 40001, 2, 1), (F32, 64, 30000, 1, 2), (BF16, 128, 20000, 33, 4)])
def test_long_histories_are_shared_over_the_chip(dtype, dh, L, n, G):
    check(build(dtype, [n, 1], [L, 9], 1, G, dh, 64, seed=8), slopes=slopes(G))


@pytest.mark.parametrize("dtype,dh,n", [(BF16, 128, 1), (BF16, 64, 200), (F32, 64, 3)])
def test_offsets_beyond_32_bits(dtype, dh, n):
    page, Hkv = 64, 8
    size = torch.finfo(dtype).bits // 8
    n_pages = int(5.1e9) // (page * Hkv * dh * size)      # the pool's last pages are 5 GB from its start
    K = torch.empty((n_pages, page, Hkv, dh), dtype=dtype, device="cuda")
    V = torch.empty_like(K)
    lens = [n + 300, n]
    ids = [n_pages - 1 - i for i in range(12)]
    used = torch.tensor(ids).cuda()
    K[used] = torch.randn((12, page, Hkv, dh), device="cuda").to(dtype)
    V[used] = torch.randn((12, page, Hkv, dh), device="cuda").to(dtype)
    table = torch.tensor([ids[:6] + [0] * 2, ids[6:] + [0] * 2], dtype=torch.int32).cuda()
    off = torch.tensor([0, n, 2 * n], dtype=torch.int32)
    lens[0] = min(lens[0], 6 * page)
    Q = torch.randn((2 * n, Hkv, dh), device="cuda").to(dtype)
    case = {"K": K, "V": V, "table": table, "lens": torch.tensor(lens, dtype=torch.int32).cuda(), "offsets": off.tolist(),
            "slots": torch.tensor([0, 1], dtype=torch.int32).cuda(), "plan": rocs.plan_create(off.cuda(), off), "Q": Q}
    check(case)


def test_many_requests():
    rng = random.Random(9)
    lens = [rng.randint(0, 90) for _ in range(700)]
    check(build(BF16, [rng.randint(0, 2) for _ in lens], lens, 1, 2, 64, 16, seed=9))
    check(build(BF16, [rng.randint(0, 40) for _ in lens], lens, 1, 2, 64, 16, seed=9), causal=False)


@pytest.mark.parametrize("dtype,dh,counts", [(BF16, 64, [1, 1, 1, 1]), (BF16, 128, [60, 200, 3, 1]), (F32, 64, [20, 1, 5, 9])])
def test_another_requests_values_change_no_bit(dtype, dh, counts):
    lens = [300, 400, 90, 333]
    case = build(dtype, counts, lens, 2, 2, dh, 16, seed=10)
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    one = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"]).clone()
    again = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"])
    assert torch.equal(one, again)
    mine = case["table"][case["slots"][1].long()][:-(-400 // 16)].long()
    case["K"][mine] *= 100
    case["V"][mine] = float("nan")
    a, b = case["offsets"][1:3]
    case["Q"][a:b] *= 3
    two = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"])
    keep = torch.ones(one.shape[0], dtype=torch.bool)
    keep[a:b] = False
    assert torch.equal(one[keep.cuda()], two[keep.cuda()])


@pytest.mark.parametrize("dtype,dh,counts", [(BF16, 64, [1, 1, 1]), (BF16, 128, [150, 3, 64]), (F32, 64, [20, 1, 5])])
def test_a_captured_call_works_on_what_it_finds(dtype, dh, counts):
    lens = [300, 80, 190]
    case = build(dtype, counts, lens, 2, 2, dh, 16, seed=11)
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    out = torch.empty_like(case["Q"])
    ws = torch.empty(rocs.cache_attention_workspace(cache, case["plan"], 4), dtype=torch.uint8, device="cuda")
    rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], out=out, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], out=out, workspace=ws)
    for change in (0, 50):
        case["lens"][case["slots"][0].long()] = 300 - change
        case["slots"].copy_(case["slots"].clone())
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist())
        assert bool(((out.double() - O).abs() <= bound(dtype, O, A, S, 300, dh)).all())


def test_calls_on_two_streams_at_once():
    cases = [build(BF16, [1, 90, 300], [4000, 2000, 900], 2, 2, 128, 64, seed=12 + i) for i in range(2)]
    caches = [rocs.cache_create(c["K"], c["V"], c["table"], c["lens"]) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = []
    for c, cache, s in zip(cases, caches, streams):
        with torch.cuda.stream(s):
            off = torch.tensor(c["offsets"], dtype=torch.int32)
            c["plan"] = rocs.plan_create(off.cuda(), off)
            for _ in range(5):
                got = rocs.cache_attention(cache, c["plan"], c["Q"], slots=c["slots"])
            outs.append(got)
    torch.cuda.synchronize()
    for c, got in zip(cases, outs):
        O, A, S = plain.attention(c["K"], c["V"], c["table"], c["lens"], c["offsets"], c["Q"], c["slots"].tolist())
        assert bool(((got.double() - O).abs() <= bound(BF16, O, A, S, 4000, 128)).all())


def test_the_general_kernel_takes_every_shape():
    case = build(BF16, [1, 90, 300], [400, 200, 900], 2, 2, 128, 64, seed=14)
    rocs.set_path(rocs.PATH_GENERAL)
    try:
        check(case, cap=3.0)
    finally:
        rocs.set_path(rocs.PATH_AUTO)
    check(case, cap=3.0)


def test_all_visible_scores_at_the_lowest_value_and_beyond():
    # scores of about -3e38: the row's softmax is that of their differences; of -inf: no softmax, as 0 / 0
    case = build(F32, [1, 4], [70, 40], 1, 1, 64, 16, seed=15)
    case["Q"].fill_(1.0)
    held = ~torch.isnan(case["K"])
    case["K"][held] = -4.0e37
    got = check(case, scale=0.1)
    assert torch.isfinite(got).all()
    case["K"][held] = -float("inf")
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    got = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"])
    assert torch.isnan(got).all()


@pytest.mark.parametrize("dh,page,counts", [(64, 16, [1, 1, 4]), (128, 64, [2, 16, 1]), (64, 24, [1, 4, 30]), (64, 16, [40, 300, 129])])
def test_equal_scores_next_to_the_lowest_value(dh, page, counts):
    """All visible scores are the same product, -3.08e38 in powers of two: the result is the mean of the values."""
    case = build(BF16, counts, [90, 400, 300], 1, 1, dh, page, seed=20)
    case["Q"].zero_()
    case["Q"][..., 0] = 2.0 ** 63
    case["K"][~torch.isnan(case["K"])] = -(2.0 ** 64)
    got = rocs.cache_attention(rocs.cache_create(case["K"], case["V"], case["table"], case["lens"]), case["plan"], case["Q"],
                               slots=case["slots"], scale=1.255)
    O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist(), scale=1.255)
    assert bool(((got.double() - O).abs() <= bound(BF16, O, A, torch.zeros_like(S), 400, dh)).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dh,counts", [(128, [1, 1, 1]), (64, [2, 1, 3]), (128, [40, 300, 129]), (64, [200, 90, 30]), (32, [60, 2, 40])])
@pytest.mark.parametrize("toward", ["first", "last"])
def test_scores_that_grow_by_hundreds(dtype, dh, counts, toward):
    """Keys that are multiples of one direction: scores climb (or fall) by about 25 per key, far beyond fp32's exponents over a
    sequence; every row's softmax is all but its largest visible key's value."""
    lens = [700, 400, 513]
    case = build(dtype, counts, lens, 1, 2, dh, 16, seed=16)
    direction = torch.zeros(dh, device="cuda")
    direction[0] = 1.0
    for r, L in enumerate(lens):
        row = case["table"][case["slots"][r].long()]
        for j in range(L):
            at = j if toward == "last" else L - 1 - j
            case["K"][int(row[j // 16]), j % 16] = (direction * 2.0 * at).to(dtype)
    case["Q"][:] = (direction * 12.5).to(dtype)
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    got = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], scale=1.0)
    O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist(), scale=1.0)
    # the products are exact: one term each, 12.5 x an even number of at most 1400 (bf16 rounds it to 8 bits, alike for both)
    assert torch.isfinite(got).all()
    most = bound(dtype, O, A, torch.full_like(S, 64.0), 700, dh)
    assert bool(((got.double() - O).abs() <= most).all())


@pytest.mark.parametrize("dtype,dh,n,page", [(BF16, 64, 130, 16), (BF16, 64, 300, 128), (BF16, 128, 130, 16), (BF16, 64, 50, 24), (BF16, 64, 1, 16),
                                             (BF16, 128, 9, 64), (F32, 64, 20, 16)])
@pytest.mark.parametrize("score", [60.0, 95.0, 1600.0, float("nan")])
def test_one_key_far_above_all_others(dtype, dh, n, page, score):
    """One key of each request, at another place of 16, whose score all rows see; far beyond fp32's exponents the softmax is its
    value alone, and a row that sees a NaN is NaN."""
    R, L = 16, 700
    case = build(dtype, [n] * R, [L] * R, 1, 1, dh, page, seed=19)
    case["K"][..., 0] = torch.where(case["K"][..., 0].isnan(), case["K"][..., 0], 0.0)
    case["Q"][..., 0] = 8.0
    for r in range(R):
        j = 192 + r
        row = case["table"][case["slots"][r].long()]
        case["K"][int(row[j // page]), j % page, 0, 0] = score
    if score == score:
        check(case, scale=0.125)
    else:
        cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
        assert torch.isnan(rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], scale=0.125)).all()


@pytest.mark.parametrize("dtype,dh,page", [(BF16, 64, 16), (BF16, 128, 24), (F32, 32, 8)])
@pytest.mark.parametrize("R,n", [(130, 1), (200, 3), (200, 40), (300, 20), (140, 90)])
def test_more_tiles_than_a_block_keeps(dtype, dh, page, R, n):
    rng = random.Random(17)
    lens = [rng.randint(0, 60) + n for _ in range(R)]
    counts = [rng.randint(0, n) for _ in range(R)]
    case = build(dtype, counts, lens, 1, 1, dh, page, seed=17)
    begin = []
    for c, L in zip(counts, lens):
        begin += [max(0, (L - c + t) - 20) for t in range(c)]
    check(case)
    check(case, begin=torch.tensor(begin, dtype=torch.int32).cuda(), slopes=slopes(1))


def test_refusals():
    case = build(BF16, [1, 90], [400, 200], 2, 2, 64, 16, seed=18)
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    Q, plan, slots = case["Q"], case["plan"], case["slots"]
    out = torch.full_like(Q, 7.0)

    def refused(error, match=None, **how):
        args = dict(slots=slots, out=out)
        q = how.pop("Q", Q)
        args.update(how)
        with pytest.raises(error, match=match):
            rocs.cache_attention(cache, plan, q, **args)

    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    refused(AssertionError, slots=ints(0))
    refused(AssertionError, slots=slots.long())
    refused(AssertionError, slots=slots.cpu())
    refused(AssertionError, Q=Q[:5])
    refused(AssertionError, Q=Q.float())
    refused(AssertionError, Q=Q.cpu())
    refused(AssertionError, Q=Q[:, :, :32])
    refused(ValueError, Q=Q[0])
    refused(rocs.RocsError, "invalid", Q=Q[:, :3].contiguous(), out=None)       # heads that do not share the key heads evenly
    refused(AssertionError, slopes=slopes(3))
    refused(AssertionError, begin=ints(0, 0))
    refused(AssertionError, prefix=ints(0))
    refused(rocs.RocsError, "invalid", prefix=ints(0, 0), causal=False)
    refused(rocs.RocsError, "invalid", cap=-1.0)
    refused(rocs.RocsError, "invalid", cap=float("inf"))
    refused(rocs.RocsError, "invalid", scale=float("nan"))
    refused(rocs.RocsError, "invalid", layer=1)
    refused(rocs.RocsError, "invalid", layer=-1)
    refused(rocs.RocsError, "workspace", workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    refused(AssertionError, workspace=torch.empty(1 << 20, dtype=torch.float32, device="cuda"))
    wide = torch.empty((Q.shape[0], 4, 66), dtype=BF16, device="cuda")
    refused(rocs.RocsError, "align", out=wide[:, :, :64])
    refused(rocs.RocsError, "invalid", out=Q[:1].expand_as(Q))                  # rows that share memory
    torch.cuda.synchronize()
    assert torch.all(out == 7.0)
    cache.close()
    refused(ValueError, "closed")
    with pytest.raises(rocs.RocsError):
        rocs.cache_create(case["K"], case["V"], case["table"], torch.zeros(case["table"].shape[0] + 1, dtype=torch.int32, device="cuda")[1:])


def test_outputs_that_share_memory_and_scales_without_a_value_are_refused():
    case = build(BF16, [1, 90], [400, 200], 2, 2, 64, 16, seed=18)
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    flat = torch.full((91 * 4 * 64 + 64,), 7.0, dtype=BF16, device="cuda")
    for strides in ((64, 64, 1), (128, 64, 1), (248, 64, 1), (64, 90 * 64, 1), (0, 64, 1), (256, 0, 1)):
        with pytest.raises(rocs.RocsError, match="invalid"):
            rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], out=flat.as_strided((91, 4, 64), strides))
    for how in (dict(scale=3e38), dict(scale=1.0, cap=1e-39)):
        with pytest.raises(rocs.RocsError, match="invalid"):
            rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], out=flat[:91 * 256].view(91, 4, 64), **how)
    torch.cuda.synchronize()
    assert torch.all(flat == 7.0)
    check(case, out=flat.as_strided((91, 4, 64), (64, 91 * 64, 1)))
    check(case, out=flat.as_strided((91, 4, 64), (256, 64, 1)))


def test_views_of_the_pool_that_overlap_are_refused():
    K = torch.zeros((4, 16, 2, 64), dtype=BF16, device="cuda")
    table, lens = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for view in (K[:1].expand(4, 16, 2, 64), K[:, :, :1].expand(4, 16, 2, 64)):
        with pytest.raises(rocs.RocsError, match="invalid"):
            rocs.cache_create(view, view, table, lens)
    rocs.cache_create(K, K.clone(), table, lens)
