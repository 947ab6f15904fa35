"""The paged cache where one tile, one row or one call leaves something to the next."""
import random

import pytest
import torch

import _cache_ref as plain
from paper_2607_27744_b200 import binding as rocs
from test_gpu_cache_attention import BF16, F32, bound, build, check, slopes
from test_gpu_cache_books import Pair, ints, plan_of

pytestmark = pytest.mark.gpu

# one call for each kernel: (dtype, dh, page, new rows of each request)
KERNELS = [(BF16, 128, 16, [1, 1, 1]), (BF16, 64, 64, [5, 1, 4]), (BF16, 32, 16, [3, 8, 1]), (BF16, 64, 24, [1, 5, 2]),
           (BF16, 32, 16, [60, 3, 17]), (BF16, 64, 16, [70, 200, 3]), (BF16, 128, 64, [300, 40, 130]), (BF16, 48, 16, [9, 1, 20]),
           (F32, 64, 16, [20, 1, 5])]


@pytest.mark.parametrize("dh", [64, 128])
def test_small_tiles_behind_tiles_that_are_computed_again(dh):
    """Chunks of 200 rows whose last event holds NaN (all other rows are computed again, on what a tile's warps told one
    another at its end), each followed by a chunk that has one block of keys."""
    counts, lens = [], []
    for r in range(120):
        counts += [200, 40 + r % 80]
        lens += [300 + r, 128 - r % 5]
    case = build(BF16, counts, lens, 1, 1, dh, 16, seed=31)
    O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist())
    keep = torch.ones(case["offsets"][-1], dtype=torch.bool, device="cuda")
    for r in range(0, 240, 2):
        id = int(case["table"][int(case["slots"][r]), (lens[r] - 1) // 16])
        case["K"][id, (lens[r] - 1) % 16] = float("nan")
        case["V"][id, (lens[r] - 1) % 16] = float("nan")
        keep[case["offsets"][r + 1] - 1] = False
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    most = bound(BF16, O, A, S, 420, dh)
    for _ in range(5):
        got = rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"])
        assert bool(((got.double() - O).abs() <= most)[keep].all())
        assert torch.isnan(got[~keep]).all()
    rocs.last_device_status()


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("cap", [1e3, 1e4, 1e6, 1e9, 1e30])
@pytest.mark.parametrize("bias", [False, True])
def test_caps_far_above_the_scores(dtype, dh, page, counts, cap, bias):
    """A score is right to fp32's roundings of it, however far the cap is above it."""
    case = build(dtype, counts, [700, 450, 177], 2, 2, dh, page, seed=33)
    check(case, cap=cap, slopes=slopes(4) if bias else None)


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("cap", [30.0, 200.0, 1e4])
def test_scores_of_hundreds_under_a_cap(dtype, dh, page, counts, cap):
    check(build(dtype, counts, [700, 450, 177], 2, 2, dh, page, seed=34, std=40.0), cap=cap)


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("cap", [50.0, 1e4, 1e6, 1e9])
def test_one_score_beyond_the_cap_below_all_others(dtype, dh, page, counts, cap):
    """Keys whose scores end at -cap, and weigh nothing, beside others whose scores are far from it: how far those may be off goes
    by their own size."""
    lens = [700, 450, 177]
    case = build(dtype, counts, lens, 2, 2, dh, page, seed=35)
    case["K"][..., 0] = torch.where(case["K"][..., 0].isnan(), case["K"][..., 0], 0.0)
    case["Q"][..., 0] = 8.0
    _, _, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist(), scale=0.125)
    for r in range(3):
        for j in (3, 40, 100):
            row = case["table"][case["slots"][r].long()]
            case["K"][int(row[j // page]), j % page, :, 0] = -2.0 * cap
    O, A, _ = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist(),
                              scale=0.125, cap=cap)
    got = rocs.cache_attention(rocs.cache_create(case["K"], case["V"], case["table"], case["lens"]), case["plan"], case["Q"],
                               slots=case["slots"], scale=0.125, cap=cap)
    off = (got.double() - O).abs()
    most = bound(dtype, O, A, S, 700, dh)
    assert bool((off <= most).all()), f"off by {float((off / most).max()):.3f} of the bound"


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("cap", [1e37, 3e38, torch.finfo(F32).max])
def test_caps_at_the_end_of_what_fp32_holds(dtype, dh, page, counts, cap):
    case = build(dtype, counts, [700, 450, 177], 2, 2, dh, page, seed=38)
    check(case, cap=cap)
    cache = rocs.cache_create(case["K"], case["V"], case["table"], case["lens"])
    out = torch.full_like(case["Q"], 7.0)
    for how in (dict(cap=3e38, scale=4.0), dict(cap=10.0, scale=1e-38), dict(cap=1e19, scale=1e-30)):
        with pytest.raises(rocs.RocsError, match="invalid"):
            rocs.cache_attention(cache, case["plan"], case["Q"], slots=case["slots"], out=out, **how)
    torch.cuda.synchronize()
    assert torch.all(out == 7.0)


@pytest.mark.parametrize("n_pages,n_slots,width,n", [(10, 3, 40, 40), (5000, 5, 2000, 2000), (10, 1500, 2, 1), (4097, 1500, 4, 4), (9000, 3, 4000, 4000)])
def test_how_many_pages_are_missing(n_pages, n_slots, width, n):
    pair = Pair(BF16, 1, n_pages, 1, 1, 8, n_slots + 1, width)
    pair.extend([n_slots], [2])
    pair.extend(list(range(n_slots)), [n] * n_slots)
    assert pair.report.tolist() == [1, n * n_slots - (n_pages - 2)]


def test_nearly_as_many_pages_are_missing_as_rows_can_be_named():
    pair = Pair(BF16, 1, 10, 1, 1, 8, 2047, 1)
    wide = torch.full((2047, 1 << 20), -1, dtype=torch.int32, device="cuda")
    cache = rocs.cache_create(pair.K, pair.V, wide, pair.lens, pair.refs)
    off = torch.arange(2048, dtype=torch.int32) * (1 << 20)
    first = rocs.cache_extend(cache, rocs.plan_create(off.cuda(), off), report=pair.report)
    assert pair.report.tolist() == [1, 2047 * (1 << 20) - 10] and bool((first == -1).all())
    assert bool((pair.lens == 0).all()) and bool((pair.refs == 0).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
def test_a_key_that_weighs_nothing_but_is_seen(dtype, dh, page, counts, value):
    """exp of a score far below the others is 0 in fp32, and 0 x NaN or Inf is NaN: whatever masks the block and its other rows have."""
    lens = [700, 450, 177]
    case = build(dtype, counts, lens, 1, 2, dh, page, seed=36)
    case["K"][..., 0] = torch.where(case["K"][..., 0].isnan(), case["K"][..., 0], 0.0)
    case["Q"][..., 0] = 8.0
    sees = torch.zeros(case["offsets"][-1], dtype=torch.bool)
    for r, (n, L) in enumerate(zip(counts, lens)):
        j = L - 1 - n // 2
        row = case["table"][case["slots"][r].long()]
        case["K"][int(row[j // page]), j % page, :, 0] = -1e6
        case["V"][int(row[j // page]), j % page] = value
        sees[case["offsets"][r] + n - 1 - n // 2:case["offsets"][r + 1]] = True
    got = rocs.cache_attention(rocs.cache_create(case["K"], case["V"], case["table"], case["lens"]), case["plan"], case["Q"],
                               slots=case["slots"], scale=0.125)
    assert not torch.isfinite(got[sees.cuda()]).any()
    assert torch.isfinite(got[~sees.cuda()]).all()


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("base", [2.0 ** 10, 2.0 ** 24, 2.0 ** 26, 2.0 ** 28])
@pytest.mark.parametrize("causal", [True, False])
def test_large_scores_that_pass_the_first_keys_by_little(dtype, dh, page, counts, base, causal):
    """Exact scores of `base`, and of 32 more for every 50th key but the last 500: the result is the mean over those.  A reference
    found in the last keys has to move by 46 powers of two, which fp32 cannot add to numbers of this size."""
    lens = [1700, 1450, 977]
    case = build(dtype, counts, lens, 40, 2, dh, page, seed=39)   # (heads enough for pieces of many blocks)
    case["Q"].zero_()
    case["Q"][..., 0] = 2.0 ** 10
    case["Q"][..., 1] = 8.0
    case["K"][..., :2] = torch.where(case["K"][..., :2].isnan(), case["K"][..., :2], 0.0)
    case["K"][..., 0] += base / 2.0 ** 10
    for r, L in enumerate(lens):
        row = case["table"][case["slots"][r].long()]
        for j in range(0, L - 500, 50):
            case["K"][int(row[j // page]), j % page, :, 1] = 4.0
    got = rocs.cache_attention(rocs.cache_create(case["K"], case["V"], case["table"], case["lens"]), case["plan"], case["Q"],
                               slots=case["slots"], scale=1.0, causal=causal)
    O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"], case["slots"].tolist(),
                              scale=1.0, causal=causal)
    # (the other keys' weights are e^-32 each, of a sum of ten and more: their errors are far below a rounding)
    off, most = (got.double() - O).abs(), bound(dtype, O, A, torch.zeros_like(S), 1700, dh)
    assert bool((off <= most).all()), f"off by {float((off / most).max()):.3f} of the bound"


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("size", [2.0 ** 28, 1.5 * 2.0 ** 30, 2.0 ** 31, 1.25 * 2.0 ** 33, 1.5 * 2.0 ** 40])
@pytest.mark.parametrize("top", [False, True])
@pytest.mark.parametrize("heads", [1, 40])   # pieces of one block, or of many
def test_scores_beyond_32_bits(dtype, dh, page, counts, size, top, heads):
    """Scores so large that fp32's next one is 2^5 to 2^17 away: all equal (products of powers of two and 3 or 5, exact), or one
    above the others; the mean of the values, or the one's."""
    lens = [1700, 1450, 977]
    case = build(dtype, counts, lens, heads, 2, dh, page, seed=37)
    case["Q"].zero_()
    case["Q"][..., 0] = 2.0 ** 10
    case["K"][..., 0] = torch.where(case["K"][..., 0].isnan(), case["K"][..., 0], size / 2.0 ** 10)
    if top:
        for r in range(3):
            row = case["table"][case["slots"][r].long()]
            case["K"][int(row[600 // page]), 600 % page, :, 0] *= 1.03125
    for scale in (0.11, 0.3, 0.7, 0.9, 1.3, 3.3) if heads == 1 else (0.7, 1.3):
        for causal in (True, False) if heads == 1 else (True,):
            got = rocs.cache_attention(rocs.cache_create(case["K"], case["V"], case["table"], case["lens"]), case["plan"], case["Q"],
                                       slots=case["slots"], scale=scale, causal=causal)
            O, A, S = plain.attention(case["K"], case["V"], case["table"], case["lens"], case["offsets"], case["Q"],
                                      case["slots"].tolist(), scale=scale, causal=causal)
            off, most = (got.double() - O).abs(), bound(dtype, O, A, torch.zeros_like(S), 1700, dh)
            assert bool((off <= most).all()), (scale, causal, f"off by {float((off / most).max()):.3f} of the bound")


@pytest.mark.parametrize("dtype,dh,page,counts", KERNELS)
@pytest.mark.parametrize("heads", [1, 24])
@pytest.mark.parametrize("seed", range(6))
def test_scores_that_pass_the_first_keys_by_all_of_fp32s_exponents(dtype, dh, page, counts, heads, seed):
    """Scores of 0, and here and there, but not among the last keys, of 87 to 95: their weights relative to the last keys' are at the
    end of fp32's range or beyond it, in one block or on one side of a tile and nearly as large on the other.  (Values are
    small, so that weights of 2^127 times values have a place in fp32.)"""
    rng = random.Random(seed)
    lens = [1700, 1450, 977]
    case = build(dtype, counts, lens, heads, 2, dh, page, seed=40 + seed)
    case["V"] *= 0.125
    case["Q"].zero_()
    case["Q"][..., 0] = 1.0
    case["K"][..., 0] = torch.where(case["K"][..., 0].isnan(), case["K"][..., 0], 0.0)
    for r, L in enumerate(lens):
        row = case["table"][case["slots"][r].long()]
        last = L // 128 * 128
        some = rng.sample(range(last), 8) if seed < 3 else [rng.randrange(last - 128, last), rng.randrange(last - 256, last - 128),
                                                            rng.randrange(last - 384, last - 256)]
        for j in some:
            score = rng.choice([88.0, 88.25] if seed < 2 else [87.5, 88.25, 88.5, 95.0]) if seed < 3 else 88.5 if j >= last - 128 else 87.5
            case["K"][int(row[j // page]), j % page, :, 0] = score
    for causal in (True, False):
        check(case, scale=1.0, causal=causal)


def test_more_free_pages_than_are_kept_near():
    """Calls that take more than 4096 pages, found between held ones and beyond the first 4096 of the pool."""
    rng = random.Random(6)
    pair = Pair(BF16, 1, 14000, 1, 1, 8, 2000, 40)
    pair.extend(list(range(100)), [30] * 100)
    pair.truncate(list(range(0, 100, 2)), [rng.randint(0, 20) for _ in range(50)])

    def grow(slots, counts):
        status, pages, first, copies = pair.books.extend(slots, counts)
        got = rocs.cache_extend(pair.cache, plan_of(counts), slots=ints(slots), report=pair.report)
        assert got.tolist() == first
        pair.check(status, pages)

    grow(list(range(100, 400)), [rng.randint(15, 25) for _ in range(300)])
    pair.truncate(list(range(100, 400, 3)))
    grow(list(range(400, 1900)), [rng.randint(0, 6) for _ in range(1500)])


def test_more_slots_than_a_block_has_bits_for():
    """Above 262144 slots a slot named twice is found by a word in the workspace."""
    n = 32 * 8192 + 100
    pair = Pair(BF16, 1, 50, 4, 1, 8, n, 2)
    pair.extend([n - 1, 5, n - 60, 0], [6, 3, 8, 1])
    pair.extend([n - 1, 7, n - 1], [1, 1, 1])
    assert pair.report.tolist() == [2, 0]
    pair.fork([n - 60, n - 1], [9, 100000])
    pair.fork([5, 5], [n - 2, n - 2])
    pair.extend([n - 1, 100000], [1, 1])
    pair.truncate([n - 1, 9, n - 1])
    assert pair.report.tolist() == [2, 0]
    pair.truncate([n - 1, 9, 5], [4, 0, 0])
    pair.compact()
