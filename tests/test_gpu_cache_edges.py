"""The paged cache where one tile, one row or one call leaves something to the next."""
import pytest
import torch

import _cache_ref as plain
from paper_2607_27744_b200 import binding as rocs
from test_gpu_cache_attention import BF16, bound, build

pytestmark = pytest.mark.gpu


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
