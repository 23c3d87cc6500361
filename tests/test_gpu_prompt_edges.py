"""Corners of the prompt model's operators against float64."""
import pytest
import torch

from tests.gpu_check import say
from tests.test_gpu_prompt_ops import KINDS, check_attend, make_attend, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def apc():
    import paper_2502_06798_amd as apc
    apc.load()
    assert torch.cuda.is_available()
    return apc


# ---- attention: many query heads -----------------------------------------------

@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("group,d", [(8193, 64), (8193, 128), (4097, 256), (20000, 128)])
def test_attend_more_query_tiles_than_compute_units(apc, orc, cache, dtype, group, d):
    """One key-value head for thousands of query heads over tables that are cut: every output is written."""
    say(f"attend query tiles {dtype} over {cache} group={group} d={d}")
    lens = [3000, 0, 70]
    pool, table, q = make_attend(group + d, len(lens), 1, group, d, 64, 47, cache, dtype)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = run_attend(apc, pool, table, q, n, d ** -0.5)
    assert torch.equal(torch.isneginf(lse).all(dim=1).cpu(), torch.tensor([False, True, False]))
    assert (out[1] == 0).all() and not (out[::2] == 7.0).all(dim=2).any() and not (lse == 7.0).any()
    at = torch.tensor([0, 15, 16, 31, 32, group // 2, group - 2, group - 1], device="cuda")
    check_attend(orc, cache, dtype, pool, table, q[:, at], n, d ** -0.5, 0, out[:, at], lse[:, at])
