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


def test_attend_empty_sequence_of_2_to_31_elements(apc):
    """A sequence that holds nothing, its output of 2^31 elements: all of them are written."""
    heads, group, d, page = 1 << 19, 16, 256, 16
    say("attend 2^31 elements of an empty sequence")
    k, v = (torch.empty((1, heads, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = apc.KvCache(k, v)
    q = torch.empty((1, heads * group, d), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    table, lens = torch.zeros((1, 128), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    apc.apc_attend(c, q, table, lens, 0.1, out, apc.attend_workspace_tensor(c, 1, heads * group, 128), lse)
    torch.cuda.synchronize()
    assert not out.view(torch.int32).any() and torch.isneginf(lse).all()
