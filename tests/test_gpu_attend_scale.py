"""GPU parity of attention of single tokens with scales whose product with log2(e) is beyond float32."""
import pytest
import torch

from tests.gpu_check import say
from tests.test_gpu_prompt_ops import KINDS, check_attend, gen, make_attend, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def apc():
    import paper_2502_06798_amd as apc
    apc.load()
    assert torch.cuda.is_available()
    return apc


@pytest.mark.parametrize("cache,dtype", KINDS)
@pytest.mark.parametrize("scale", [2.3e38, 3e38, -3.4e38])
@pytest.mark.parametrize("group,d,lens", [(4, 64, [1, 40, 1000]), (2, 128, [5000, 3]), (20, 256, [300, 33])])
def test_attend_scales_at_the_end_of_the_range(apc, orc, cache, dtype, scale, group, d, lens):
    """Products of 0 score 0, and tiny ones what they should: of p 2^-122, 56 p and less (f16 holds none so small)."""
    say(f"attend scale {scale} {dtype} over {cache} group={group} d={d}")
    pool, table, q = make_attend(d, len(lens), 2, group, d, 64, -(-max(lens) // 64), cache, dtype)
    p = torch.randint(-2, 3, pool[0].shape[:3], device="cuda", generator=gen(4)).float()
    q.zero_()
    pool[0].view(torch.uint8).zero_()
    if cache == "e4m3":
        pool[0][..., 0] = p.to(pool[0].dtype)
        q[..., 0] = 2.0 ** -10
        pool[2].fill_(2.0 ** -112)
    elif cache == "bf16":
        pool[0][..., 0] = (p * 2.0 ** -61).to(pool[0].dtype)
        q[..., 0] = 2.0 ** -61
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    check_attend(orc, cache, dtype, pool, table, q, n, scale, 0, *run_attend(apc, pool, table, q, n, scale))
