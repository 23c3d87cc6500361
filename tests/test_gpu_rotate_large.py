"""Rotary positions of calls with more threads than a launch has: every row as small calls turn it, bit for bit."""
import pytest
import torch

from tests.gpu_check import say
from tests.test_gpu_prompt_ops import gen

pytestmark = pytest.mark.gpu

LAUNCH = 2 ** 20 * 256                                       # threads of the largest launch (csrc/rotate.hip, MAX_GRID)
PERIOD = 4_194_301                                           # prime: no two rows of a tensor hold the same elements for long


@pytest.fixture(scope="module")
def apc():
    import paper_2502_06798_amd as apc
    apc.load()
    assert torch.cuda.is_available()
    return apc


def fill(flat, pattern):
    for i in range(0, flat.numel(), PERIOD):
        flat[i:i + PERIOD] = pattern[:flat.numel() - i]


def part(pattern, start, n):
    """What fill() put at elements start to start + n."""
    return pattern[(start + torch.arange(n, device="cuda")) % PERIOD]


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_steps_over_the_grid(apc, interleaved):
    """Pieces of one pair and four heads a thread: 3 10^8 threads, so that threads take a second step; some tokens left out."""
    t, heads, d = 1_000_000, 400, 6
    assert t * (heads // 4) * (d // 2) > LAUNCH
    pattern = torch.randn(PERIOD, device="cuda", generator=gen(1)).half()
    x = torch.empty((t, heads, d), dtype=torch.float16, device="cuda")
    fill(x.view(-1), pattern)
    at = torch.randint(-50_000, 1_000_000, (t,), device="cuda", generator=gen(2), dtype=torch.int32)
    r = apc.Rotary(torch.from_numpy(apc.apc_rotary_freqs(d)).cuda(), interleaved, 1.5)
    say(f"rotate {t} x {heads} x {d} in place interleaved={interleaved}")
    apc.apc_rotate(r, x, at, x)
    torch.cuda.synchronize()
    for i in range(0, t, 5000):
        was = part(pattern, i * heads * d, 5000 * heads * d).view(5000, heads, d)
        want = was.clone()
        apc.apc_rotate(r, was, at[i:i + 5000], want)
        assert same(want, x[i:i + 5000]), i
    assert not same(was, want)                               # (they are turned)


def test_rotate_every_head_of_as_many_as_a_call_takes(apc):
    """One token of 2^31 - 1 heads: each of them."""
    heads, d, step = 2 ** 31 - 1, 2, 2 ** 25
    pattern = torch.randn(PERIOD, device="cuda", generator=gen(3)).half()
    x = torch.empty((1, heads, d), dtype=torch.float16, device="cuda")
    fill(x.view(-1), pattern)
    at = torch.tensor([12345], dtype=torch.int32, device="cuda")
    r = apc.Rotary(torch.from_numpy(apc.apc_rotary_freqs(d)).cuda())
    say("rotate 2^31 - 1 heads in place")
    apc.apc_rotate(r, x, at, x)
    torch.cuda.synchronize()
    for i in range(0, heads, step):
        n = min(step, heads - i)
        was = part(pattern, i * d, n * d).view(1, n, d)
        want = torch.empty_like(was)
        apc.apc_rotate(r, was, at, want)
        assert same(want, x[:, i:i + n]), i
    assert not same(was, want)
