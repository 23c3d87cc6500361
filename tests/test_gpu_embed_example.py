"""The example that runs the prompt model's operators together and on into the
matching step: unchanged prompts find themselves, and a prefix whose pages are
shared gives the embeddings of one that every sequence read for itself.  A
step's state is checked against a float64 forward from the formulas."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_prompts_find_their_source():
    import embed_and_match as ex
    found, source, top, score = ex.main(n_cached=64, b=16)
    assert (top[::2] == source[::2]).all()                       # unchanged prompts
    assert (score[::2] > 0.999).all()
    assert found >= 12


def test_shared_prefix_equals_own_prefix():
    import paper_2502_06798_amd as apc
    import embed_and_match as ex
    apc.load()
    rng = np.random.default_rng(3)
    model = ex.TextModel(layers=2)
    instruction = rng.integers(0, 1000, 32).tolist()
    prompts = [rng.integers(0, 1000, n).tolist() for n in (1, 7, 16, 17, 40)]
    a, sa = ex.embed(model, instruction, prompts, shared=True)
    b, sb = ex.embed(model, instruction, prompts, shared=False)
    torch.cuda.synchronize()
    # torch's products may add in another order for one row than for five
    x, y = a.float() * sa[:, None], b.float() * sb[:, None]
    assert (torch.nn.functional.cosine_similarity(x, y, dim=1) > 0.995).all()


def test_step_equals_formulas(orc):
    """One block over 20 tokens, each step's attention against float64 from the cache's own values."""
    import paper_2502_06798_amd as apc
    import embed_and_match as ex
    apc.load()
    rng = np.random.default_rng(5)
    model = ex.TextModel(layers=1)
    reader = ex.Reader(model, 3, 12, 4)
    ids = rng.integers(0, 1000, (20, 3))
    for t in range(20):
        live = np.array([True, t < 11, t % 2 == 0 or t > 15])
        reader.step(torch.from_numpy(ids[t]).cuda(), live)
    torch.cuda.synchronize()
    c, block = reader.caches[0], model.blocks[0]
    f64 = lambda x: x.float().cpu().numpy().astype(np.float64)
    # the last step's state, from its tokens on
    lens = reader.lengths.cpu().numpy()
    assert lens.tolist() == [20, 11, 12]
    place = lens - np.array([1, 0, 1])                            # sequence 1 had no token: its place is unchanged
    r = f64((model.emb[torch.from_numpy(ids[19]).cuda()] + model.pos[torch.from_numpy(place).cuda()]))
    x, _ = orc.norm_rows(r, None, f64(block["n1"]), 1e-6)
    q = (x @ f64(block["qkv"]).T).reshape(3, -1, model.d)[:, :model.q_heads]
    out, _, spread, top = orc.attend("e4m3", q, c.k.view(torch.uint8).cpu().numpy(), c.v.view(torch.uint8).cpu().numpy(),
                                     c.k_scale.cpu().numpy(), c.v_scale.cpu().numpy(), reader.table.cpu().numpy(), lens,
                                     model.d ** -0.5)
    # x and q are rounded to bf16 (2^-8 each, and the product's order): scores off by 2^-6 of top at most
    tol = spread * (2 * 2.0 ** -6 * top)[..., None] + np.abs(out) * 2.0 ** -8 + 1e-3 * spread
    got = f64(reader.heads_out)
    assert (np.abs(got - out) <= tol).all()
    # the cache holds what was written: the last token's keys
    k = (x @ f64(block["qkv"]).T).reshape(3, -1, model.d)[:, model.q_heads:model.q_heads + model.heads]
    for i in (0, 2):
        slot = reader.rows[i][(lens[i] - 1) // 16], (lens[i] - 1) % 16
        held = orc.e4m3_values()[c.k.view(torch.uint8)[slot[0], :, slot[1]].cpu().numpy()] * f64(c.k_scale[slot[0], :, slot[1]])[:, None]
        assert (np.abs(held - k[i]) <= np.abs(k[i]).max(axis=-1, keepdims=True) * (2.0 ** -4 + 2.0 ** -6)).all()
