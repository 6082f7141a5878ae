"""The example's beam search with the library's own cache and attention."""
import os
import sys

import pytest
import torch

from wg_workloads import flatten, grammars, make_vocab

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("storage", ["bf16", "e4m3", "int8"])
def test_the_example_runs(storage):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import beam_search as ex
    import paper_2507_16768_b200 as wg
    vocab = make_vocab(2000, seed=1)
    grammar = wg.Grammar(flatten(grammars.json_reference_lookup(doc_nodes=30)))
    prompts, steps, K = [[11, 12, 13], list(range(40, 61))], 40, 4
    most = 21 + steps + 1
    cache = ex.LibraryCache(2 * K, most, 2 * K * (-(-most // ex.BLOCK) + 1), K, storage)
    out, score, finished = ex.search(ex.ToyModel(vocab), vocab, grammar, prompts, K, steps, cache)
    assert out.shape == (2, K, steps) and (out >= 0).any() and (out < vocab.size).all()
    assert torch.isfinite(score).any() and not torch.isnan(score).any()
    # every hypothesis obeys the grammar, token by token
    tokens = vocab.tokens()
    for line in out.reshape(-1, steps).tolist():
        state = grammar.start_state
        for t in line:
            if t < 0:
                break
            state = grammar.step_token(state, t, [256] if t == vocab.eos_id else list(tokens[t]))
            assert state != 0


def test_attention_steps_agree_with_the_plain_cache():
    """The same tokens appended to both caches: the library's context is the plain one's, up to the roundings to bf16 (the plain
    one rotates nothing, so that all positions are taken to be the first)."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import beam_search as ex
    vocab = make_vocab(500, seed=1)
    model = ex.ToyModel(vocab)
    plain, own = ex.PagedCache(4, 40, 16), ex.LibraryCache(4, 40, 16, 2)
    own.rope.table[:, :ex.DIM // 2], own.rope.table[:, ex.DIM // 2:] = 1.0, 0.0
    n_new = torch.tensor([5, 0, 17, 1], dtype=torch.int32, device="cuda")
    tokens = torch.arange(23, device="cuda") * 7 % 500
    for cache in (plain, own):
        cache.append(n_new, tokens, model)
    last = torch.tensor([4, 0, 21, 22], device="cuda")
    keys, values = plain.read()
    e = model.embed[tokens[last]].to(torch.bfloat16).double()
    k, v = keys.to(torch.bfloat16).double(), values.to(torch.bfloat16).double()
    w = (k @ e[:, :, None])[:, :, 0]
    w = torch.softmax(torch.where(torch.arange(w.shape[1], device="cuda")[None] < n_new[:, None], w, -1e30), 1)
    want = (w[:, :, None] * v).sum(1)
    want[1] = 0.0
    mass = (w[:, :, None] * v.abs()).sum(1)
    got = own.attend().double()
    # a weight and the result are rounded to bf16; scores are sums of 64 products in fp32
    size = (k.abs() @ e.abs()[:, :, None]).amax(1)
    assert ((got - want).abs() <= want.abs() * 2.0 ** -8 + mass * (2.0 ** -8 + 2 * size * 80 * 2.0 ** -23 + 2.0 ** -18)).all()
