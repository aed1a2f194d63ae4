"""Rotary positions and the cache held in 8 bits as one program uses them: a search of several plies against the plain models, step by step, and the example."""
import os
import random
import sys

import pytest
import torch

import paper_2303_17503_amd as pg
from test_gpu_cache import bits, ints
from test_gpu_cache8 import check_attend, new, ref_of, same
from test_gpu_rotary import check as check_turned

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype,heads,kv_heads,head_dim,page_size,interleaved", [(torch.bfloat16, 8, 2, 64, 16, False), (torch.float16, 6, 3, 96, 32, True), (torch.bfloat16, 40, 2, 32, 16, True)])
def test_a_search_of_several_plies(dtype, heads, kv_heads, head_dim, page_size, interleaved):
    """Games with a prompt, then rounds of: children forked from parents, their queries and keys turned by the child's place, attention that writes the token, some games
    freed, pages moved together, the children read back.  Queries and keys as they were turned go to the plain cache, and are held against 64 bits themselves."""
    r, g = random.Random(heads), torch.Generator("cuda").manual_seed(heads)
    games, layers, T = 9, 2, 40
    cache = pg.PagedCache.empty(3 * games, 400, 96, layers, kv_heads, head_dim, page_size, dtype, bits=8)
    cache.kv.view(torch.uint8).zero_()
    ref = ref_of(cache)
    f = pg.rotary_frequencies(head_dim // 2)
    counts = [r.randint(1, T) for _ in range(games)]
    cache.advance(ints(range(games)), ints(counts))
    ref.advance(range(games), counts)
    places = torch.arange(T, dtype=torch.int32, device="cuda").expand(games, T)
    for layer in range(layers):
        product = new(g, dtype, games, T, 2 * kv_heads * head_dim, size=2.0 ** (layer - 1))
        k, v = product[..., : kv_heads * head_dim].unflatten(-1, (kv_heads, head_dim)), product[..., kv_heads * head_dim:].unflatten(-1, (kv_heads, head_dim))
        turned = pg.rotate(k, places, f, interleaved=interleaved)
        check_turned(turned, k, places, f, interleaved, 1.0, False)
        cache.write(layer, turned, v, ints(range(games)))
        ref.write(layer, turned, v, range(games))
    same(cache, ref)
    for ply in range(4):
        parents = [r.randrange(games) if ply % 2 == 0 else games + r.randrange(games) for _ in range(games)]
        children = list(range(games, 2 * games)) if ply % 2 == 0 else list(range(2 * games, 3 * games))
        parents = [p if int(ref.lengths[p]) else 0 for p in parents]
        cache.fork(ints(parents), ints(children))
        ref.fork(parents, children)
        positions = cache.lengths[torch.tensor(children, device="cuda")]
        cache.advance(ints(children))
        ref.advance(children, [1] * games)
        for layer in range(layers):
            q, k = new(g, dtype, games, heads, head_dim), new(g, dtype, games, kv_heads, head_dim, size=2.0 ** r.randint(-2, 2))
            v = new(g, dtype, games, kv_heads, head_dim, size=2.0 ** r.randint(-2, 2))
            qt, kt = pg.rotate((q, k), positions, f, interleaved=interleaved)
            check_turned(qt, q, positions, f, interleaved, 1.0, False)
            check_turned(kt, k, positions, f, interleaved, 1.0, False)
            out, lse = cache.attend(layer, qt, ints(children), k=kt, v=v, lse=True)
            ref.write_last(layer, kt, v, children)
            check_attend(cache, ref, out, lse, layer, qt, children, head_dim ** -0.5)
        same(cache, ref)
        gone = r.sample(range(games), 2)
        cache.free(ints(gone))
        ref.free(gone)
        cache.compact()
        ref.compact()
        same(cache, ref)
        k, v = cache.read(1, 96, ints(children))
        want = ref.read(1, 96, children, [0] * games, dtype)
        assert torch.equal(bits(k), bits(want[0])) and torch.equal(bits(v), bits(want[1]))


@pytest.mark.parametrize("rotary,bits_", [(True, 8), (True, 16), (False, 8)])
def test_the_example_runs(rotary, bits_):
    """self-play, a learning step and an expansion; and the features of a ply by the calls one after the other are those of the step that does all at once"""
    import sequence_policy as sp

    games, size, plies = 16, 9, 40
    policy = sp.SequencePolicy(82, 162, dim=64, seed=3, rotary=rotary, bits=bits_)
    batch = sp.self_play(policy, games, size, plies, seed=5)
    cache, begun = batch["cache"], batch["begun"].tolist()
    assert int(batch["env"].export_state()["illegal"].sum()) == 0 and torch.isfinite(batch["features"].float()).all()
    assert cache.lengths.tolist() == [plies - b for b in begun] and (cache.scales is None) == (bits_ == 16)
    assert torch.isfinite(sp.learn(policy, batch))
    again = pg.PagedCache(*(t.clone() for t in (cache.kv, cache.table, cache.lengths, cache.refs)), **({} if bits_ == 16 else dict(scales=cache.scales.clone(), dtype=policy.out.dtype)))
    tokens = batch["tokens"]
    got = policy.features(cache, tokens)
    again.advance()
    places = again.lengths - 1
    x = policy.embed(tokens, places)
    for i in range(policy.layers):
        q, k, v = policy.split(i, x)
        if rotary: q, k = pg.rotate(q, places, policy.frequencies), pg.rotate(k, places, policy.frequencies)
        again.write(i, k, v)
        x = policy.finish(i, x, again.attend(i, q))
    assert torch.equal(policy.norm(x), got)
    pool = pg.GoEnv(2 * games, size, seed=1)
    tree = policy.new_cache(2 * games, 8 * games, 162)
    roots = torch.arange(games, device="cuda", dtype=torch.int32)
    logits = policy.logits(policy.features(tree, torch.full((games,), policy.start, dtype=torch.int32, device="cuda"), roots))
    moves, _ = pg.sample_actions(logits, mask=pool.legal_mask()[:games])
    priors, _, _ = sp.expand(policy, pool, tree, roots, moves, roots + games, moves)
    mask = pool.mask_view(pool.legal_mask())[games:]
    assert torch.equal(torch.isfinite(priors), mask != 0)


def test_distance_is_what_counts():
    """scores of turned queries and keys depend on how far apart they are: the same game further on attends alike, up to the roundings of its keys and queries"""
    g = torch.Generator("cuda").manual_seed(2)
    n, D = 30, 64
    q, k, v = (torch.randn(n if i else 1, 2, D, generator=g, device="cuda") for i in range(3))
    f, outs = pg.rotary_frequencies(D), []
    for shift in (0, 1000, 100000):
        cache = pg.PagedCache.empty(1, 4, 64, 1, 2, D, dtype=torch.float16, bits=16)
        cache.advance(counts=n)
        kt = pg.rotate(k, torch.arange(n, dtype=torch.int32, device="cuda") + shift, f).half()
        cache.write(0, kt[None], v[None].half())
        qt = pg.rotate(q, ints([n - 1 + shift]), f).half()
        outs.append(cache.attend(0, qt).double())
    # a key's and a query's roundings, 2^-11 each of their elements, move a score by at most 2 * 2^-11 |q| |k| / 8, a probability by twice that of itself, an output by as much of the largest |v|; and its own rounding
    most = float(q.norm(dim=-1).max() * k.norm(dim=-1).max()) / 8
    for out in outs[1:]:
        assert (out - outs[0]).abs().max() <= 2 * (2 * 2 * 2.0 ** -11 * most * float(v.abs().max())) + 2 * 2.0 ** -11 * float(v.abs().max())
