"""The operators as one program uses them (examples/sequence_policy.py): self-play, learning and a search's expansions on the Go environment,
each held against the whole sequence computed at once in plain form."""
import os
import sys

import pytest
import torch

import paper_2303_17503_amd as pg

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def whole(policy, tokens):
    """The last token's features from all tokens of one game at once, plain attention in 64 bits between the policy's own products."""
    n = len(tokens)
    x = policy.embed(torch.tensor(tokens, device="cuda"), torch.arange(n, device="cuda"))
    for i in range(policy.layers):
        q, k, v = (t.double() for t in policy.split(i, x))
        group = policy.heads // policy.kv_heads
        out = torch.empty_like(q)
        for t in range(n):
            for h in range(policy.heads):
                p = torch.softmax((k[: t + 1, h // group] * q[t, h]).sum(1) * policy.head_dim ** -0.5, 0)
                out[t, h] = (p[:, None] * v[: t + 1, h // group]).sum(0)
        x = policy.finish(i, x, out.to(x.dtype))
    return policy.norm(x)[-1].float()


def near(a, b):
    """Two ways of summing in bfloat16 (products of one row and of many): a few roundings of 2^-8 of the features' size, which the norm makes 1."""
    return float((a.float() - b).norm() / b.norm()) < 4 * 2.0 ** -8


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_self_play_and_learning(dtype):
    import sequence_policy as sp

    games, size, plies = 24, 9, 45
    policy = sp.SequencePolicy(82, 162, dim=64, seed=3, dtype=dtype)
    batch = sp.self_play(policy, games, size, plies, seed=5)
    assert int(batch["env"].export_state()["illegal"].sum()) == 0
    moves, begun, cache = batch["moves"], batch["begun"].tolist(), batch["cache"]
    assert (moves >= 0).all() and (batch["mask"].gather(2, moves.long()[:, :, None]) == 1).all()
    assert cache.lengths.tolist() == [plies - b for b in begun] and int((cache.refs > 0).sum()) == sum(-(-(plies - b) // 16) for b in begun)
    for e in (0, 7, games - 1):
        if begun[e] < plies:
            tokens = [policy.start] + moves[begun[e]: plies - 1, e].tolist()
            assert near(batch["features"][-1, e], whole(policy, tokens))
    # the learner's step is the gradient of its loss: the loss falls by the rate times the gradient's square, to first order
    batch["result"] = torch.where(torch.rand(plies, games, generator=torch.Generator("cuda").manual_seed(1), device="cuda") < 0.5, 1.0, -1.0)
    before = policy.out.clone()
    first = float(sp.learn(policy, batch, rate=0.5))
    step = (before.float() - policy.out.float()) / 0.5
    second = float(sp.learn(policy, batch, rate=0.0))
    fall = first - second
    assert 0.5 * 0.5 * float(step.square().sum()) < fall < 0.5 * 1.5 * float(step.square().sum())


def test_a_search_copies_states_and_caches_together():
    import sequence_policy as sp

    n, size, depth = 30, 9, 20
    policy = sp.SequencePolicy(82, 162, dim=64, seed=4)
    env = pg.GoEnv(3 * n, size, seed=2)
    cache = policy.new_cache(3 * n, 3 * n * 3, 162)
    roots = torch.arange(n, device="cuda", dtype=torch.int32)
    g = torch.Generator("cuda").manual_seed(1)
    token = torch.full((n,), policy.start, dtype=torch.int32, device="cuda")
    played = [[policy.start] for _ in range(n)]
    everyone = torch.full((3 * n,), -1, dtype=torch.int32, device="cuda")
    for _ in range(depth):
        x = policy.features(cache, token, roots)
        token, _ = pg.sample_actions(policy.logits(x), noise=sp.gumbel((n, 82), g), mask=env.legal_mask()[:n])
        everyone[:n] = token
        env.step(everyone)
        for i, a in enumerate(token.tolist()):
            played[i].append(a)
    policy.features(cache, token, roots)
    x = policy.embed(token, cache.lengths[:n] - 1)          # (the newest move is in the cache now)
    # two children of each root, by different moves, then a grandchild of the first in the place of the second
    legal = env.mask_view(env.legal_mask())[:n].float()
    pair = torch.multinomial(legal, 2, generator=g).int()
    first, second = roots + n, roots + 2 * n
    a = sp.expand(policy, env, cache, roots, pair[:, 0].contiguous(), first, pair[:, 0])[0]
    b = sp.expand(policy, env, cache, roots, pair[:, 1].contiguous(), second, pair[:, 1])[0]
    mask = env.mask_view(env.legal_mask())
    assert torch.equal(torch.isfinite(a), mask[n:2 * n] != 0) and torch.equal(torch.isfinite(b), mask[2 * n:] != 0)
    best = a.argmax(1).int()
    c = sp.expand(policy, env, cache, first, best, second, best)[0]
    for i in (0, 11, n - 1):
        line = played[i] + [int(pair[i, 0]), int(best[i])]
        want = policy.logits(whole(policy, line).to(policy.out.dtype)[None]).float()[0]
        live = torch.isfinite(c[i])
        assert near(c[i][live], torch.log_softmax(want[live], 0))
    assert (cache.lengths[:n] == depth + 1).all() and (cache.lengths[second.long()] == depth + 3).all()
    cache.free(torch.cat([first, second]))
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache.compact(used)
    assert int(used) == n * -(-(depth + 1) // 16) and int(cache.refs[: int(used)].min()) == 1
    again = policy.features(cache, token, roots)
    assert torch.isfinite(again.float()).all() and x.shape == again.shape
