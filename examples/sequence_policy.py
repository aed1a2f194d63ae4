#!/usr/bin/env python3
"""A policy that reads a Go game as its sequence of moves, on the environments and operators of this library.

  self-play   every ply: room for a token in each game's cache slot, the layers' attention over the moves so far (which writes the new
              token's keys and values), logits, a legal move drawn from them, the environment's step; a game that ended gives its pages back
  learning    the recorded moves weighted by their games' results: loss and gradient of the logits, a step on the output weights
  search      one expansion per game in a pool of state slots: the environment's state and the cache's slot are copied together,
              the new states' move probabilities are the children's priors

A move's place in its game is learned as a table of vectors or, with --rotary, turned into queries and keys; with --bits 8 the cache holds keys and values in half the memory.
The network is small and its weights are random: what is shown is how the calls fit together.  `python examples/sequence_policy.py`
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2303_17503_amd as pg  # noqa: E402


class SequencePolicy:
    """A small transformer over move tokens: 0 .. N*N the moves, N*N + 1 the beginning of a game."""

    def __init__(self, actions, max_plies, layers=2, heads=8, kv_heads=2, head_dim=64, dim=128, seed=0, dtype=torch.bfloat16, device="cuda",
                 rotary=False, bits=16):
        g = torch.Generator(device).manual_seed(seed)
        new = lambda *s: (torch.randn(*s, generator=g, device=device) * s[0] ** -0.5).to(dtype)  # noqa: E731
        self.actions, self.start, self.layers, self.heads, self.kv_heads, self.head_dim = actions, actions, layers, heads, kv_heads, head_dim
        self.move = new(actions + 1, dim) * dim ** 0.5
        self.ply = new(max_plies + 1, dim) * dim ** 0.5
        self.qkv = [new(dim, (heads + 2 * kv_heads) * head_dim) for _ in range(layers)]
        self.back = [new(heads * head_dim, dim) for _ in range(layers)]
        self.up, self.down = [new(dim, 4 * dim) for _ in range(layers)], [new(4 * dim, dim) for _ in range(layers)]
        self.out = new(dim, actions)
        self.frequencies = pg.rotary_frequencies(head_dim, device=device) if rotary else None
        self.bits = bits

    def split(self, layer, x):
        """query, key and value heads of one product, as views into it"""
        h, kv, d = self.heads, self.kv_heads, self.head_dim
        y = self.norm(x) @ self.qkv[layer]
        return y[:, :h * d].unflatten(1, (h, d)), y[:, h * d:(h + kv) * d].unflatten(1, (kv, d)), y[:, (h + kv) * d:].unflatten(1, (kv, d))

    @staticmethod
    def norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(1, keepdim=True) + 1e-6)).to(x.dtype)

    def embed(self, tokens, plies):
        x = self.move[tokens.long()]
        return x if self.frequencies is not None else x + self.ply[plies.long()]

    def finish(self, layer, x, attended):
        x = x + attended.flatten(1) @ self.back[layer]
        return x + torch.relu(self.norm(x) @ self.up[layer]) @ self.down[layer]

    def features(self, cache, tokens, slots=None):
        """The newest token of each slot, [n][dim], with its keys and values written to the cache: one launch per layer beside the products."""
        cache.advance(slots)
        lengths = cache.lengths if slots is None else cache.lengths[slots.clamp(min=0).long()]
        plies = lengths - 1
        x = self.embed(tokens, plies)
        for i in range(self.layers):
            q, k, v = self.split(i, x)
            if self.frequencies is not None:
                q, k = pg.rotate((q, k), plies, self.frequencies)
            x = self.finish(i, x, cache.attend(i, q, slots, k=k, v=v))
        return self.norm(x)

    def logits(self, features):
        return features @ self.out

    def new_cache(self, slots, pages, max_plies, page_size=16):
        return pg.PagedCache.empty(slots, pages, max_plies + 1, self.layers, self.kv_heads, self.head_dim, page_size, self.out.dtype, bits=self.bits)


def gumbel(shape, g):
    return -torch.log(-torch.log(torch.rand(shape, generator=g, device="cuda").clamp(1e-7, 1 - 1e-7)))


def self_play(policy, games, size, plies, seed=0, explore=30):
    """A recorded batch: moves [plies][games], log-probabilities, legal masks, features, results for the player who moved."""
    most = 2 * size * size
    env = pg.GoEnv(games, size, seed=seed, auto_reset=True, line_padded=True)
    mask, rewards = env.new_mask(), torch.zeros(games, 2, device="cuda")
    terminated = torch.zeros(games, dtype=torch.uint8, device="cuda")
    env.bind_outputs(mask, None, rewards, terminated)
    cache = policy.new_cache(games, games * ((most + 16) // 16), most)
    g = torch.Generator("cuda").manual_seed(seed)
    every = torch.arange(games, device="cuda", dtype=torch.int32)
    tokens = torch.full((games,), policy.start, dtype=torch.int32, device="cuda")
    moves = torch.full((plies, games), -1, dtype=torch.int32, device="cuda")
    begun = torch.zeros(games, dtype=torch.int32, device="cuda")     # the recorded ply at which the present game began
    game_of = torch.zeros(plies, games, dtype=torch.int64, device="cuda")
    players = torch.zeros(plies, games, dtype=torch.uint8, device="cuda")
    results = torch.zeros(plies + 1, games, 2, device="cuda")        # of the game that is the i-th of its column
    logps, masks, seen = [], [], []
    game = torch.zeros(games, dtype=torch.int64, device="cuda")
    for t in range(plies):
        env.current_player(players[t])
        x = policy.features(cache, tokens)
        # moves are drawn in the opening and chosen later; a point that was played in this game already is less attractive
        temperature = torch.where(t - begun < explore, 1.0, 0.0)
        actions, logp = pg.sample_actions(policy.logits(x), noise=gumbel((games, env.A), g), mask=mask, record=moves.t(), begin=begun,
                                          end=torch.full_like(begun, t), presence=0.5, temperature=temperature)
        masks.append(mask.clone()); logps.append(logp); seen.append(x); game_of[t] = game
        moves[t] = actions
        env.step(actions)
        over = terminated != 0
        results[game, torch.arange(games, device="cuda")] = rewards
        cache.free(torch.where(over, every, -1))
        tokens = torch.where(over, policy.start, actions)
        begun = torch.where(over, t + 1, begun)
        game = game + over
    result = results.gather(0, game_of[:, :, None].expand(-1, -1, 2)).gather(2, players.long()[:, :, None])[:, :, 0]
    return {"env": env, "cache": cache, "moves": moves, "logp": torch.stack(logps), "mask": torch.stack(masks), "features": torch.stack(seen), "result": result,
            "begun": begun, "tokens": tokens}


def learn(policy, batch, rate=0.1, entropy=0.01):
    """One step of policy gradient on the output weights; returns the mean loss before it."""
    rows = batch["moves"].numel()
    features, mask = batch["features"].flatten(0, 1), batch["mask"].flatten(0, 1)
    loss, _, grad = pg.policy_loss(policy.logits(features), batch["moves"].flatten(), weight=batch["result"].flatten().contiguous(), entropy=entropy,
                                   grad_scale=1.0 / rows, mask=mask)
    policy.out = (policy.out.float() - rate * (features.t().float() @ grad.float())).to(policy.out.dtype)
    return loss.mean()


def expand(policy, env, cache, parents, actions, children, tokens):
    """One expansion per entry of a pool: children[i] = the state after actions[i] in parents[i].  Returns the children's log-priors, with
    the moves' legality from the environment, their rewards and whether they ended."""
    n = parents.shape[0]
    mask = torch.empty(n, env.mask_pitch, dtype=torch.uint8, device="cuda")
    rewards, terminated = torch.zeros(n, 2, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    env.step_slots(parents, actions, children, mask=mask, rewards=rewards, terminated=terminated)
    cache.fork(parents, children)
    x = policy.features(cache, tokens, children)
    return pg.adjust_logits(policy.logits(x), mask=mask, normalize=True), rewards, terminated


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--games", type=int, default=256)
    ap.add_argument("--size", type=int, default=9, choices=(9, 19))
    ap.add_argument("--plies", type=int, default=200)
    ap.add_argument("--rotary", action="store_true")
    ap.add_argument("--bits", type=int, default=16, choices=(8, 16))
    a = ap.parse_args()
    policy = SequencePolicy(a.size * a.size + 1, 2 * a.size * a.size, rotary=a.rotary, bits=a.bits)
    batch = self_play(policy, a.games, a.size, a.plies)
    print(f"self-play: {a.games} games, {a.plies} plies, {int((batch['result'] != 0).sum())} moves of finished games, "
          f"mean log-probability {float(batch['logp'].mean()):.3f}, {int((batch['cache'].refs > 0).sum())} pages in use")
    print(f"learning: mean loss {float(learn(policy, batch)):.4f}")
    # a tree's first expansions, from the beginning of each game: slot 2 i its root, 2 i + 1 the child
    pool = pg.GoEnv(2 * a.games, a.size, seed=1)
    cache = policy.new_cache(2 * a.games, 8 * a.games, 2 * a.size * a.size)
    roots = torch.arange(0, 2 * a.games, 2, device="cuda", dtype=torch.int32)
    start = torch.full((a.games,), policy.start, dtype=torch.int32, device="cuda")
    logits = policy.logits(policy.features(cache, start, roots))
    moves, _ = pg.sample_actions(logits, noise=gumbel(logits.shape, torch.Generator("cuda").manual_seed(2)), mask=pool.legal_mask()[roots.long()])
    priors, _, _ = expand(policy, pool, cache, roots, moves, roots + 1, moves)
    print(f"search: {a.games} expansions, entropy of the children's priors {float(-(priors.exp() * priors.clamp(min=-1e9)).sum(1).mean()):.3f}")


if __name__ == "__main__":
    main()
