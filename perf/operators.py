"""The operators of a policy that plays the games of this library as sequences of moves, as cases that can be timed and compared.

Between the environment's outputs and its next actions such a policy turns logits into moves (`adjust`, `sample`), learns from
recorded moves (`loss`), reads the keys and values of a game's earlier moves from a paged cache (`attend`), and has the cache's
slots follow the games through a tree search and through the end of games (`search`, `expand`, `turnover`).

  adjust    logits less penalties for repeated moves, plus a bias, over a temperature, illegal moves at -inf; as log-probabilities too
  sample    the same, and the move with the largest sum of that and the given Gumbel noise, with its log-probability
  loss      cross entropy against a search's visit distribution or a played move, with an entropy bonus, and the logits' gradient
  attend    one new token of each sequence over the keys and values that its pages hold
  search    one leaf of each game: a slot becomes a copy of its parent's (full pages are shared), grows by a token, which is written
  expand    the same with the layers' attention over it, which writes the token itself
  turnover  games end, the pages in use move to the front of the pool, and as many new games come in with their first moves

With `own` false everything is computed in elementary torch operations in 32 bits; with `own` true by the library's calls.
"""
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
REPETITION, FREQUENCY, PRESENCE = 1.25, 0.1, 0.2
ENTROPY = 0.01
GROUPS = 8          # a turnover replaces one game in eight
NEG = float("-inf")


def _policy(name, kind, rows, actions, dtype, **more):
    c = {"kind": kind, "rows": rows, "actions": actions, "dtype": dtype, "mask": "tight", "bias": False, "record": 0,
         "time_major": False, "temperature": False, "normalize": False, "target": "none"}
    c.update(more)
    return {"name": name, **c} if name else c


def _cache(name, kind, slots, lo, hi, dtype, heads, kv_heads, head_dim, page, layers=1):
    c = {"kind": kind, "slots": slots, "lo": lo, "hi": hi, "dtype": dtype, "heads": heads, "kv_heads": kv_heads,
         "head_dim": head_dim, "page": page, "layers": layers}
    return {"name": name, **c} if name else c


def listed():
    return [
        # an actor with a handful of 9x9 games: a launch and a row's latency are everything
        _policy("sample-go9-256", "sample", 256, 82, "f32"),
        # the largest batch of full-size games, discouraged from repeating the moves of the recorded trajectory [plies][games]
        _policy("sample-go19-65536", "sample", 65536, 362, "bf16", mask="lines", record=361, time_major=True, temperature=True),
        # priors of a batched search on Hex, an opening bias shared by all games
        _policy("adjust-hex-16384", "adjust", 16384, 122, "f16", bias=True, normalize=True),
        # full-size games with their move lists [games][plies], a ragged batch
        _policy("adjust-go19-5001", "adjust", 5001, 362, "bf16", record=200, temperature=True),
        # a learner's minibatch against visit distributions
        _policy("loss-go9-4096", "loss", 4096, 82, "f32", target="visits"),
        # a learner's pass over recorded moves of the largest batch
        _policy("loss-go19-65536", "loss", 65536, 362, "bf16", mask="lines", target="moves"),
        # one full-length game of 19x19, alone: latency, and the length split over the machine
        _cache("attend-one-722", "attend", 1, 722, 722, "bf16", 8, 2, 64, 16),
        # the games of a large self-play worker, of every age
        _cache("attend-go19-4096", "attend", 4096, 1, 722, "bf16", 8, 2, 64, 16),
        # few long sequences, as many key heads as query heads
        _cache("attend-long-3", "attend", 3, 90001, 131072, "f16", 8, 8, 128, 64),
        # one simulation of the search of 4096 full-size games
        _cache("search-go19-4096", "search", 4096, 60, 500, "bf16", 8, 2, 64, 16, layers=2),
        # one simulation of a 9x9 worker with its attention
        _cache("expand-go9-1024", "expand", 1024, 1, 160, "f16", 8, 2, 64, 16, layers=2),
        # 256 of 2048 full-size games are replaced by new ones in mid-game
        _cache("turnover-go19-2048", "turnover", 2048, 60, 500, "bf16", 8, 2, 64, 16, layers=2),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm; odd more often than not."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    return min(hi, n | 1) if rng.random() < 0.6 else n


def draw(rng):
    most = max(max(work(c)["bytes"] for c in listed() if (c["kind"] in ("adjust", "sample", "loss")) == p) for p in (True, False))
    while True:
        kind = rng.choice(["sample", "adjust", "loss", "attend", "attend", "search", "expand", "turnover"])
        if kind in ("sample", "adjust", "loss"):
            actions = rng.choice([82, 122, 362, _between(rng, 1, 1500)])
            record = 0 if kind == "loss" or rng.random() < 0.4 else _between(rng, 1, 722)
            c = _policy(None, kind, _between(rng, 1, 65536), actions, rng.choice(["f32", "bf16", "f16"]),
                        mask=rng.choice(["tight", "lines", "none"]), bias=rng.random() < 0.4, record=record,
                        time_major=record > 0 and rng.random() < 0.5, temperature=rng.random() < 0.5,
                        normalize=kind == "adjust" and rng.random() < 0.5,
                        target=rng.choice(["visits", "moves"]) if kind == "loss" else "none")
        else:
            kv_heads, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 8])
            shape = (rng.choice(["bf16", "f16"]), kv_heads * group, kv_heads, rng.choice([32, 64, 64, 128]), rng.choice([16, 32, 64]))
            if kind == "attend":
                hi = _between(rng, 1, 131072)
                c = _cache(None, kind, _between(rng, 1, 4096), rng.randint(0, hi), hi, *shape)
            else:
                hi = _between(rng, 20, 722)
                slots = _between(rng, GROUPS, 4096)
                slots -= slots % GROUPS if kind == "turnover" else 0
                c = _cache(None, kind, slots, rng.randint(0, hi), hi, *shape, layers=rng.randint(1, 2))
        held = 0 if "rows" in c else c["slots"] * c["hi"] * _token_bytes(c)
        if work(c)["bytes"] <= most and held <= 4e9 and (kind != "attend" or c["slots"] * c["hi"] * c["kv_heads"] * c["head_dim"] <= 1e9):
            return c


def _token_bytes(case):
    return 2 * case["layers"] * case["kv_heads"] * case["head_dim"] * BYTES[case["dtype"]]


def _pages(tokens, page):
    return (tokens + page - 1) // page


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    g = torch.Generator("cuda").manual_seed(seed)
    if "rows" in case:
        _prepare_policy(s, case, g)
    else:
        _prepare_cache(s, case, g)
    return s


def _prepare_policy(s, case, g):
    B, A, T = case["rows"], case["actions"], case["record"]
    rand = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    whole = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    s.logits = (normal(B, A) * 2).to(DTYPES[case["dtype"]])
    s.mask = s.bias = s.record = s.begin = s.end = s.temperature = None
    if case["mask"] != "none":   # the environment's buffer: boards of every age, and a game in 500 in which nothing can be played
        pitch = A if case["mask"] == "tight" else (A + 127) // 128 * 128
        s.mask = torch.zeros(B, pitch, dtype=torch.uint8, device="cuda")
        s.mask[:, :A] = rand(B, A) < rand(B, 1)
        s.mask[:, A - 1] = 1
        s.mask[rand(B) < 0.002] = 0
    if case["bias"]:
        s.bias = normal(A) * 0.5
    if T:   # a game's moves so far: those from begin to end, -1 where it did not move
        moves = torch.minimum(whole(0, A, T, B) if case["time_major"] else whole(0, A, B, T).t(), whole(0, 4 * A, T, 1))
        moves = torch.where(rand(T, B) < 0.01, torch.full_like(moves, -1), moves)
        s.record = moves.contiguous().t() if case["time_major"] else moves.t().contiguous()
        s.begin = (rand(B) * T * 0.2).int()
        s.end = T - (rand(B) * T * 0.2).int()
    if case["temperature"]:   # the moves of a game's beginning are drawn, the later ones nearly or wholly greedy
        s.temperature = torch.where(rand(B) < 0.3, torch.where(rand(B) < 0.5, 0.0, 0.25), 1.0)
    if case["kind"] == "sample":
        s.noise = -torch.log(-torch.log(rand(B, A).clamp(1e-7, 1 - 1e-7)))
    if case["kind"] == "loss":
        s.weight = normal(B)
        if case["target"] == "visits":
            visits = torch.floor(rand(B, A).pow(8) * 32)
            s.target = visits / visits.sum(1, keepdim=True).clamp(min=1)
        else:
            s.target = whole(-1, A, B)


def _prepare_cache(s, case, g):
    n, lo, hi, P, layers = case["slots"], case["lo"], case["hi"], case["page"], case["layers"]
    H, KV, D, dtype = case["heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    kind = case["kind"]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    whole = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    children = kind in ("search", "expand")
    slots, width = 2 * n if children else n, _pages(hi + 1, P)
    s.lengths = torch.zeros(slots, dtype=torch.int32, device="cuda")
    s.lengths[:n] = whole(lo, hi + 1, n)
    need = _pages(s.lengths[:n].long(), P)
    used = int(need.sum())
    pages = used + 5 if kind == "attend" else n * width + 3 * n * children + 5
    s.kv = normal(pages, layers, 2, KV, P, D)
    s.table = torch.full((slots, width), -1, dtype=torch.int32, device="cuda")
    # pages in the order in which games that grew side by side took them: none
    order = torch.randperm(used if kind == "turnover" else pages, generator=g, device="cuda")[:used].int()
    s.table[:n][torch.arange(width, device="cuda") < need[:, None]] = order
    s.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    s.refs[order.long()] = 1
    if kind == "attend":
        s.q = normal(n, H, D)
    if children:
        s.src, s.dst = whole(0, n, n), torch.arange(n, 2 * n, device="cuda", dtype=torch.int32)
        s.q, s.k, s.v = normal(layers, n, H, D), normal(layers, n, KV, D), normal(layers, n, KV, D)
    if kind == "turnover":
        m, s.passes = n // GROUPS, 0
        s.groups = torch.randperm(n, generator=g, device="cuda").int().reshape(GROUPS, m)
        s.counts = whole(lo, hi + 1, m)
        s.k, s.v = normal(layers, m, hi, KV, D), normal(layers, m, hi, KV, D)
    s.cache = None


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2303_17503_amd as pg

    c = s.case
    if "rows" in c:
        how = dict(mask=s.mask, bias=s.bias, temperature=s.temperature)
        if s.record is not None:
            how.update(record=s.record, begin=s.begin, end=s.end, repetition=REPETITION, frequency=FREQUENCY, presence=PRESENCE)
        if c["kind"] == "adjust":
            return pg.adjust_logits(s.logits, normalize=c["normalize"], **how)
        if c["kind"] == "sample":
            return pg.sample_actions(s.logits, noise=s.noise, **how)
        return pg.policy_loss(s.logits, s.target, weight=s.weight, entropy=ENTROPY, grad_scale=1.0 / c["rows"], **how)
    if s.cache is None:   # the handle that a program keeps; the memory is the program's
        s.cache = pg.PagedCache(s.kv, s.table, s.lengths, s.refs)
    cache = s.cache
    if c["kind"] == "attend":
        return cache.attend(0, s.q, lse=True)
    out = []
    if c["kind"] == "turnover":
        group = s.groups[s.passes % GROUPS]
        s.passes += 1
        cache.free(group)
        cache.compact()
        cache.advance(group, s.counts)
        for i in range(c["layers"]):
            cache.write(i, s.k[i], s.v[i], group)
    else:
        cache.fork(s.src, s.dst)
        cache.advance(s.dst)
        for i in range(c["layers"]):
            if c["kind"] == "search":
                cache.write(i, s.k[i], s.v[i], s.dst)
            else:
                out.append(cache.attend(i, s.q[i], s.dst, k=s.k[i], v=s.v[i]))
    return out, s.kv, s.table, s.lengths, s.refs


# ---- the plain forms ------------------------------------------------------------------------------------------------


def _adjusted(s):
    """(logits as adjusted, which moves are possible, d adjusted / d logits)"""
    c, A = s.case, s.case["actions"]
    z = s.logits.float()
    slope = torch.ones_like(z)
    if s.record is not None:
        T = c["record"]
        t = torch.arange(T, device="cuda")
        counts = (t >= s.begin[:, None]) & (t < s.end[:, None]) & (s.record >= 0) & (s.record < A)
        times = torch.zeros_like(z).scatter_add_(1, s.record.long().clamp(0, A - 1), counts.float())
        rate = torch.full_like(z, REPETITION)
        slope = torch.where(times > 0, torch.where(z > 0, 1 / rate, rate), slope)
        z = torch.where(times > 0, torch.where(z > 0, z / rate, z * rate), z)
        z = z - times * FREQUENCY
        z = torch.where(times > 0, z - PRESENCE, z)
    if s.bias is not None:
        z = z + s.bias
    if s.temperature is not None:
        over = torch.where(s.temperature > 0, s.temperature, 1.0)[:, None].expand_as(z)
        z, slope = z / over, slope / over
    if s.mask is not None:
        z = torch.where(s.mask[:, :A] != 0, z, NEG)
    return z, z > NEG, slope


def _log_softmax(z, possible):
    top = z.amax(1, keepdim=True)
    top = torch.where(top > NEG, top, 0.0)
    total = torch.exp(z - top).sum(1, keepdim=True)
    return torch.where(possible, z - top - torch.log(total), NEG)


def _run_plain(s):
    c = s.case
    if c["kind"] == "adjust":
        z, possible, _ = _adjusted(s)
        return _log_softmax(z, possible) if c["normalize"] else z
    if c["kind"] == "sample":
        return _sample(s)
    if c["kind"] == "loss":
        return _loss(s)
    if c["kind"] == "attend":
        return _attend(s, 0, s.q, s.table, s.lengths)
    out = []
    if c["kind"] == "turnover":
        group = s.groups[s.passes % GROUPS].long()
        s.passes += 1
        _free(s, group)
        _compact(s)
        _advance(s, group, s.counts)
        _write(s, s.k, s.v, group, s.counts)
    else:
        dst = s.dst.long()
        _fork(s, s.src.long(), dst)
        _advance(s, dst, torch.ones_like(s.dst))
        _write(s, s.k[:, :, None], s.v[:, :, None], dst, torch.ones_like(s.dst))
        if c["kind"] == "expand":
            out = [_attend(s, i, s.q[i], s.table[dst], s.lengths[dst])[0] for i in range(c["layers"])]
    return out, s.kv, s.table, s.lengths, s.refs


def _sample(s):
    z, possible, _ = _adjusted(s)
    drawn = z + s.noise
    if s.temperature is not None:   # temperature 0: the largest logit, no noise
        drawn = torch.where(s.temperature[:, None] > 0, drawn, z)
    best = drawn.amax(1, keepdim=True)
    first = torch.where(possible & (drawn == best), torch.arange(z.shape[1], device="cuda"), z.shape[1]).amin(1)
    some = possible.any(1)
    logp = _log_softmax(z, possible).gather(1, first.clamp(max=z.shape[1] - 1)[:, None])[:, 0]
    return torch.where(some, first, -1).int(), torch.where(some, logp, 0.0)


def _loss(s):
    z, possible, slope = _adjusted(s)
    logp = torch.where(possible, _log_softmax(z, possible), 0.0)
    p = torch.where(possible, torch.exp(logp), 0.0)
    if s.case["target"] == "visits":
        target = s.target
    else:
        target = (torch.arange(z.shape[1], device="cuda") == s.target[:, None]).float()
    target = torch.where(possible, target, 0.0)
    entropy = -(p * logp).sum(1)
    loss = s.weight * -(target * logp).sum(1) - ENTROPY * entropy
    grad = s.weight[:, None] * (target.sum(1, keepdim=True) * p - target) + ENTROPY * p * (logp + entropy[:, None])
    return loss, entropy, (torch.where(possible, grad * slope, 0.0) / z.shape[0]).to(s.logits.dtype)


def _attend(s, layer, q, table, lengths):
    c = s.case
    KV, D, P = c["kv_heads"], c["head_dim"], c["page"]
    n, H, G = q.shape[0], c["heads"], c["heads"] // c["kv_heads"]
    L = table.shape[1] * P
    held = s.kv[:, layer][table.clamp(min=0).long()]                      # [n][width][2][KV][P][D]
    k, v = held.permute(2, 0, 3, 1, 4, 5).reshape(2, n * KV, L, D).float()
    scores = torch.bmm(k, (q.float() * D ** -0.5).reshape(n * KV, G, D).transpose(1, 2).contiguous())   # [n * KV][L][G]
    there = (torch.arange(L, device="cuda") < lengths[:, None]).repeat_interleave(KV, 0)[:, :, None]
    scores = torch.where(there, scores, NEG)
    top = scores.amax(1, keepdim=True)
    top = torch.where(top > NEG, top, 0.0)
    p = torch.exp(scores - top)
    total = p.sum(1, keepdim=True)
    o = torch.bmm((p / total.clamp(min=1e-30)).transpose(1, 2).contiguous(), v)
    return o.reshape(n, H, D).to(q.dtype), (top + torch.log(total)).reshape(n, H)


def _free(s, slots):
    held = s.table[slots]
    s.refs.scatter_add_(0, held.clamp(min=0).long().flatten(), -(held >= 0).int().flatten())
    s.table[slots] = -1
    s.lengths[slots] = 0


def _advance(s, slots, counts):
    """Room for counts more tokens; the lowest free pages go to the slots in their order."""
    P = s.case["page"]
    old = s.lengths[slots]
    new = old + counts
    column = torch.arange(s.table.shape[1], device="cuda")
    wanted = (column >= _pages(old, P)[:, None]) & (column < _pages(new, P)[:, None])
    row, column = wanted.nonzero(as_tuple=True)
    taken = (s.refs == 0).nonzero()[: row.numel(), 0]
    s.table[slots[row], column] = taken.int()
    s.refs[taken] = 1
    s.lengths[slots] = new


def _write(s, k, v, slots, counts):
    """The last counts tokens of the slots, in every layer; k, v: [layers][n][T][KV][D]."""
    P = s.case["page"]
    row, t = (torch.arange(k.shape[2], device="cuda") < counts[:, None]).nonzero(as_tuple=True)
    at = (s.lengths[slots] - counts)[row] + t
    page = s.table[slots[row], at // P].long()
    s.kv[page, :, 0, :, at % P] = k[:, row, t].transpose(0, 1)
    s.kv[page, :, 1, :, at % P] = v[:, row, t].transpose(0, 1)


def _fork(s, src, dst):
    """dst becomes src: full pages are shared, a partly filled last one is copied. What dst held is free for later calls."""
    P = s.case["page"]
    length, table, old = s.lengths[src], s.table[src], s.table[dst]
    part = (length % P).nonzero()[:, 0]
    taken = (s.refs == 0).nonzero()[: part.numel(), 0]
    last = (length // P).long()[part]
    kept = s.kv[taken]
    filled = (torch.arange(P, device="cuda") < (length % P)[part, None])[:, None, None, None, :, None]
    s.kv[taken] = torch.where(filled, s.kv[table[part, last].long()], kept)
    full = torch.arange(table.shape[1], device="cuda") < (length // P)[:, None]
    s.refs.scatter_add_(0, table.clamp(min=0).long().flatten(), full.int().flatten())
    s.refs.scatter_add_(0, old.clamp(min=0).long().flatten(), -(old >= 0).int().flatten())
    s.refs[taken] = 1
    table[part, last] = taken.int()
    s.table[dst] = table
    s.lengths[dst] = length


def _compact(s):
    """The pages in use at and above their number move, in order, into the unused ones below it."""
    used = s.refs > 0
    count = int(used.sum())
    holes, moved = (~used[:count]).nonzero()[:, 0], used[count:].nonzero()[:, 0] + count
    s.kv[holes] = s.kv[moved]
    s.refs[holes] = s.refs[moved]
    s.refs[moved] = 0
    at = torch.arange(used.numel(), device="cuda", dtype=torch.int32)
    at[moved] = holes.int()
    s.table.copy_(torch.where(s.table >= 0, at[s.table.clamp(min=0).long()], s.table))


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if "rows" in case:
        return _exact_policy(s, case)
    if case["kind"] == "attend":
        everything = range(case["slots"])
        out, lse = _exact_attend(s, case, s.q, 0, everything, lambda i: None)
        return out, lse
    if case["kind"] == "expand":   # the cache's own contents are copies
        outs = [_exact_attend(s, case, s.q[i], i, s.src.tolist(), lambda j, i=i: (s.k[i, j], s.v[i, j]))[0] for i in range(case["layers"])]
        return outs, None, None, None, None
    return None   # copies


def _exact_policy(s, case):
    A = case["actions"]
    x = s.logits.double()
    factor = torch.ones_like(x)
    if s.record is not None:
        seen = torch.zeros_like(x)
        for t in range(case["record"]):
            a = s.record[:, t].long()
            live = (s.begin <= t) & (t < s.end) & (a >= 0) & (a < A)
            rows = live.nonzero()[:, 0]
            seen[rows, a[rows]] += 1
        factor[(seen > 0) & (x > 0)] = 1 / REPETITION
        factor[(seen > 0) & (x <= 0)] = REPETITION
        x = x * factor - FREQUENCY * seen - PRESENCE * (seen > 0)
    if s.bias is not None:
        x = x + s.bias.double()
    if s.temperature is not None:
        t = s.temperature.double()
        t[t == 0] = 1
        x, factor = x / t[:, None], factor / t[:, None]
    dead = torch.zeros_like(x, dtype=torch.bool) if s.mask is None else s.mask[:, :A] == 0
    x = x.masked_fill(dead, NEG)
    some = ~dead.all(1)
    logp = x - torch.logsumexp(torch.where(some[:, None], x, 0.0), 1, keepdim=True)
    if case["kind"] == "adjust":
        return logp if case["normalize"] else x
    if case["kind"] == "sample":
        actions, _ = _sample(s)   # which move a draw means is a whole number, fixed in 32 bits; its log-probability is what is computed here
        picked = logp.gather(1, actions.clamp(min=0).long()[:, None])[:, 0]
        return None, torch.where(some, picked, 0.0)
    p, flat = logp.exp(), logp.masked_fill(dead, 0.0)
    entropy = -(p * flat).sum(1)
    if case["target"] == "visits":
        y = s.target.double().masked_fill(dead, 0.0)
    else:
        y = torch.zeros_like(x)
        rows = (s.target >= 0).nonzero()[:, 0]
        y[rows, s.target[rows].long()] = 1
        y = y.masked_fill(dead, 0.0)
    w = s.weight.double()
    loss = -w * (y * flat).sum(1) - ENTROPY * entropy
    grad = (w[:, None] * (y.sum(1, keepdim=True) * p - y) + ENTROPY * p * (flat + entropy[:, None])) * factor / case["rows"]
    return loss, entropy, grad


def _exact_attend(s, case, q, layer, slots, extra):
    KV, D, H = case["kv_heads"], case["head_dim"], case["heads"]
    lengths = s.lengths.tolist()
    outs, lses = [], []
    for i, slot in enumerate(slots):
        n, more = lengths[slot], extra(i)
        pages = s.table[slot, : _pages(n, case["page"])].long()
        kv = s.kv[pages, layer].double().permute(1, 2, 0, 3, 4).reshape(2, KV, -1, D)[:, :, :n]
        if more is not None:
            kv = torch.cat([kv, torch.stack(more).double()[:, :, None]], 2)
        k, v = kv
        scores = (k @ q[i].double().reshape(KV, H // KV, D).transpose(1, 2).contiguous()) / D ** 0.5    # [KV][n][group]
        p = torch.softmax(scores, 1)
        outs.append((p.transpose(1, 2).contiguous() @ v).reshape(H, D))
        lses.append(torch.logsumexp(scores, 1).reshape(H))
    return torch.stack(outs), torch.stack(lses)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    """Bytes: inputs read once and outputs written once; of the cache what is read, copied or written of it, with lengths at their mean."""
    if "rows" in case:
        B, A, kind = case["rows"], case["actions"], case["kind"]
        bytes_ = B * A * (BYTES[case["dtype"]] + (case["mask"] != "none")) + A * 4 * case["bias"] + B * 4 * case["temperature"]
        bytes_ += B * 8 + B * 4 * 0.8 * case["record"] if case["record"] else 0
        if kind == "adjust":
            bytes_ += B * A * 4
        elif kind == "sample":
            bytes_ += B * (A * 4 + 8)
        else:
            bytes_ += B * (A * (4 if case["target"] == "visits" else 0) + 4 * (case["target"] == "moves") + A * BYTES[case["dtype"]] + 12)
        return {"bytes": float(bytes_), "flops": 0.0}
    n, mean, P, layers, kind = case["slots"], (case["lo"] + case["hi"]) / 2, case["page"], case["layers"], case["kind"]
    token, size = _token_bytes(case), BYTES[case["dtype"]]
    heads = 2 * layers * n * case["heads"] * case["head_dim"]
    if kind == "attend":
        return {"bytes": n * (mean * token + mean / P * 4 + 4) + heads * size + n * case["heads"] * 4.0, "flops": 2.0 * heads * mean}
    if kind == "turnover":   # pages of the games that ended are filled from the end of the pool, and the new games' moves are written
        m = n // GROUPS
        return {"bytes": float(m * 4 * mean * token + n * mean / P * 4 * 2), "flops": 0.0}
    tables = n * (3 * mean / P * 4 + 8 * mean / P + 24)   # two rows read, one written; a shared page's and a released page's counter
    if kind == "search":
        return {"bytes": float(n * (P / 2 * token * 2 + 2 * token) + tables), "flops": 0.0}
    return {"bytes": float(n * (P / 2 * token * 2 + (mean + 2) * token) + heads * size + tables), "flops": 2.0 * heads * mean}
