"""The operators of a sequence policy whose keys and values are held in 8 bits, as cases that can be timed and compared.

A game's earlier moves take half the memory that 16 bits take: elements are e4m3 numbers times a scale, one for each 16 tokens of a layer, a head
and of keys or values.  A move's place in its game is put into queries and keys by turning them (rotary positions).

  rotate    queries and keys of new tokens, or gradients of them (inverse), turned by their positions
  search    one leaf of each game: a slot becomes a copy of its parent's, grows by a token, whose keys and values are rounded to 8 bits
  expand    the same with turned queries and keys and the layers' attention, which writes the token itself
  turnover  games end, the pages in use move to the front, new games come in with their first moves, which are read back as they are held
  read      keys and values of whole games as they are held
  attend    one new token of each sequence over the keys and values that its pages hold in 8 bits

With `own` false everything is computed in elementary torch operations in 32 bits (positions times frequencies in 64); with `own` true by the
library's calls.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
E4M3 = torch.float8_e4m3fn
BLOCK = 16                      # tokens that share a scale
MOST, LEAST = 448.0, 2.0 ** -100   # the largest e4m3 number; the smallest scale
GROUPS = 8                      # a turnover replaces one game in eight
BASE, FACTOR, ORIGINAL = 10000.0, 16.0, 8192   # of the frequencies; for far positions: stretched by, trained up to
NEG = float("-inf")


def _rotate(name, games, tokens, heads, kv_heads, head_dim, part, dtype, reach, interleaved=False, scaled=False, inverse=False):
    c = {"kind": "rotate", "games": games, "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "part": part, "dtype": dtype,
         "reach": reach, "interleaved": interleaved, "scaled": scaled, "inverse": inverse}
    return {"name": name, **c} if name else c


def _cache(name, kind, slots, lo, hi, dtype, heads, kv_heads, head_dim, page, layers=1):
    c = {"kind": kind, "slots": slots, "lo": lo, "hi": hi, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page,
         "layers": layers}
    return {"name": name, **c} if name else c


def listed():
    return [
        # an actor's ply: the newest token's queries and keys, views into the product that made them; latency
        _rotate("rotate-step-256", 256, 1, 8, 2, 64, 64, "bf16", 722),
        # a learner's pass over the recorded games of a batch
        _rotate("rotate-games-512", 512, 361, 8, 2, 64, 64, "bf16", 361),
        # gradients of one long sequence, neighbouring elements paired, half of the head, frequencies stretched for far positions
        _rotate("rotate-long-back", 1, 40001, 8, 8, 128, 64, "f32", 131072, interleaved=True, scaled=True, inverse=True),
        # one simulation of the search of 4096 full-size games
        _cache("search8-go19-4096", "search", 4096, 60, 500, "bf16", 8, 2, 64, 16, layers=2),
        # a simulation of a handful of games with attention: latency
        _cache("expand8-go19-8", "expand", 8, 1, 722, "bf16", 8, 2, 64, 16, layers=2),
        # one simulation of a 9x9 worker with its attention
        _cache("expand8-go9-1024", "expand", 1024, 1, 160, "f16", 8, 2, 64, 16, layers=2),
        # 256 of 2048 full-size games are replaced by new ones in mid-game
        _cache("turnover8-go19-2048", "turnover", 2048, 60, 500, "bf16", 8, 2, 64, 16, layers=2),
        # a learner or another cache takes the games of a batch as they are held
        _cache("read8-go19-1024", "read", 1024, 1, 722, "bf16", 8, 2, 64, 16),
        # one full-length game of 19x19, alone: latency, and the length split over the machine
        _cache("attend8-one-722", "attend", 1, 722, 722, "bf16", 8, 2, 64, 16),
        # the games of a large self-play worker, of every age
        _cache("attend8-go19-4096", "attend", 4096, 1, 722, "bf16", 8, 2, 64, 16),
        # a batch whose 20 query heads share one wide key head
        _cache("attend8-shared-201", "attend", 201, 1, 4001, "bf16", 20, 1, 256, 64),
        # few long sequences, as many key heads as query heads
        _cache("attend8-long-3", "attend", 3, 90001, 131072, "f16", 8, 8, 128, 64),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm; odd more often than not."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    return min(hi, n | 1) if rng.random() < 0.6 else n


def draw(rng):
    most = {p: max(work(c)["bytes"] for c in listed() if (c["kind"] == "rotate") == p) for p in (True, False)}
    while True:
        kind = rng.choice(["rotate", "rotate", "search", "expand", "turnover", "read", "attend", "attend"])
        if kind == "rotate":
            D = rng.choice([32, 64, 96, 128, 256, 2 * _between(rng, 1, 128)])
            kv_heads = rng.choice([1, 2, 3, 4, 8])
            tokens = rng.choice([1, _between(rng, 1, 40001)])
            c = _rotate(None, _between(rng, 1, 4096), tokens, kv_heads * rng.choice([1, 2, 4, 5, 8]), kv_heads, D,
                        D if rng.random() < 0.6 else 2 * rng.randint(1, D // 2), rng.choice(["f32", "bf16", "f16"]), tokens + _between(rng, 1, 1 << 20),
                        interleaved=rng.random() < 0.5, scaled=rng.random() < 0.5, inverse=rng.random() < 0.3)
            held = 0
        else:
            kv_heads, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 8, 20])
            shape = (rng.choice(["bf16", "f16"]), kv_heads * group, kv_heads, rng.choice([32, 64, 64, 96, 128, 256]), rng.choice([16, 32, 64]))
            if kind in ("attend", "read"):
                hi = _between(rng, 1, 131072)
                c = _cache(None, kind, _between(rng, 1, 4096), rng.randint(0, hi), hi, *shape)
            else:
                hi = _between(rng, 20, 722)
                slots = _between(rng, GROUPS, 4096)
                slots -= slots % GROUPS if kind == "turnover" else 0
                c = _cache(None, kind, slots, rng.randint(0, hi), hi, *shape, layers=rng.randint(1, 2))
            held = c["slots"] * c["hi"] * _token_elements(c)
        if work(c)["bytes"] <= most[kind == "rotate"] and held <= 2e9 and (kind not in ("attend", "read") or held <= 1e9):
            return c


def _token_elements(case):
    return 2 * case["layers"] * case["kv_heads"] * case["head_dim"]


def _pages(tokens, page):
    return (tokens + page - 1) // page


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case = case
    g = torch.Generator("cuda").manual_seed(seed)
    if case["kind"] == "rotate":
        _prepare_rotate(s, case, g)
    else:
        _prepare_cache(s, case, g)
    return s


def _frequencies(part, scaled):
    """Radians per position of each pair of elements.  Stretched for far positions: those that turn often within the original length stay,
    those that hardly turn are divided by the factor, the ones between are mixed."""
    f = BASE ** (-torch.arange(0, part, 2, dtype=torch.float64) / part)
    if scaled:
        keep = ((ORIGINAL * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f * keep + f / FACTOR * (1 - keep)
    return f.cuda()


def _prepare_rotate(s, case, g):
    n, T, H, KV, D = (case[x] for x in ("games", "tokens", "heads", "kv_heads", "head_dim"))
    product = torch.randn(n, T, (H + 2 * KV) * D, generator=g, device="cuda", dtype=DTYPES[case["dtype"]])   # queries, keys and values of one product
    s.q, s.k = product[..., :H * D].unflatten(-1, (H, D)), product[..., H * D:(H + KV) * D].unflatten(-1, (KV, D))
    first = torch.randint(0, max(case["reach"] - T, 0) + 1, (n, 1), generator=g, device="cuda", dtype=torch.int32)
    s.positions = first + torch.arange(T, device="cuda", dtype=torch.int32)
    if T == 1:
        s.q, s.k, s.positions = s.q[:, 0], s.k[:, 0], s.positions[:, 0].contiguous()
    s.frequencies = _frequencies(case["part"], case["scaled"])
    s.magnitude = 0.1 * math.log(FACTOR) + 1 if case["scaled"] else 1.0


def _scale_of(largest):
    """The smallest power of two with which the largest magnitude is at most 448, no smaller than 2^-100."""
    m, e = torch.frexp(largest / MOST)   # (0.5 <= m < 1; the division is exact enough: powers of two times 448 divide exactly)
    return torch.ldexp(torch.ones_like(largest), torch.where(m > 0.5, e, e - 1)).clamp(min=LEAST)


def _prepare_cache(s, case, g):
    n, lo, hi, P, layers = case["slots"], case["lo"], case["hi"], case["page"], case["layers"]
    H, KV, D, dtype = case["heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    kind = case["kind"]
    rand = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    whole = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    children = kind in ("search", "expand")
    slots, width = 2 * n if children else n, _pages(hi + 1, P)
    s.lengths = torch.zeros(slots, dtype=torch.int32, device="cuda")
    s.lengths[:n] = whole(lo, hi + 1, n)
    need = _pages(s.lengths[:n].long(), P)
    used = int(need.sum())
    pages = used + 5 if kind in ("attend", "read") else n * width + 3 * n * children + 5
    # tokens of several sizes, as layers and heads have them, rounded as a write rounds them
    s.kv = torch.empty(pages, layers, 2, KV, P, D, dtype=E4M3, device="cuda")
    s.scales = torch.empty(pages, layers, 2, KV, P // BLOCK, dtype=torch.float32, device="cuda")
    size = torch.exp(rand(layers, 2, KV, 1, 1) * 2 - 1)
    step = max(1, (1 << 28) // (layers * 2 * KV * P * D))
    for i in range(0, pages, step):
        x = torch.randn(min(step, pages - i), layers, 2, KV, P, D, generator=g, device="cuda") * size
        blocks = x.unflatten(4, (P // BLOCK, BLOCK))
        scale = _scale_of(blocks.abs().amax((5, 6)))
        s.scales[i:i + step] = scale
        s.kv[i:i + step] = (blocks / scale[..., None, None]).flatten(4, 5).to(E4M3)
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
        loud = torch.exp2(torch.floor(rand(n, 1, 1) * 4) - 1).to(dtype)   # some tokens are larger than those before them
        s.k, s.v = s.k * loud, s.v * loud
        s.positions = s.lengths[s.src.long()]
        s.frequencies = _frequencies(D, False)
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
    if c["kind"] == "rotate":
        return pg.rotate((s.q, s.k), s.positions, s.frequencies, interleaved=c["interleaved"], magnitude=s.magnitude, inverse=c["inverse"])
    if s.cache is None:   # the handle that a program keeps; the memory is the program's
        s.cache = pg.PagedCache(s.kv, s.table, s.lengths, s.refs, scales=s.scales, dtype=DTYPES[c["dtype"]])
    cache = s.cache
    if c["kind"] == "attend":
        return cache.attend(0, s.q, lse=True)
    if c["kind"] == "read":
        return cache.read(0, c["hi"])
    out = []
    if c["kind"] == "turnover":
        group = s.groups[s.passes % GROUPS]
        s.passes += 1
        cache.free(group)
        cache.compact()
        cache.advance(group, s.counts)
        for i in range(c["layers"]):
            cache.write(i, s.k[i], s.v[i], group)
            out.append(cache.read(i, c["hi"], group))
    else:
        cache.fork(s.src, s.dst)
        cache.advance(s.dst)
        for i in range(c["layers"]):
            if c["kind"] == "search":
                cache.write(i, s.k[i], s.v[i], s.dst)
            else:
                q, k = pg.rotate((s.q[i], s.k[i]), s.positions, s.frequencies)
                out.append(cache.attend(i, q, s.dst, k=k, v=s.v[i]))
    return out, s.kv, s.scales, s.table, s.lengths, s.refs


# ---- the plain forms ------------------------------------------------------------------------------------------------


def _run_plain(s):
    c = s.case
    if c["kind"] == "rotate":
        return tuple(_turned(x, s.positions, s.frequencies, c["interleaved"], s.magnitude, c["inverse"]) for x in (s.q, s.k))
    if c["kind"] == "attend":
        return _attend(s, 0, s.q, s.table, s.lengths)
    if c["kind"] == "read":
        return _read(s, 0, c["hi"], torch.arange(c["slots"], device="cuda"))
    out = []
    if c["kind"] == "turnover":
        group = s.groups[s.passes % GROUPS].long()
        s.passes += 1
        _free(s, group)
        _compact(s)
        _advance(s, group, s.counts)
        for i in range(c["layers"]):
            _write(s, i, s.k[i], s.v[i], group, s.counts)
            out.append(_read(s, i, c["hi"], group))
    else:
        dst, one = s.dst.long(), torch.ones_like(s.dst)
        _fork(s, s.src.long(), dst)
        _advance(s, dst, one)
        for i in range(c["layers"]):
            k = s.k[i]
            if c["kind"] == "expand":
                k = _turned(k, s.positions, s.frequencies, False, 1.0, False)
            _write(s, i, k[:, None], s.v[i][:, None], dst, one)
            if c["kind"] == "expand":
                q = _turned(s.q[i], s.positions, s.frequencies, False, 1.0, False)
                out.append(_attend(s, i, q, s.table[dst], s.lengths[dst])[0])
    return out, s.kv, s.scales, s.table, s.lengths, s.refs


def _turned(x, positions, frequencies, interleaved, magnitude, inverse):
    R = 2 * frequencies.numel()
    angle = positions[..., None, None].double() * frequencies
    cos, sin = (torch.cos(angle) * magnitude).float(), (torch.sin(angle) * magnitude).float()
    if inverse:
        sin = -sin
    part = x[..., :R].float()
    if interleaved:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = part[..., :R // 2], part[..., R // 2:]
        part = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((part.to(x.dtype), x[..., R:]), -1)


def _bits(t):   # (indexing works on bytes)
    return t.view(torch.uint8)


def _held(s, layer, table):
    """[2][n][KV][tokens][D] float32: what the pages of each row hold"""
    c = s.case
    at = table.clamp(min=0).long()
    kv = _bits(s.kv)[:, layer][at].view(E4M3).float()                     # [n][width][2][KV][P][D]
    kv = kv * s.scales[:, layer][at].repeat_interleave(BLOCK, 4)[..., None]
    return kv.permute(2, 0, 3, 1, 4, 5).reshape(2, table.shape[0], c["kv_heads"], table.shape[1] * c["page"], c["head_dim"])


def _attend(s, layer, q, table, lengths):
    c = s.case
    KV, D = c["kv_heads"], c["head_dim"]
    n, H, G = q.shape[0], c["heads"], c["heads"] // c["kv_heads"]
    k, v = _held(s, layer, table).flatten(1, 2)
    L = k.shape[1]
    scores = torch.bmm(k, (q.float() * D ** -0.5).reshape(n * KV, G, D).transpose(1, 2).contiguous())   # [n * KV][L][G]
    there = (torch.arange(L, device="cuda") < lengths[:, None]).repeat_interleave(KV, 0)[:, :, None]
    scores = torch.where(there, scores, NEG)
    top = scores.amax(1, keepdim=True)
    top = torch.where(top > NEG, top, 0.0)
    p = torch.exp(scores - top)
    total = p.sum(1, keepdim=True)
    o = torch.bmm((p / total.clamp(min=1e-30)).transpose(1, 2).contiguous(), v)
    return o.reshape(n, H, D).to(q.dtype), (top + torch.log(total)).reshape(n, H)


def _read(s, layer, tokens, slots):
    """the first tokens of the slots, 0 behind a slot's last; [n][tokens][KV][D] keys and values"""
    there = torch.arange(tokens, device="cuda") < s.lengths[slots][:, None]
    kv = _held(s, layer, s.table[slots])[:, :, :, :tokens].transpose(2, 3)
    k, v = torch.where(there[:, :, None, None], kv, 0.0).to(DTYPES[s.case["dtype"]])
    return k, v


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


def _write(s, layer, k, v, slots, counts):
    """The last counts tokens of the slots; k, v: [n][T][KV][D].  A block's scale is that of its largest new element; a block that had tokens
    before keeps its scale where that is larger, and has them rounded once more where it is smaller."""
    P, D, T = s.case["page"], s.case["head_dim"], k.shape[1]
    first = (s.lengths[slots] - counts).long()
    blocks = (T + BLOCK - 1) // BLOCK + 1
    t = (first // BLOCK * BLOCK)[:, None] + torch.arange(blocks * BLOCK, device="cuda")         # [n][blocks * 16]
    before, new = t < first[:, None], (t >= first[:, None]) & (t < (first + counts)[:, None])
    page = s.table[slots[:, None], (t // P).clamp(max=s.table.shape[1] - 1)].clamp(min=0).long()
    x = torch.stack((k, v)).gather(2, (t - first[:, None]).clamp(0, T - 1)[None, :, :, None, None].expand(2, -1, -1, *k.shape[2:])).float()
    x = torch.where(new[:, :, None, None], x, 0.0).unflatten(2, (blocks, BLOCK))                # [2][n][blocks][16][KV][D]
    scale = _scale_of(x.abs().amax((3, 5)))                                                     # [2][n][blocks][KV]
    at, inside = page[:, ::BLOCK], (t // BLOCK % (P // BLOCK))[:, ::BLOCK]                      # [n][blocks]
    was = s.scales[at, layer, :, :, inside].permute(2, 0, 1, 3)
    had = before[:, ::BLOCK][None, :, :, None]
    scale = torch.where(had, torch.maximum(scale, was), scale)
    kept = _bits(s.kv)[page, layer, :, :, t % P].view(E4M3).float().permute(2, 0, 1, 3, 4).unflatten(2, (blocks, BLOCK))
    kept = kept * torch.where(had, was / scale, 1.0)[:, :, :, None, :, None]
    bytes_ = _bits(torch.where(before.unflatten(1, (blocks, BLOCK))[None, :, :, :, None, None], kept, x / scale[:, :, :, None, :, None]).to(E4M3)).flatten(2, 3)
    some = new.unflatten(1, (blocks, BLOCK)).any(2)                                             # blocks that get tokens
    row, place = ((before | new) & some.repeat_interleave(BLOCK, 1)).nonzero(as_tuple=True)
    _bits(s.kv)[page[row, place], layer, :, :, (t % P)[row, place]] = bytes_[:, row, place].transpose(0, 1)
    row, place = some.nonzero(as_tuple=True)
    s.scales[at[row, place], layer, :, :, inside[row, place]] = scale[:, row, place].transpose(0, 1)


def _fork(s, src, dst):
    """dst becomes src: full pages are shared, a partly filled last one is copied. What dst held is free for later calls."""
    P = s.case["page"]
    length, table, old = s.lengths[src], s.table[src], s.table[dst]
    part = (length % P).nonzero()[:, 0]
    taken = (s.refs == 0).nonzero()[: part.numel(), 0]
    last = table[part, (length // P).long()[part]].long()
    inside = (length % P)[part, None]
    filled = (torch.arange(P, device="cuda") < inside)[:, None, None, None, :, None]
    kv = _bits(s.kv)
    kv[taken] = torch.where(filled, kv[last], kv[taken])
    filled = (torch.arange(0, P, BLOCK, device="cuda") < inside)[:, None, None, None, :]
    s.scales[taken] = torch.where(filled, s.scales[last], s.scales[taken])
    full = torch.arange(table.shape[1], device="cuda") < (length // P)[:, None]
    s.refs.scatter_add_(0, table.clamp(min=0).long().flatten(), full.int().flatten())
    s.refs.scatter_add_(0, old.clamp(min=0).long().flatten(), -(old >= 0).int().flatten())
    s.refs[taken] = 1
    table[part, (length // P).long()[part]] = taken.int()
    s.table[dst] = table
    s.lengths[dst] = length


def _compact(s):
    """The pages in use at and above their number move, in order, into the unused ones below it."""
    used = s.refs > 0
    count = int(used.sum())
    holes, moved = (~used[:count]).nonzero()[:, 0], used[count:].nonzero()[:, 0] + count
    kv = _bits(s.kv)
    kv[holes] = kv[moved]
    s.scales[holes] = s.scales[moved]
    s.refs[holes] = s.refs[moved]
    s.refs[moved] = 0
    at = torch.arange(used.numel(), device="cuda", dtype=torch.int32)
    at[moved] = holes.int()
    s.table.copy_(torch.where(s.table >= 0, at[s.table.clamp(min=0).long()], s.table))


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotate":
        turn = -1.0 if case["inverse"] else 1.0
        return tuple(_exact_turned(x, s.positions, s.frequencies, case["interleaved"], s.magnitude, turn) for x in (s.q, s.k))
    if kind == "attend":
        return _exact_attend(s, case, s.q, lambda i: _exact_sequence(s, case, 0, i))
    if kind == "read":
        return _exact_read(s, case)
    if kind == "turnover":   # the new games begin with a block, so nothing of what was held counts; the rest are copies
        back = []
        there = (torch.arange(case["hi"], device="cuda") < s.counts[:, None])[:, :, None, None]
        for i in range(case["layers"]):
            back.append(tuple(torch.where(there, _exact_rounded(torch.where(there, x[i].double(), 0.0)), 0.0) for x in (s.k, s.v)))
        return back, None, None, None, None, None
    return _exact_children(s, case)


def _exact_turned(x, positions, frequencies, interleaved, magnitude, turn):
    """Pairs as complex numbers, times a power of e."""
    R = 2 * frequencies.numel()
    y = x.double()
    pairs = y[..., :R].unflatten(-1, (R // 2, 2)) if interleaved else y[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
    z = torch.view_as_complex(pairs.contiguous())
    angle = turn * positions.double()[..., None, None] * frequencies
    z = torch.view_as_real(z * torch.polar(torch.full_like(angle, magnitude), angle))
    z = z if interleaved else z.transpose(-1, -2)
    return torch.cat((z.flatten(-2), y[..., R:]), -1)


def _exact_e4m3(x):
    """The nearest number of four binary digits, ties to even, in steps of 2^-9 at least."""
    _, e = torch.frexp(x)
    step = torch.exp2(torch.clamp(e.double() - 1, min=-6) - 3)
    return torch.round(x / step) * step


def _exact_scale(largest):
    return torch.exp2(torch.clamp(torch.ceil(torch.log2(largest) - math.log2(448) - 1e-12), min=-100.0))


def _exact_rounded(x):
    """[n][T][KV][D], the sequences beginning with the first token: the values that are held"""
    n, T, KV, D = x.shape
    y = torch.zeros(n, -(-T // 16) * 16, KV, D, dtype=torch.float64, device="cuda")
    y[:, :T] = x
    y = y.reshape(n, -1, 16, KV, D)
    scale = _exact_scale(y.abs().amax((2, 4), keepdim=True))
    return (_exact_e4m3(y / scale) * scale).reshape(n, -1, KV, D)[:, :T]


def _exact_sequence(s, case, layer, slot):
    """[2][KV][length][D]"""
    n = int(s.lengths[slot])
    pages = s.table[slot, : _pages(n, case["page"])].long()
    kv = _bits(s.kv)[pages, layer].view(E4M3).double()
    scale = s.scales[pages, layer].double().repeat_interleave(16, 3)
    return (kv * scale[..., None]).permute(1, 2, 0, 3, 4).reshape(2, case["kv_heads"], -1, case["head_dim"])[:, :, :n]


def _exact_attend(s, case, q, sequence):
    KV, D, H = case["kv_heads"], case["head_dim"], case["heads"]
    outs, lses = [], []
    for i in range(q.shape[0]):
        k, v = sequence(i)
        scores = (k @ q[i].double().reshape(KV, H // KV, D).transpose(1, 2).contiguous()) / D ** 0.5    # [KV][n][group]
        p = torch.softmax(scores, 1)
        outs.append((p.transpose(1, 2).contiguous() @ v).reshape(H, D))
        lses.append(torch.logsumexp(scores, 1).reshape(H))
    return torch.stack(outs), torch.stack(lses)


def _exact_read(s, case):
    n, T = case["slots"], case["hi"]
    k = torch.zeros(n, T, case["kv_heads"], case["head_dim"], dtype=torch.float64, device="cuda")
    v = torch.zeros_like(k)
    for i in range(n):
        held = _exact_sequence(s, case, 0, i)
        k[i, : held.shape[2]], v[i, : held.shape[2]] = held[0].transpose(0, 1), held[1].transpose(0, 1)
    return k, v


def _exact_children(s, case):
    """A child's last block is its parent's with the new token."""
    P, dtype, layers, n = case["page"], DTYPES[case["dtype"]], case["layers"], case["slots"]
    src, dst = s.src.long(), s.dst.long()
    length = s.lengths[src].long()
    _fork(s, src, dst)                          # which page is whose: whole numbers
    _advance(s, dst, torch.ones_like(s.dst))
    page = s.table[dst, length // P].long()
    kv, scales = s.kv.double(), s.scales.double()
    keys = s.k
    if case["kind"] == "expand":
        keys = _exact_turned(s.k, s.positions, s.frequencies, False, 1.0, 1.0).to(dtype)
    at = length % P // 16                       # the block in its page
    inside = torch.arange(16, device="cuda")
    for i in range(layers):
        for which, new in ((0, keys[i].double()), (1, s.v[i].double())):
            rows = at[:, None] * 16 + inside                                                   # [n][16]
            old = _bits(s.kv)[page[:, None], i, which, :, rows].view(E4M3).double()             # [n][16][KV][D]
            earlier = (inside < (length % 16)[:, None])[:, :, None, None]
            scale, was = _exact_scale(new.abs().amax(-1)), s.scales[page, i, which, :, at].double()
            was = torch.where((length % 16 > 0)[:, None], was, 0.0)
            scale = torch.maximum(scale, was)                                                  # [n][KV]
            old = torch.where(earlier, _exact_e4m3(old * (was / scale)[:, None, :, None]), old)
            old = torch.where((inside == (length % 16)[:, None])[:, :, None, None], _exact_e4m3(new / scale[:, :, None])[:, None], old)
            kv[page[:, None], i, which, :, rows] = old
            scales[page, i, which, :, at] = scale
    outs = []
    if case["kind"] == "expand":
        lengths, tables = (length + 1).tolist(), s.table[dst].long()
        for i in range(layers):
            def sequence(j, i=i):
                pages = tables[j, : _pages(lengths[j], P)]
                held = kv[pages, i] * scales[pages, i].repeat_interleave(16, 3)[..., None]
                return held.permute(1, 2, 0, 3, 4).reshape(2, case["kv_heads"], -1, case["head_dim"])[:, :, : lengths[j]]
            q = _exact_turned(s.q[i], s.positions, s.frequencies, False, 1.0, 1.0).to(dtype)
            outs.append(_exact_attend(s, case, q, sequence)[0])
    return outs, kv, scales, None, None, None


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    """Bytes: inputs read once and outputs written once; of the cache what is read, copied or written of it, with lengths at their mean."""
    size = BYTES[case["dtype"]]
    if case["kind"] == "rotate":
        tokens = case["games"] * case["tokens"]
        return {"bytes": float(tokens * ((case["heads"] + case["kv_heads"]) * case["head_dim"] * 2 * size + 4)), "flops": 0.0}
    n, mean, P, layers, kind = case["slots"], (case["lo"] + case["hi"]) / 2, case["page"], case["layers"], case["kind"]
    new = _token_elements(case) * size                                                  # a token as it comes
    token = _token_elements(case) + 2 * layers * case["kv_heads"] * 4 / BLOCK           # a token as it is held, with its share of the scales
    heads = 2 * layers * n * case["heads"] * case["head_dim"]
    if kind == "attend":
        return {"bytes": n * (mean * token + mean / P * 4 + 4) + heads * size + n * case["heads"] * 4.0, "flops": 2.0 * heads * mean}
    if kind == "read":
        return {"bytes": float(n * (mean * token + mean / P * 4 + 4 + case["hi"] * new)), "flops": 0.0}
    if kind == "turnover":   # pages of the games that ended are filled from the end of the pool; the new games' moves are written and read back
        m = n // GROUPS
        return {"bytes": float(m * mean * (2 * token + new + token + token) + m * case["hi"] * new + n * mean / P * 4 * 2), "flops": 0.0}
    tables = n * (3 * mean / P * 4 + 8 * mean / P + 24)   # two rows read, one written; a shared page's and a released page's counter
    if kind == "search":
        return {"bytes": float(n * (P / 2 * token * 2 + new + token) + tables), "flops": 0.0}
    return {"bytes": float(n * (P / 2 * token * 2 + new + (mean + 1) * token) + heads * size + tables), "flops": 2.0 * heads * mean}
