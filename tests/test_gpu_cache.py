"""PagedCache against the plain model of tests/cache_ref.py: pages, tables and counters to the bit, attention against 64 bits.

Tolerance of attention.  u = 2^-24.  A score is a sum of D products of 16-bit numbers, exact by themselves, added in 32 bits: off by at most D u
times the sum of their magnitudes, then scaled: es = (D + 4) u A, A the largest such sum times the scale.  A probability is off relatively by 2 es
(its own score and the others' in the sum), by what the exponential adds (4 u + the argument's rounding, 2 A u) and by the
two-number form, 2^-17 for bfloat16.  The sum over n tokens adds at most (n / 8 + 64) u.  All of it times the largest
|v|, and the rounding to the type on top.  The logarithm's sum: es + 2 A u + (n / 8 + 64) u, and 4 u of its own size."""
import os
import random
import subprocess
import sys

import pytest
import torch

import paper_2303_17503_amd as pg
from cache_ref import RefCache

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUNDING = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype in ROUNDING else torch.int32).cpu()


def same(cache, ref):
    for name in ("table", "lengths", "refs", "kv"):
        assert torch.equal(bits(getattr(cache, name)), bits(getattr(ref, name))), name


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def ref_of(cache):
    return RefCache(cache.kv, cache.table, cache.lengths, cache.refs)


def filled(lengths, layers=1, kv_heads=2, head_dim=64, page_size=16, dtype=torch.bfloat16, seed=0, width=None, spare=3, junk=float("nan"), size=1.0):
    """A cache whose slots hold these lengths in shuffled pages; what no token was written to holds junk."""
    g = torch.Generator("cuda").manual_seed(seed)
    need = [-(-n // page_size) for n in lengths]
    pages, width = sum(need) + spare, width or max(max(need), 1)
    kv = torch.randn(pages, layers, 2, kv_heads, page_size, head_dim, generator=g, device="cuda", dtype=dtype) * size
    order = torch.randperm(pages, generator=g, device="cuda").int().tolist()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    inside = torch.zeros(pages, dtype=torch.int64)
    for s, n in enumerate(lengths):
        for k in range(need[s]):
            p = order.pop()
            table[s, k], refs[p], inside[p] = p, 1, min(page_size, n - k * page_size)
    behind = torch.arange(page_size, device="cuda")[None, :] >= inside.cuda()[:, None]
    kv.masked_fill_(behind[:, None, None, None, :, None], junk)
    return pg.PagedCache(kv, table.cuda(), ints(lengths), refs.cuda())


def check_attend(cache, ref, got, lse, layer, q, slots, scale):
    out, sums, _ = ref.attend(layer, q, slots, scale)
    n = int(cache.lengths.max())
    D = cache.head_dim
    finite = torch.nan_to_num(cache.kv[:, layer].float(), 0.0, 0.0, 0.0)
    big = float(q.float().abs().max()) * float(finite[:, 0].abs().max()) * D * abs(scale)     # A, from above
    vmax = float(finite[:, 1].abs().max())
    # the largest sum of magnitudes that occurs is far below that bound when D is large: by Cauchy and Schwarz
    big = min(big, float(q.float().norm(dim=-1).max()) * float(finite[:, 0].norm(dim=-1).max()) * abs(scale))
    es = (D + 4) * U * big
    rel = 2 * es + 4 * U + 2 * big * U + 2.0 ** -17 + (n / 8 + 64) * U
    err = (got.cpu().double() - out).abs()
    assert not torch.isnan(got.float()).any()
    assert (err <= ROUNDING[cache.dtype] * out.abs() * 1.01 + rel * vmax + 2.0 ** -24).all(), float((err - ROUNDING[cache.dtype] * out.abs()).max())
    if lse is not None:
        lse, live = lse.cpu().double(), torch.isfinite(sums)
        assert torch.equal(torch.isfinite(lse), live) and (lse[~live] == float("-inf")).all()
        assert ((lse - sums)[live].abs() <= es + 2 * big * U + (n / 8 + 64) * U + 4 * U * sums[live].abs()).all()


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 100, 127, 128, 129, 200, 361, 722]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("page_size", [16, 64])
def test_attention_over_lengths_and_head_sizes(head_dim, page_size, dtype):
    kv_heads, heads = 2, 6
    cache = filled(EDGES, 2, kv_heads, head_dim, page_size, dtype, seed=head_dim)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(1)
    q = torch.randn(len(EDGES), heads, head_dim, generator=g, device="cuda", dtype=dtype)
    for layer in (0, 1):
        out, lse = cache.attend(layer, q, lse=True)
        check_attend(cache, ref, out, lse, layer, q, range(len(EDGES)), head_dim ** -0.5)
    assert torch.equal(bits(cache.attend(0, q)), bits(cache.attend(0, q, ints(range(len(EDGES))))))


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (3, 1), (1, 5), (2, 8), (1, 16), (2, 17), (1, 40)])
def test_attention_over_groups(kv_heads, group):
    lengths = [5, 33, 150, 0, 700]
    cache = filled(lengths, 1, kv_heads, 64, 32, torch.bfloat16, seed=group)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(2)
    q = torch.randn(5, kv_heads * group, 64, generator=g, device="cuda", dtype=torch.bfloat16)
    out, lse = cache.attend(0, q, lse=True)
    check_attend(cache, ref, out, lse, 0, q, range(5), 0.125)


@pytest.mark.parametrize("n", [1, 3, 40, 700, 2100, 4100])
def test_attention_is_the_same_however_rows_are_spread(n):
    """few rows are split over blocks and wavefronts, many have a wavefront each: each against 64 bits on the same slots"""
    lengths = [random.Random(7).choice(EDGES + [400, 650]) for _ in range(12)]
    cache = filled(lengths + [0] * max(0, n - 12), 1, 2, 64, 16, torch.float16, seed=3)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(4)
    slots = [i % 12 for i in range(n)]            # (attention only reads: entries may repeat)
    q = torch.randn(12, 4, 64, generator=g, device="cuda", dtype=torch.float16)
    out, lse = cache.attend(0, q[torch.tensor(slots)], ints(slots), lse=True)
    first = min(n, 12)
    check_attend(cache, ref, out[:first], lse[:first], 0, q[:first], slots[:first], 0.125)
    for i in range(12, n, 12):
        k = min(12, n - i)
        assert torch.equal(bits(out[i:i + k]), bits(out[:k])) and torch.equal(bits(lse[i:i + k]), bits(lse[:k]))


@pytest.mark.parametrize("head_dim,kv_heads,group,dtype", [(64, 1, 8, torch.bfloat16), (128, 2, 1, torch.float16), (256, 1, 3, torch.bfloat16)])
def test_long_sequences(head_dim, kv_heads, group, dtype):
    lengths = [20001, 4097, 1, 32768, 0]
    cache = filled(lengths, 1, kv_heads, head_dim, 64, dtype, seed=9)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(5)
    q = torch.randn(5, kv_heads * group, head_dim, generator=g, device="cuda", dtype=dtype)
    for _ in range(2):   # the second call finds its counters as the first did
        out, lse = cache.attend(0, q, lse=True)
        check_attend(cache, ref, out, lse, 0, q, range(5), head_dim ** -0.5)


def test_scores_that_rise_fall_and_saturate():
    n = 300
    for how in ("rising", "falling", "spike", "equal", "large"):
        cache = filled([n, n], 1, 1, 64, 16, torch.float16, seed=6, junk=0.0)
        q = torch.zeros(2, 2, 64, dtype=torch.float16, device="cuda")
        q[:, 0, 0], q[:, 1, 0] = 8.0, -8.0
        line = {"rising": torch.arange(n) * 0.25, "falling": 40 - torch.arange(n) * 0.25, "spike": (torch.arange(n) == 201) * 60.0, "equal": torch.zeros(n),
                "large": (torch.arange(n) % 7 - 3.0) * 8000}[how]
        pages = cache.table[:, : (n + 15) // 16].long()
        for s in range(2):
            for t in range(n):
                cache.kv[pages[s, t // 16], 0, 0, 0, t % 16] = 0
                cache.kv[pages[s, t // 16], 0, 0, 0, t % 16, 0] = float(line[t])
        ref = ref_of(cache)
        out, lse = cache.attend(0, q, lse=True, scale=1.0)
        check_attend(cache, ref, out, lse, 0, q, range(2), 1.0)


def test_entries_that_are_no_slots_and_strides():
    lengths = [50, 0, 7, 300]
    cache = filled(lengths, 1, 2, 64, 16, torch.bfloat16, seed=8)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(6)
    slots = [3, -1, 0, 4]
    fused = torch.randn(4, 4 * 64 + 2 * 2 * 64 + 3, generator=g, device="cuda", dtype=torch.bfloat16)[:, 1:]   # q, k and v of a product in one row
    q = fused[:, :256].view(4, 4, 64) if fused[:, :256].is_contiguous() else fused[:, :256].unflatten(1, (4, 64))
    wide = torch.full((4, 9, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out, lse = cache.attend(0, q, ints(slots), out=wide[:, 1::2], lse=torch.empty(4, 4, device="cuda"))
    check_attend(cache, ref, out, lse, 0, q, slots, 0.125)
    assert (out[1] == 0).all() and (out[3] == 0).all() and (wide[:, ::2] == 7).all()
    assert cache.attend(0, q[:0], ints([])).shape == (0, 4, 64)


@pytest.mark.parametrize("page_size,kv_heads,head_dim,layers,dtype", [(16, 2, 64, 2, torch.bfloat16), (32, 1, 32, 1, torch.float16), (64, 3, 96, 1, torch.float16), (16, 1, 256, 3, torch.bfloat16)])
@pytest.mark.parametrize("seed", range(3))
def test_random_histories(page_size, kv_heads, head_dim, layers, dtype, seed):
    """Every call in random order on a pool that runs out now and then; everything compared after each."""
    r, g = random.Random(seed), torch.Generator().manual_seed(seed)
    slots, width = 23, 5
    cache = pg.PagedCache.empty(slots, 30, width * page_size, layers, kv_heads, head_dim, page_size, dtype)
    cache.kv.fill_(3.0)
    ref = ref_of(cache)
    said = set()
    for step in range(60):
        n = r.randint(0, slots)
        entries = r.sample(range(slots), n)
        entries = [r.choice([-1, -1, -5, slots, 2 ** 30]) if r.random() < 0.1 else s for s in entries]
        what = r.choice(["advance", "advance", "advance", "fork", "fork", "free", "compact"])
        if what == "advance":
            counts = [r.choice([0, 1, 1, 1, 2, page_size - 1, page_size, page_size + 1, 3 * page_size, -2]) for _ in entries]
            one = r.random() < 0.3
            status = torch.full((n,), 99, dtype=torch.uint8, device="cuda")
            cache.advance(ints(entries), 1 if one else ints(counts), status)
            want = ref.advance(entries, [1] * n if one else counts)
            assert status.tolist() == want
            said |= set(want)
            assert cache.lengths.tolist() == ref.lengths.tolist()
            tokens = r.choice([1, 2, 3 * page_size])
            k, v = torch.randn(2, n, tokens, kv_heads, head_dim, generator=g).to(dtype).cuda()
            for layer in range(layers):
                if tokens == 1 and r.random() < 0.5: cache.write(layer, k[:, 0], v[:, 0], ints(entries))
                else: cache.write(layer, k.transpose(1, 2).contiguous().transpose(1, 2), v, ints(entries))
                ref.write(layer, k, v, entries)
        elif what == "fork":
            live = [s for s in entries if 0 <= s < slots]
            half = len(live) // 2
            src = [r.choice(live[:half]) if half else -1 for _ in live[half:]]
            pairs = list(zip(src, live[half:])) + [(s, s) for s in live[:half] if r.random() < 0.2]
            pairs = [r.choice([(-1, d), (slots + 3, d), (s, -1), (s, -7)]) if r.random() < 0.1 else (s, d) for s, d in pairs]
            status = torch.full((len(pairs),), 99, dtype=torch.uint8, device="cuda")
            cache.fork(ints([s for s, _ in pairs]), ints([d for _, d in pairs]), status)
            want = ref.fork([s for s, _ in pairs], [d for _, d in pairs])
            assert status.tolist() == want
            said |= set(want)
        elif what == "free":
            entries = entries[: r.randint(0, 8)]
            cache.free(ints(entries))
            ref.free(entries)
        else:
            used = ints([0])
            cache.compact(used)
            assert int(used) == ref.compact()
        same(cache, ref)
    assert {0, 1, 255} <= said


def test_all_slots_by_default_and_more_entries_than_a_block():
    slots, page_size = 3000, 16
    cache = pg.PagedCache.empty(slots, 9001, 48, 1, 1, 32, page_size, torch.float16)
    cache.kv.zero_()
    ref, g, r = ref_of(cache), torch.Generator().manual_seed(0), random.Random(3)
    for counts in ([r.randint(0, 40) for _ in range(slots)], [1] * slots, [16] * slots):
        status = torch.zeros(slots, dtype=torch.uint8, device="cuda")
        cache.advance(counts=ints(counts), status=status)
        assert status.tolist() == ref.advance(range(slots), counts)
        k, v = torch.randn(2, slots, 16, 1, 32, generator=g).half().cuda()
        cache.write(0, k, v)
        ref.write(0, k, v, range(slots))
    same(cache, ref)
    src, dst = list(range(1500)), list(range(1500, 3000))
    cache.fork(ints(src), ints(dst))
    ref.fork(src, dst)
    same(cache, ref)
    cache.free(ints(dst[::2]))
    ref.free(dst[::2])
    used = ints([0])
    cache.compact(used)
    assert int(used) == ref.compact()
    same(cache, ref)
    cache.compact()
    same(cache, ref)
    cache.free()
    assert int(cache.refs.sum()) == 0 and int(cache.lengths.sum()) == 0 and (cache.table == -1).all()


@pytest.mark.parametrize("n", [1024, 1025, 2900, 4096, 4097])
@pytest.mark.parametrize("pages", [1300, 9000])
def test_one_count_for_many_entries(n, pages):
    """Few and many new pages, up to one per entry and more, in a pool that runs out in the middle of the entries."""
    slots = 4100
    cache = pg.PagedCache.empty(slots, pages, 64, 1, 1, 32, 16, torch.float16)
    cache.kv.zero_()
    ref, r = ref_of(cache), random.Random(n)
    start = [r.choice([0, 1, 8, 14, 15]) for _ in range(slots)]
    cache.advance(counts=ints(start))
    ref.advance(range(slots), start)
    for count in (1, 0, 1, 16, 17, 1):
        entries = r.sample(range(slots), n)
        entries = [r.choice([-1, -4, slots]) if r.random() < 0.02 else s for s in entries]
        status = torch.full((n,), 99, dtype=torch.uint8, device="cuda")
        cache.advance(ints(entries), count, status)
        assert status.tolist() == ref.advance(entries, [count] * n)
        same(cache, ref)


@pytest.mark.parametrize("n", [5, 4200])
@pytest.mark.parametrize("length", [0, 15, 16, 31, 32, 100])
def test_attention_that_writes_the_new_token(length, n):
    kv_heads, heads, D = 2, 40, 64       # three head tiles read what the call writes
    g = torch.Generator("cuda").manual_seed(1)
    a, b = (filled([length] * 5 + [0] * (n - 5), 2, kv_heads, D, 16, torch.bfloat16, seed=2, width=9, spare=3 * n) for _ in range(2))
    q, k, v = (torch.randn(n, h, D, generator=g, device="cuda", dtype=torch.bfloat16) for h in (heads, kv_heads, kv_heads))
    for cache in (a, b):
        cache.advance()
    b.write(1, k, v)
    got = a.attend(1, q, k=k, v=v, lse=True)
    want = b.attend(1, q, lse=True)
    assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
    assert torch.equal(bits(a.kv), bits(b.kv))
    check_attend(b, ref_of(b), got[0][:5], got[1][:5], 1, q[:5], range(5), D ** -0.5)
    before = a.kv.clone()
    a.advance(counts=0)                   # no room was made: nothing is written
    again = a.attend(1, q, k=k + 1, v=v + 1)
    assert torch.equal(bits(again), bits(got[0])) and torch.equal(bits(a.kv), bits(before))


def test_offsets_beyond_32_bits():
    pages = 5 * 2 ** 30 // (2 * 8 * 64 * 128 * 2)           # 5 GB of pages
    kv = torch.zeros(pages, 1, 2, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator("cuda").manual_seed(3)
    last = list(range(pages - 3, pages))
    kv[last] = torch.randn(3, 1, 2, 8, 64, 128, generator=g, device="cuda", dtype=torch.bfloat16)
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[pages - 4] = 0
    cache = pg.PagedCache(kv, ints([last + [-1], [-1] * 4]), ints([130, 0]), refs)
    small = RefCache(kv[last], ints([[0, 1, 2, -1], [-1] * 4]), ints([130, 0]), ints([1, 1, 1]))
    q = torch.randn(2, 8, 128, generator=g, device="cuda", dtype=torch.bfloat16)
    want, lse, _ = small.attend(0, q, [0, 1], 128 ** -0.5)
    out = cache.attend(0, q)
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -12).all() and want[0].abs().max() > 0.1
    cache.fork(ints([0]), ints([1]))
    assert cache.table[1].tolist() == last[:2] + [pages - 4, -1] and torch.equal(kv[pages - 4, ..., :2, :], kv[pages - 1, ..., :2, :])
    assert torch.equal(bits(cache.attend(0, q[:1], ints([1]))), bits(out[:1]))
    cache.refs[5:9] = 0
    cache.rescan()
    cache.compact()
    assert cache.table[0].tolist() == [5 + [pages - 4, pages - 3, pages - 2, pages - 1].index(p) for p in last] + [-1]
    assert torch.equal(bits(cache.attend(0, q[:1], ints([0]))), bits(out[:1]))


def test_a_captured_step_is_replayed():
    """fork, advance and attention in a graph: each replay as the same calls made one by one"""
    lengths = [40, 16, 0, 99, 7, 64]
    a, b = (filled(lengths + [0] * 6, 2, 2, 64, 16, torch.bfloat16, seed=5, width=9, spare=40) for _ in range(2))
    src, dst = ints(range(6)), ints(range(6, 12))
    g = torch.Generator("cuda").manual_seed(3)
    q, k, v = (torch.randn(6, h, 64, generator=g, device="cuda", dtype=torch.bfloat16) for h in (8, 2, 2))
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = pg.PagedCache(a.kv, a.table, a.lengths, a.refs)       # a handle on the stream that is captured

    def step(cache, into):
        cache.fork(src, dst)
        cache.advance(dst)
        for layer in (0, 1):
            cache.attend(layer, q, dst, k=k, v=v, out=into)

    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(c, out)
    eager = torch.empty_like(out)
    for t in range(5):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(b, eager)
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(eager))
        for name in ("kv", "table", "lengths", "refs"):
            assert torch.equal(bits(getattr(a, name)), bits(getattr(b, name))), name
        q.copy_(torch.randn(6, 8, 64, generator=g, device="cuda"))
        k.mul_(-1)


def test_a_saved_cache_goes_on():
    cache = filled([40, 16, 3], 1, 1, 32, 16, torch.float16, seed=5, width=6, spare=9)
    ref = ref_of(cache)
    again = pg.PagedCache(*(t.clone() for t in (cache.kv, cache.table, cache.lengths, cache.refs)))
    for c in (ref,):
        c.advance([2, 0], [14, 9])
    again.advance(ints([2, 0]), ints([14, 9]))
    same(again, ref)


def cache_and_more():
    cache = filled([20, 5], 2, 2, 64, 16, torch.bfloat16)
    return cache, torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")


REFUSED = [
    ("layer beyond the last", lambda c, q, k: c.attend(2, q)),
    ("layer below 0", lambda c, q, k: c.write(-1, k, k)),
    ("q in another type", lambda c, q, k: c.attend(0, q.half())),
    ("q on the host", lambda c, q, k: c.attend(0, q.cpu())),
    ("heads no multiple", lambda c, q, k: c.attend(0, q[:, :3])),
    ("no heads", lambda c, q, k: c.attend(0, q[:, :0])),
    ("head size", lambda c, q, k: c.attend(0, q[:, :, :32])),
    ("q strided inside", lambda c, q, k: c.attend(0, torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda")[:, :, ::2])),
    ("k without v", lambda c, q, k: c.attend(0, q, k=k)),
    ("k of other heads", lambda c, q, k: c.attend(0, q, k=q, v=q)),
    ("scale", lambda c, q, k: c.attend(0, q, scale=float("nan"))),
    ("entries of q", lambda c, q, k: c.attend(0, q, ints([0]))),
    ("lse of other size", lambda c, q, k: c.attend(0, q, lse=torch.zeros(2, 3, device="cuda"))),
    ("slots of long", lambda c, q, k: c.free(torch.zeros(1, dtype=torch.int64, device="cuda"))),
    ("more entries than slots", lambda c, q, k: c.advance(ints([0, 1, -1]))),
    ("negative count", lambda c, q, k: c.advance(counts=-1)),
    ("counts of other size", lambda c, q, k: c.advance(counts=ints([1]))),
    ("status of other type", lambda c, q, k: c.advance(status=ints([0, 0]))),
    ("dst of other size", lambda c, q, k: c.fork(ints([0]), ints([0, 1]))),
    ("used of other size", lambda c, q, k: c.compact(ints([0, 1]))),
    ("v of other tokens", lambda c, q, k: c.write(0, torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device="cuda"), k)),
    ("page size", lambda c, q, k: pg.PagedCache.empty(2, 4, 32, 1, 1, 64, page_size=24)),
    ("head dimension", lambda c, q, k: pg.PagedCache.empty(2, 4, 32, 1, 1, 48)),
    ("kv in float32", lambda c, q, k: pg.PagedCache.empty(2, 4, 32, 1, 1, 64, dtype=torch.float32)),
    ("refs of other size", lambda c, q, k: pg.PagedCache(c.kv, c.table, c.lengths, c.refs[:-1])),
    ("table transposed", lambda c, q, k: pg.PagedCache(c.kv, torch.zeros(3, 2, dtype=torch.int32, device="cuda").t(), c.lengths, c.refs)),
]


@pytest.mark.parametrize("what", [n for n, _ in REFUSED])
def test_refusals(what):
    with pytest.raises(pg.PgxGoError):
        dict(REFUSED)[what](*cache_and_more())


@pytest.mark.parametrize("what", [n for n, _ in REFUSED])
def test_refusals_without_the_native_checks(what, monkeypatch):
    monkeypatch.setattr(pg.cache_binding, "_fast", None)
    test_refusals(what)


def test_native_and_python_checks_make_the_same_calls(monkeypatch):
    def history():
        g = torch.Generator("cuda").manual_seed(1)
        new = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
        cache = filled([20, 5, 0, 33], 2, 2, 64, 16, torch.bfloat16, width=6, spare=20, junk=0.0)
        out, status = [], torch.zeros(3, dtype=torch.uint8, device="cuda")
        cache.advance()
        cache.write(0, new(4, 2, 64), new(4, 2, 64))
        cache.advance(ints([3, -1, 9]), ints([2, 1, 1]), status)
        cache.write(1, new(3, 2, 64), new(3, 2, 64), ints([3, -1, 9]))
        out += [status.clone(), cache.attend(0, new(4, 6, 64)), *cache.attend(1, new(2, 2, 64), ints([3, 0]), k=new(2, 2, 64), v=new(2, 2, 64), scale=1, lse=True)]
        out += [*cache.attend(1, new(4, 2, 64), out=torch.empty(4, 2, 64, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(4, 2, device="cuda"))]
        cache.fork(ints([3, 0, -1]), ints([1, 2, 0]), status)
        cache.free(ints([3, -1]))
        cache.advance(ints([0, 3]), 5)
        many = new(2, 7, 2, 64)
        cache.write(0, many, many.flip(1), ints([0, 3]))
        cache.write(1, new(2, 2, 7, 64).transpose(1, 2), many, ints([0, 3]))
        return out + [status, cache.kv, cache.table, cache.lengths, cache.refs]

    assert pg.cache_binding._fast is not None
    native = history()
    monkeypatch.setattr(pg.cache_binding, "_fast", None)
    for a, b in zip(native, history()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n,head_dim,heads", [(6, 64, 4), (6, 256, 2), (600, 32, 6), (1300, 96, 2), (3, 128, 24)])
def test_a_pool_beyond_every_cache_gives_the_same(n, head_dim, heads):
    """pools of more than 256 MB are read with another hint"""
    r = random.Random(1)
    lengths = [r.choice(EDGES[:14] if n > 100 else [33, 722, 5000]) for _ in range(n)]
    small = filled(lengths, 1, 1, head_dim, 16, torch.bfloat16, seed=4)
    more = (300 << 20) // (2 * 16 * head_dim * 2)
    kv = torch.cat([small.kv, torch.full((more, *small.kv.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")])
    big = pg.PagedCache(kv, small.table, small.lengths, torch.cat([small.refs, torch.zeros(more, dtype=torch.int32, device="cuda")]))
    q = torch.randn(n, heads, head_dim, device="cuda", dtype=torch.bfloat16)
    a, b = small.attend(0, q, lse=True), big.attend(0, q, lse=True)
    assert torch.equal(bits(a[0]), bits(b[0])) and torch.equal(bits(a[1]), bits(b[1])) and torch.isfinite(a[0][torch.tensor(lengths) > 0].float()).all()


def test_a_cache_that_lives_until_the_interpreter_ends():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", "import paper_2303_17503_amd as pg\nclass S: pass\ns = S(); s.cache = pg.PagedCache.empty(2, 4, 32, 1, 1, 64)\nimport sys; sys.kept = s"],
                       cwd=root, capture_output=True, text=True)
    assert r.returncode == 0 and "Traceback" not in r.stderr, r.stderr


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,width,count", [(1, 12, 160), (1030, 12, 160), (1, 50, 721), (3, 2049, 131071)])
def test_many_small_probabilities_beside_a_large_one(rows, width, count, dtype):
    """One token takes nearly all of the weight, and its value is 0: the output is what the tail adds, however small each of its probabilities is.

    Values of one sign in the tail, so each error is relative to the output: the type's rounding; 2^-17 by the two numbers; the
    score's (exact here: one product), its scaling to powers of two and the exponential's argument, (4 + 2 A) u with A = 64 the largest score; the sums'
    (n / 8 + 64) u, of which none add up over more than 64 tiles of 32 in one register here.  And half a step of a subnormal output."""
    page, D = (16, 64) if count < 1000 else (64, 64)
    for at in (0, count // 2, count):                    # where the large one stands
        for below in (2.0, 9.0, 12.0, 15.0, 17.5, 20.0, 30.0):
            pages = -(-(count + 1) // page)
            kv = torch.zeros(pages, 1, 2, 1, page, D, dtype=dtype, device="cuda")
            kv[:, 0, 0, :, :, 0] = -below
            kv[:, 0, 1] = torch.arange(1, D + 1, device="cuda") / 8
            kv[at // page, 0, :, 0, at % page] = 0.0
            kv[at // page, 0, 0, 0, at % page, 0] = 1.0
            table = torch.full((rows, max(width, pages)), -1, dtype=torch.int32, device="cuda")
            table[:, :pages] = torch.arange(pages, device="cuda")        # (attention only reads: rows may share their pages)
            cache = pg.PagedCache(kv, table, torch.full((rows,), count + 1, dtype=torch.int32, device="cuda"), torch.full((pages,), rows, dtype=torch.int32, device="cuda"))
            q = torch.zeros(rows, 2, D, dtype=dtype, device="cuda")
            q[:, 0, 0], q[:, 1, 0] = 1.0, 2.0
            out, lse = cache.attend(0, q, scale=1.0, lse=True)
            for h, times in ((0, 1.0), (1, 2.0)):
                gap = torch.tensor((below + 1.0) * times, dtype=torch.float64)
                tail = count * torch.exp(-gap)
                want = tail / (1 + tail) * torch.arange(1, D + 1, dtype=torch.float64) / 8
                rel = ROUNDING[dtype] * 1.01 + 2.0 ** -17 + (4 + 2 * 64) * U + (64 * 32 / 8 + 64) * U
                got = out[:, h].cpu().double()
                assert ((got - want).abs() <= rel * want + (2.0 ** -25 if dtype is torch.float16 else 0)).all(), (at, below, h, float(((got - want) / want).abs().max()))
                assert ((lse[:, h].cpu().double() - (times + torch.log1p(tail))).abs() <= (64 * 32 / 8 + 64 + 4 + 2 * 64 + 4 * 64) * U).all()


@pytest.mark.parametrize("head_dim,kv_heads,group", [(32, 2, 3), (64, 2, 4), (96, 1, 2), (128, 1, 17), (256, 2, 1)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_scores_of_every_spread_and_order(head_dim, kv_heads, group, dtype):
    """tiles whose largest scores lie far apart, rising, falling and alternating, up to far beyond what counts"""
    lengths = [160, 700, 33, 1]
    g = torch.Generator("cuda").manual_seed(head_dim)
    for spread in (0.5, 4.0, 30.0):
        cache = filled(lengths, 1, kv_heads, head_dim, 16, dtype, seed=11, junk=0.0)
        for s, n in enumerate(lengths):
            for t in range(0, n, 16):
                level = {0: t / 16, 1: -t / 16, 2: (t // 32 % 3 - 1) * 9, 3: 0}[s]
                cache.kv[int(cache.table[s, t // 16]), 0, 0, :, :, 0] += level * spread
        q = torch.randn(4, kv_heads * group, head_dim, generator=g, device="cuda", dtype=dtype) * 0.25
        q[..., 0] = 1.0
        q[..., 0] *= torch.tensor([1.0, -1.0], device="cuda").repeat(kv_heads * group)[: kv_heads * group]
        out, lse = cache.attend(0, q, lse=True, scale=1.0)
        check_attend(cache, ref_of(cache), out, lse, 0, q, range(4), 1.0)


@pytest.mark.parametrize("short", [False, True])
def test_entries_that_need_more_than_a_million_pages_before_others(short):
    """The pages of entry 2048 follow those of entries 0 and 1024, which are added up by one thread; a pool of 2 KB pages beyond what fits LDS."""
    each, last = 524800, 5
    pages = 2 * each + (last - 1 if short else last)
    cache = pg.PagedCache.empty(2049, pages, (each + 1) * 16, 1, 1, 32, 16, torch.float16)
    counts = torch.zeros(2049, dtype=torch.int32, device="cuda")
    counts[0] = counts[1024] = each * 16
    counts[2048] = last * 16
    status = torch.full((2049,), 99, dtype=torch.uint8, device="cuda")
    cache.advance(counts=counts, status=status)
    pages_in_order = torch.arange(pages, dtype=torch.int32, device="cuda")
    assert torch.equal(cache.table[0, :each], pages_in_order[:each]) and torch.equal(cache.table[1024, :each], pages_in_order[each: 2 * each])
    assert status[:2048].max() == 0 and int(status[2048]) == (1 if short else 0)
    assert cache.table[2048, :last].tolist() == ([-1] * last if short else list(range(2 * each, pages))) and int(cache.lengths[2048]) == (0 if short else 16 * last)
    assert int(cache.refs.sum()) == 2 * each + (0 if short else last) and int(cache.refs.max()) == 1 and int((cache.table >= 0).sum()) == int(cache.refs.sum())
    cache.fork(ints([2048, 0]), ints([1, 2]))                          # whole pages only: shared
    cache.free(ints([0]))
    cache.free(ints([2]))
    used = ints([0])
    cache.compact(used)
    assert int(used) == each + (0 if short else last) and torch.equal(cache.refs, (pages_in_order < int(used)).int() + (0 if short else ((cache.table[1, :last, None] == pages_in_order).any(0)).int()))
    moved = cache.table[1024, :each]
    assert int(moved.min()) >= 0 and int(moved.max()) < int(used) and moved.unique().numel() == each
    assert torch.equal(cache.table[1], cache.table[2048])


def test_room_that_was_made_is_still_there_after_a_rescan():
    cache = pg.PagedCache.empty(2, 6, 64, 1, 1, 64)
    cache.kv.zero_()
    ref = ref_of(cache)
    k, v = torch.randn(2, 2, 3, 1, 64, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    cache.advance(counts=3)
    ref.advance(range(2), [3, 3])
    cache.refs[5] = ref.refs[5] = 1                    # a page that the caller keeps for itself
    cache.rescan()
    cache.write(0, k, v)
    ref.write(0, k, v, range(2))
    same(cache, ref)
    status = torch.full((2,), 99, dtype=torch.uint8, device="cuda")
    cache.advance(counts=ints([32, 32]), status=status)
    assert status.tolist() == ref.advance(range(2), [32, 32]) == [0, 1]
    same(cache, ref)


@pytest.mark.parametrize("native", [True, False])
def test_outputs_that_overlap_are_refused(native, monkeypatch):
    cache, q, _ = cache_and_more()
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    new = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for out in (new(1, 4, 64).expand(2, 4, 64), new(2, 1, 64).expand(2, 4, 64), new(4000).as_strided((2, 4, 64), (1000, 32, 1)), new(4000).as_strided((2, 4, 64), (63, 64, 1))):
        with pytest.raises(pg.PgxGoError):
            cache.attend(0, q, out=out)
    want = cache.attend(0, q)
    for out in (new(4, 2, 64).transpose(0, 1), new(2, 9, 64)[:, ::2][:, :4], new(4000).as_strided((2, 4, 64), (300, 64, 1))):    # heads first, every other head, rows apart
        assert torch.equal(cache.attend(0, q, out=out), want)
    one = cache.attend(0, q[:1, :2], ints([0]), out=new(1, 2, 64).as_strided((1, 2, 64), (0, 64, 1)))
    assert torch.equal(one, cache.attend(0, q[:1, :2], ints([0])))


@pytest.mark.parametrize("native", [True, False])
def test_new_outputs_belong_to_the_handles_stream(native, monkeypatch):
    """so that their memory is not at the same time another's on the stream that happens to be current"""
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    here = torch.cuda.current_stream()
    torch.cuda.synchronize()
    for mine, now in ((side, here), (here, side), (side, other)):
        with torch.cuda.stream(mine):
            cache = filled([20, 5], 2, 2, 64, 16, torch.bfloat16)
        torch.cuda.synchronize()
        with torch.cuda.stream(now):
            q = torch.randn(2, 4, 64, device="cuda").bfloat16()
            now.synchronize()
            out, lse = cache.attend(0, q, lse=True)
            assert torch.cuda.current_stream() == now
        for t in (out, lse):
            at = t.data_ptr()
            assert [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]] == [mine.cuda_stream]
        mine.synchronize()
        check_attend(cache, ref_of(cache), out, lse, 0, q, range(2), 0.125)


def test_lists_on_another_device_are_left_alone():
    """A handle that says it is on another device stands for a list on another device: neither the native checks nor Python's pass it on."""
    cache, q, k = cache_and_more()
    before = cache.lengths.clone()
    one, status = ints([0]), torch.zeros(1, dtype=torch.uint8, device="cuda")
    cache._shape = cache._shape[:4] + (1,) + cache._shape[5:]
    cache.device = torch.device("cuda:1")
    for call in (lambda: cache.advance(one), lambda: cache.advance(one, one, status), lambda: cache.free(one), lambda: cache.fork(one, ints([1])), lambda: cache.compact(one),
                 lambda: cache.write(0, k[:1], k[:1], one), lambda: cache.attend(0, q[:1], one), lambda: cache.advance(status=torch.zeros(2, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(pg.PgxGoError):
            call()
    assert torch.equal(cache.lengths, before)


@pytest.mark.parametrize("native", [True, False])
def test_what_is_no_tensor_is_refused(native, monkeypatch):
    cache, q, _ = cache_and_more()
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    for call in (lambda: cache.fork(ints([0]), [1]), lambda: cache.advance(status=[0, 0]), lambda: cache.attend(0, q, lse=1), lambda: cache.compact(3), lambda: cache.free([0])):
        with pytest.raises(pg.PgxGoError):
            call()


def spread_of_lengths(most, count, seed):
    """`count` different lengths up to `most`, the edges of a tile of 32 among them"""
    edges = [0, 1, 31, 32, 33, 64, most - 1, most]
    r = random.Random(seed)
    lengths = edges + r.sample([n for n in range(2, most - 1) if n not in edges], count - len(edges))
    assert len(set(lengths)) == count
    r.shuffle(lengths)
    return lengths


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("tiles,n", [(8, 20), (8, 520), (9, 20), (9, 520), (32, 20), (32, 300), (33, 5), (80, 20), (80, 300), (600, 2)])
def test_attention_in_each_way_that_rows_are_spread(tiles, n, head_dim, dtype):
    """By how long a slot can be and how many rows there are (2 key heads here): one wavefront to a row (8 tiles of 32 tokens, 1024 rows or more), four, or four
    in each of several blocks (more than 32 tiles, 256 rows or fewer).  Different lengths, each row against 64 bits."""
    some = min(n, 16)
    lengths = spread_of_lengths(tiles * 32, max(some, 8), 7)[:some]
    if n <= 5:
        lengths = [tiles * 32, 0, 33, tiles * 32 - 1, 1][:n]
    cache = filled(lengths + [0] * (n - len(lengths)), 1, 2, head_dim, 16, dtype, seed=3, width=tiles * 2)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(4)
    slots = [i % len(lengths) for i in range(n)]
    q = torch.randn(len(lengths), 6, head_dim, generator=g, device="cuda", dtype=dtype)
    out, lse = cache.attend(0, q[torch.tensor(slots)], ints(slots), lse=True)
    check_attend(cache, ref, out[: len(lengths)], lse[: len(lengths)], 0, q, range(len(lengths)), head_dim ** -0.5)
    for i in range(n):
        assert torch.equal(bits(out[i]), bits(out[i % len(lengths)])) and torch.equal(bits(lse[i]), bits(lse[i % len(lengths)]))


@pytest.mark.parametrize("tiles,n", [(8, 600), (8, 7), (20, 40), (60, 6), (60, 300)])
@pytest.mark.parametrize("head_dim,dtype", [(64, torch.bfloat16), (128, torch.float16), (32, torch.float16), (256, torch.bfloat16)])
def test_the_new_token_is_read_in_a_pool_that_is_streamed(head_dim, dtype, tiles, n):
    """what a call writes and reads with the hint of a large pool, in each way that rows are spread; against write and attend one after the other"""
    lengths = [m % (tiles * 32) for m in (0, 15, 16, 31, 32, 33, 200, tiles * 32 - 1)]
    lengths = [lengths[i % 8] for i in range(n)]
    a, b = (filled(lengths, 1, 2, head_dim, 16, dtype, seed=2, width=tiles * 2, spare=n + (270 << 20) // (2 * 2 * 16 * head_dim * 2)) for _ in range(2))
    assert a.kv.numel() * 2 > 256 << 20
    g = torch.Generator("cuda").manual_seed(1)
    q, k, v = (torch.randn(n, h, head_dim, generator=g, device="cuda", dtype=dtype) for h in (40, 2, 2))
    for cache in (a, b):
        cache.advance()
    b.write(0, k, v)
    got, want = a.attend(0, q, k=k, v=v, lse=True), b.attend(0, q, lse=True)
    assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
    assert torch.equal(a.kv.view(torch.int16), b.kv.view(torch.int16))
    some = min(n, 8)
    check_attend(b, ref_of(b), got[0][:some], got[1][:some], 0, q[:some], range(some), head_dim ** -0.5)


@pytest.mark.parametrize("n", [4097, 9000, 20011])
def test_as_many_slots_as_the_largest_batches_have(n):
    """plans of many blocks, in a pool that runs out among the last entries"""
    r = random.Random(n)
    cache = pg.PagedCache.empty(2 * n, 11 * n // 5, 4, 1, 1, 32, 16, torch.float16)
    cache = pg.PagedCache(cache.kv.zero_(), torch.full((2 * n, 4), -1, dtype=torch.int32, device="cuda"), cache.lengths, cache.refs)
    ref = ref_of(cache)
    order = r.sample(range(n), n)
    status = torch.full((n,), 99, dtype=torch.uint8, device="cuda")
    counts = [r.choice([0, 1, 15, 16, 17, 40, 64, 65]) for _ in order]
    cache.advance(ints(order), ints(counts), status)
    assert status.tolist() == ref.advance(order, counts)
    same(cache, ref)
    src, dst = r.sample(range(n), n), r.sample(range(n, 2 * n), n)
    said = []
    for k in range(2):                                       # the second gives up what the first made
        cache.fork(ints(src), ints(dst), status)
        assert status.tolist() == ref.fork(src, dst)
        said += status.tolist()
        same(cache, ref)
        cache.advance(ints(dst), 1, status)
        assert status.tolist() == ref.advance(dst, [1] * n)
        said += status.tolist()
        same(cache, ref)
        src = r.sample(range(n), n)
    assert {0, 1} <= set(said)
    gone = r.sample(range(2 * n), n)
    cache.free(ints(gone))
    ref.free(gone)
    used = ints([0])
    cache.compact(used)
    assert int(used) == ref.compact()
    same(cache, ref)


def test_a_pool_with_more_pages_than_lds_holds_bits_for():
    """270000 pages of 2 KB, some of them the caller's own"""
    pages, slots = 270001, 40
    r, g = random.Random(5), torch.Generator("cuda").manual_seed(2)
    cache = pg.PagedCache.empty(slots, pages, 50 * 16, 1, 1, 32, 16, torch.float16)
    cache.kv.normal_(generator=g)
    kept = torch.randint(0, pages, (9000,), generator=g, device="cuda")
    cache.refs[kept] = 1
    cache.refs[:400] = 1
    cache.rescan()
    ref = ref_of(cache)
    for step in range(6):
        entries = r.sample(range(slots), 20)
        counts = [r.choice([0, 1, 16, 100, 300]) for _ in entries]
        status = torch.full((20,), 99, dtype=torch.uint8, device="cuda")
        cache.advance(ints(entries), ints(counts), status)
        assert status.tolist() == ref.advance(entries, counts)
        src, dst = entries[:10], entries[10:]
        cache.fork(ints(src), ints(dst))
        ref.fork(src, dst)
        same(cache, ref)
        if step % 2:
            cache.free(ints(entries[:3]))
            ref.free(entries[:3])
            used = ints([0])
            cache.compact(used)
            assert int(used) == ref.compact()
            same(cache, ref)


@pytest.mark.parametrize("native", [True, False])
def test_numbers_of_tokens_and_layers_are_whole(native, monkeypatch):
    cache, q, k = cache_and_more()
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    for call in (lambda: cache.advance(counts=1.5), lambda: cache.advance(counts=None), lambda: cache.attend(0.7, q), lambda: cache.write(1.2, k, k), lambda: cache.write("0", k, k), lambda: cache.attend(2 ** 32, q), lambda: cache.write(2 ** 32 + 1, k, k)):
        with pytest.raises(pg.PgxGoError):
            call()
    assert cache.lengths.tolist() == [20, 5]
    cache.advance(counts=torch.ones(1, dtype=torch.int64).numpy()[0])
    assert cache.lengths.tolist() == [21, 6]


def sparse(slots, kv_heads, width, bits_):
    """two pages and no tokens"""
    return pg.PagedCache.empty(slots, 2, width * 16, 1, kv_heads, 32, bits=bits_)


@pytest.mark.parametrize("bits_", [8, 16])
def test_attention_of_more_rows_than_a_launch_takes(bits_):
    n, kv_heads = 4104, 4096
    cache = sparse(n, kv_heads, 65, bits_)                      # four wavefronts to a row: 2^32 threads
    q = torch.zeros(1, kv_heads, 32, dtype=torch.bfloat16, device="cuda").expand(n, kv_heads, 32)
    out = torch.full((n, kv_heads, 32), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pg.PgxGoError):
        cache.attend(0, q, out=out)
    assert (out == 7).all()
    some = torch.arange(n - 16, dtype=torch.int32, device="cuda")
    cache.attend(0, q[:-16], some, out=out[:-16])
    assert (out[:-16] == 0).all() and (out[-16:] == 7).all()


@pytest.mark.parametrize("bits_", [8, 16])
def test_writing_and_reading_more_than_a_launch_takes(bits_):
    n, kv_heads = 2 ** 17 + 8, 4096
    cache = sparse(n, kv_heads, 1, bits_)
    k = torch.zeros(1, 1, 1, 32, dtype=torch.bfloat16, device="cuda")
    for tokens in (1, 2, 80):
        with pytest.raises(pg.PgxGoError):
            cache.write(0, *[k.expand(n, tokens, kv_heads, 32)] * 2)
    some = torch.arange(n - 16, dtype=torch.int32, device="cuda")
    cache.write(0, *[k.expand(n - 16, 1, kv_heads, 32)] * 2, some)
    keys, values = (torch.empty(n, 1, kv_heads, 32, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    keys[-1], values[-1] = 7.0, 7.0
    with pytest.raises(pg.PgxGoError):
        cache.read(0, 1, k=keys, v=values)
    cache.read(0, 1, some, k=keys[:-16], v=values[:-16])
    assert all((part == 0).all() for t in (keys, values) for part in t[:-16].split(2 ** 14)) and (keys[-1] == 7).all() and (values[-1] == 7).all()
    del keys, values
    torch.cuda.empty_cache()


def test_forking_and_freeing_more_than_a_launch_takes():
    n = 2 ** 24
    cache = sparse(n, 64, 1, 16)                                # pages of 131072 bytes: 256 threads to an entry
    none, status = torch.full((n,), -1, dtype=torch.int32, device="cuda"), torch.full((n,), 99, dtype=torch.uint8, device="cuda")
    with pytest.raises(pg.PgxGoError):
        cache.fork(none, none, status)
    assert (status == 99).all()
    cache.fork(none[:-8], none[:-8], status[:-8])
    assert (status[:-8] == 0).all()
    n = 2 ** 26
    cache = sparse(n, 1, 1, 16)
    for refused in (None, torch.arange(n, dtype=torch.int32, device="cuda")):
        cache.lengths.fill_(1)
        with pytest.raises(pg.PgxGoError):
            cache.free(refused)
        assert (cache.lengths == 1).all()
    cache.free(refused[8:])
    assert (cache.lengths[8:] == 0).all() and (cache.lengths[:8] == 1).all()
