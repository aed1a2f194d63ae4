"""PagedCache held in 8 bits against the plain model of tests/cache8_ref.py: codes, scales, tables and counters to the bit, attention against 64 bits.

Tolerance of attention: that of tests/test_gpu_cache.py, over the values that the codes stand for.  u = 2^-24.  A score is a sum of D products of a 16-bit
number with a code of 4 binary digits, exact by themselves, added in 32 bits, then multiplied by scale and block's scale, themselves one rounded product:
es = (D + 6) u A, A the largest sum of magnitudes times both.  A probability is off relatively by 2 es, by what the exponential adds (4 u + 2 A u) and by the two
numbers that stand for it, 2^-17; times the values' scale, a power of two, exactly.  The sum over n tokens adds (n / 8 + 64) u.  All of it times the largest |v|, and the
rounding to the type on top.  The logarithm's sum: es + 2 A u + (n / 8 + 64) u, and 4 u of its own size."""
import random

import pytest
import torch

import paper_2303_17503_amd as pg
from cache8_ref import RefCache8, scale_for
from test_gpu_cache import EDGES, ROUNDING, U, bits, ints, spread_of_lengths

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def same(cache, ref):
    for name in ("table", "lengths", "refs"):
        assert torch.equal(getattr(cache, name).cpu(), getattr(ref, name)), name
    assert ((cache.scales.cpu().double() == ref.scales) | torch.isnan(ref.scales)).all()
    assert torch.equal(codes_of(cache), bytes_of(ref.kv))


def codes_of(cache):
    """bytes, the two codes of NaN as one"""
    b = cache.kv.view(torch.uint8).cpu()
    return b.masked_fill(b == 0xFF, 0x7F)


def bytes_of(codes):
    return codes.float().nan_to_num(nan=0.0).to(E4M3).view(torch.uint8).masked_fill(torch.isnan(codes), 0x7F)


def ref_of(cache):
    return RefCache8(cache.kv, cache.scales, cache.table, cache.lengths, cache.refs)


def filled(lengths, layers=1, kv_heads=2, head_dim=64, page_size=16, dtype=torch.bfloat16, seed=0, width=None, spare=3, junk=True, loud=2):
    """A cache whose slots hold these lengths in shuffled pages, codes of every size, scales of 2^-loud to 2^loud; what no token was written to holds NaN, and
    blocks without tokens have scales that are NaN, infinite and 0."""
    g = torch.Generator("cuda").manual_seed(seed)
    need = [-(-n // page_size) for n in lengths]
    pages, width = sum(need) + spare, width or max(max(need), 1)
    kv = (torch.randn(pages, layers, 2, kv_heads, page_size, head_dim, generator=g, device="cuda") * 64).clamp(-448, 448).to(E4M3)
    scales = torch.exp2(torch.randint(-loud - 6, loud - 5, (pages, layers, 2, kv_heads, page_size // 16), generator=g, device="cuda").float())
    order = torch.randperm(pages, generator=g, device="cuda").int().tolist()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    inside = torch.zeros(pages, dtype=torch.int64)
    for s, n in enumerate(lengths):
        for k in range(need[s]):
            p = order.pop()
            table[s, k], refs[p], inside[p] = p, 1, min(page_size, n - k * page_size)
    if junk:
        behind = torch.arange(page_size, device="cuda")[None, :] >= inside.cuda()[:, None]
        kv.view(torch.uint8).masked_fill_(behind[:, None, None, None, :, None], 0x7F)
        odd = torch.tensor([float("nan"), float("inf"), 0.0, -1.0], device="cuda")[torch.arange(scales.numel(), device="cuda").reshape(scales.shape) % 4]
        scales = torch.where(behind[:, ::16][:, None, None, None], odd, scales)
    return pg.PagedCache(kv, table.cuda(), ints(lengths), refs.cuda(), scales=scales, dtype=dtype)


def check_attend(cache, ref, got, lse, layer, q, slots, scale):
    out, sums, _ = ref.attend(layer, q, slots, scale)
    n, D = int(cache.lengths.max()), cache.head_dim
    held = [ref.sequence(s, layer) for s in slots if 0 <= s < cache.slots and int(cache.lengths[s])]
    big = float(q.float().norm(dim=-1).max()) * max(float(h[0].norm(dim=-1).max()) for h in held) * abs(scale) if held else 0.0   # by Cauchy and Schwarz
    vmax = max(float(h[1].abs().max()) for h in held) if held else 0.0
    es = (D + 6) * U * big
    rel = 2 * es + 4 * U + 2 * big * U + 2.0 ** -17 + (n / 8 + 64) * U
    err = (got.cpu().double() - out).abs()
    # an output beyond the type's largest number (float16: 65504, and half a step of 32) is rounded to infinity
    far = torch.isinf(got).cpu() & ((got.cpu() > 0) == (out > 0)) & (out.abs() + rel * vmax >= torch.finfo(cache.dtype).max * (1 + torch.finfo(cache.dtype).eps / 4))
    err = torch.where(far, 0.0, err)
    assert not torch.isnan(got.float()).any()
    assert (err <= ROUNDING[cache.dtype] * out.abs() * 1.01 + rel * vmax + 2.0 ** -24).all(), float((err - ROUNDING[cache.dtype] * out.abs()).max())
    if lse is not None:
        lse, live = lse.cpu().double(), torch.isfinite(sums)
        assert torch.equal(torch.isfinite(lse), live) and (lse[~live] == float("-inf")).all()
        assert ((lse - sums)[live].abs() <= es + 2 * big * U + (n / 8 + 64) * U + 4 * U * sums[live].abs()).all()


def new(g, dtype, *shape, size=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


# ---- writing and reading back ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("page_size", [16, 32, 64, 256])
def test_tokens_as_they_come(page_size, head_dim, dtype):
    """rooms of many sizes, one after the other, louder and quieter, so that blocks begin inside a call, end inside one and are raised by one; all codes and scales"""
    r, g = random.Random(head_dim + page_size), torch.Generator("cuda").manual_seed(head_dim)
    slots, kv_heads, layers = 7, 2, 2
    cache = filled([0] * slots, layers, kv_heads, head_dim, page_size, dtype, width=6, spare=6 * slots)
    ref = ref_of(cache)
    for step in range(9):
        counts = [r.choice([0, 1, 1, 2, 5, 15, 16, 17, 33]) for _ in range(slots)]
        cache.advance(counts=ints(counts))
        ref.advance(range(slots), counts)
        T = max(max(ref.grown), 1)
        size = torch.exp2(torch.randint(-4, 5, (slots, T, 1, 1), generator=g, device="cuda").float())
        product = (torch.randn(slots, T, 3 * kv_heads * head_dim, generator=g, device="cuda")).to(dtype)     # q, k and v of one product
        for layer in range(layers):
            k, v = (product[..., i * kv_heads * head_dim:][..., : kv_heads * head_dim].unflatten(-1, (kv_heads, head_dim)) for i in (1, 2))
            k = (k * size).to(dtype)
            if T == 1: cache.write(layer, k[:, 0], v[:, 0])
            else: cache.write(layer, k, v)
            ref.write(layer, k, v, range(slots))
        same(cache, ref)
        for layer in range(layers):
            k, v = cache.read(layer, 6 * page_size)
            want = ref.read(layer, 6 * page_size, range(slots), [0] * slots, dtype)
            assert torch.equal(bits(k), bits(want[0])) and torch.equal(bits(v), bits(want[1]))
    assert int(cache.lengths.max()) > min(page_size, 64) + 16


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_values_of_every_size(dtype):
    """zeros of both signs, subnormal and largest numbers, infinities and NaN, blocks of nothing else, ties of the rounding"""
    D, slots = 64, 12
    cache = filled([0] * slots, 1, 1, D, 16, dtype, width=4, spare=60)
    ref = ref_of(cache)
    tiny, most = torch.finfo(dtype).smallest_normal, torch.finfo(dtype).max
    lines = [torch.zeros(D), -torch.zeros(D), torch.full((D,), tiny / 4), torch.full((D,), most), torch.full((D,), float("inf")), torch.full((D,), float("nan")),
             torch.arange(D) - 32.0, torch.exp2(torch.arange(D) - 40.0) if dtype is torch.bfloat16 else torch.exp2(torch.arange(D) / 2 - 20.0), torch.cat([torch.tensor([float("inf"), -3.0]), torch.arange(D - 2) * 0.0625]),
             torch.arange(D) * 0.5 + 0.25, torch.full((D,), 448.0), torch.full((D,), -450.0)]
    order = random.Random(1)
    for step in range(40):
        k = torch.stack([lines[order.randrange(len(lines))] if step else lines[i] for i in range(slots)])[:, None].to(dtype).cuda()
        v = k.flip(0).contiguous()
        cache.advance()
        ref.advance(range(slots), [1] * slots)
        cache.write(0, k, v)
        ref.write(0, k[:, None], v[:, None], range(slots))
        same(cache, ref)
    k, v = cache.read(0, 40)
    want = ref.read(0, 40, range(slots), [0] * slots, dtype)
    assert torch.equal(torch.isnan(k).cpu(), torch.isnan(want[0])) and torch.isnan(k).any()
    assert torch.equal(k.cpu().nan_to_num(nan=0.0), want[0].nan_to_num(nan=0.0)) and torch.equal(v.cpu().nan_to_num(nan=0.0), want[1].nan_to_num(nan=0.0))


def test_fewer_tokens_than_there_is_room_for_and_entries_that_are_no_slots():
    cache = filled([10, 3, 16, 0], 1, 2, 64, 16, torch.bfloat16, width=6, spare=20)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(1)
    entries = [2, -1, 0, 9, 3]
    cache.advance(ints(entries[:4]), 20)
    ref.advance(entries[:4], [20] * 4)
    k, v = new(g, torch.bfloat16, 4, 7, 2, 64), new(g, torch.bfloat16, 4, 7, 2, 64)
    cache.write(0, k, v, ints(entries[:4]))
    ref.write(0, k, v, entries[:4])
    same(cache, ref)
    cache.write(0, k[:, :0], v[:, :0], ints(entries[:4]))
    again = k.flip(1).contiguous() * 4
    cache.write(0, again, v, ints(entries[:4]))            # the same tokens once more
    ref.write(0, again, v, entries[:4])
    same(cache, ref)


@pytest.mark.parametrize("bits_", [8, 16])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim,page_size", [(32, 16), (96, 32), (256, 64)])
def test_reading_back(head_dim, page_size, dtype, bits_):
    from test_gpu_cache import filled as filled16, ref_of as ref16

    lengths = [0, 1, 17, 64, 100, 33]
    if bits_ == 8:
        cache = filled(lengths, 2, 3, head_dim, page_size, dtype, seed=2)
        ref = ref_of(cache)
    else:
        cache = filled16(lengths, 2, 3, head_dim, page_size, dtype, seed=2)
        ref = ref16(cache)
        ref.read = lambda layer, tokens, slots, first, dtype: RefCache8.read(ref, layer, tokens, slots, first, dtype)
    slots, first = [4, 0, 4, -1, 2, 77], [96, 0, 3, 5, -2, 0]
    for layer, tokens in ((0, 1), (1, 3), (0, 4), (1, 9), (0, 130)):
        got = cache.read(layer, tokens, ints(slots), ints(first))
        want = ref.read(layer, tokens, slots, first, dtype)
        assert got[0].shape == (6, tokens, 3, head_dim) and torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
    wide = torch.full((2, 6, 3, 5, head_dim + 2), 7.0, dtype=dtype, device="cuda")     # heads first, rows apart
    views = [wide[i, :, :, :, 1:-1].transpose(1, 2) for i in range(2)]
    cache.read(1, 5, first=2, k=views[0], v=views[1])
    want = ref.read(1, 5, range(6), [2] * 6, dtype)
    assert torch.equal(bits(views[0]), bits(want[0])) and torch.equal(bits(views[1]), bits(want[1])) and (wide[..., 0] == 7).all() and (wide[..., -1] == 7).all()
    assert cache.read(0, 0)[0].shape == (6, 0, 3, head_dim) and cache.read(0, 2, ints([]))[1].shape == (0, 2, 3, head_dim)
    late = cache.read(0, 2, first=2 ** 31 - 1)
    assert (late[0] == 0).all() and (late[1] == 0).all()


# ---- attention -------------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("page_size", [16, 32, 64, 1024])
def test_attention_over_lengths_and_head_sizes(head_dim, page_size, dtype):
    kv_heads, heads = 2, 6
    cache = filled(EDGES, 2, kv_heads, head_dim, page_size, dtype, seed=head_dim)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(1)
    q = new(g, dtype, len(EDGES), heads, head_dim)
    for layer in (0, 1):
        out, lse = cache.attend(layer, q, lse=True)
        check_attend(cache, ref, out, lse, layer, q, range(len(EDGES)), head_dim ** -0.5)
    assert torch.equal(bits(cache.attend(0, q)), bits(cache.attend(0, q, ints(range(len(EDGES))))))


@pytest.mark.parametrize("kv_heads,group", [(1, 1), (3, 1), (1, 5), (2, 8), (1, 16), (2, 17), (1, 40)])
def test_attention_over_groups_and_strides(kv_heads, group):
    lengths = [5, 33, 150, 0, 700]
    cache = filled(lengths, 1, kv_heads, 64, 32, torch.bfloat16, seed=group)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(2)
    heads = kv_heads * group
    q = new(g, torch.bfloat16, 5, heads * 64 + 3)[:, 1:-2].unflatten(1, (heads, 64))
    wide = torch.full((5, 2 * heads + 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    slots = [4, -1, 1, 5, 2]
    out, lse = cache.attend(0, q, ints(slots), out=wide[:, 1::2], lse=True)
    check_attend(cache, ref, out, lse, 0, q, slots, 0.125)
    assert (out[1] == 0).all() and (out[3] == 0).all() and (wide[:, ::2] == 7).all()


@pytest.mark.parametrize("head_dim,kv_heads,group,dtype", [(64, 1, 8, torch.bfloat16), (128, 2, 1, torch.float16), (256, 1, 3, torch.bfloat16), (32, 1, 17, torch.float16)])
def test_long_sequences(head_dim, kv_heads, group, dtype):
    lengths = [20001, 4097, 1, 32768, 0]
    cache = filled(lengths, 1, kv_heads, head_dim, 64, dtype, seed=9)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(5)
    q = new(g, dtype, 5, kv_heads * group, head_dim)
    for _ in range(2):   # the second call finds its counters as the first did
        out, lse = cache.attend(0, q, lse=True)
        check_attend(cache, ref, out, lse, 0, q, range(5), head_dim ** -0.5)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("tiles,n", [(8, 20), (10, 520), (11, 520), (32, 512), (12, 2050), (9, 20), (32, 300), (33, 5), (40, 512), (80, 20), (80, 300), (600, 2), (200, 300), (1200, 12)])
def test_attention_in_each_way_that_rows_are_spread(tiles, n, head_dim, dtype):
    """one wavefront to a row, four, four in each of several blocks; and more than 32 tiles for a wavefront, which looks its pages up 32 tiles at a time"""
    some = min(n, 12 if tiles > 100 else 16)
    lengths = spread_of_lengths(tiles * 32, max(some, 8), 7)[:some]
    if n <= 5:
        lengths = [tiles * 32, 0, 33, tiles * 32 - 1, 1][:n]
    cache = filled(lengths + [0] * (n - len(lengths)), 1, 2, head_dim, 16, dtype, seed=3, width=tiles * 2)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(4)
    slots = [i % len(lengths) for i in range(n)]
    q = new(g, dtype, len(lengths), 6, head_dim)
    out, lse = cache.attend(0, q[torch.tensor(slots)], ints(slots), lse=True)
    check_attend(cache, ref, out[: len(lengths)], lse[: len(lengths)], 0, q, range(len(lengths)), head_dim ** -0.5)
    for i in range(n):
        assert torch.equal(bits(out[i]), bits(out[i % len(lengths)])) and torch.equal(bits(lse[i]), bits(lse[i % len(lengths)]))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim,heads", [(32, 2), (64, 4), (64, 40), (96, 2), (128, 6), (256, 2), (256, 40)])
@pytest.mark.parametrize("n,width", [(5, 9), (5, 80), (600, 9), (600, 14)])
def test_attention_that_writes_the_new_token(n, width, head_dim, heads, dtype):
    """step by step, louder and quieter tokens: codes, scales and results as those of write and attend one after the other, and of the plain model"""
    kv_heads = 2
    lengths = [0, 14, 15, 31, 100]
    lengths += [lengths[i % 5] for i in range(n - 5)]
    g = torch.Generator("cuda").manual_seed(1)
    a, b = (filled(lengths, 2, kv_heads, head_dim, 16, dtype, seed=2, width=width, spare=2 * n) for _ in range(2))
    ref = ref_of(a) if n == 5 else None
    for step in range(5):
        q = new(g, dtype, n, heads, head_dim)
        size = torch.exp2(torch.randint(-3, 4, (n, 1, 1), generator=g, device="cuda").float())
        k, v = ((torch.randn(n, kv_heads, head_dim, generator=g, device="cuda") * size).to(dtype) for _ in range(2))
        for cache in (a, b):
            cache.advance()
        b.write(1, k, v)
        got = a.attend(1, q, k=k, v=v, lse=True)
        want = b.attend(1, q, lse=True)
        assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
        assert torch.equal(a.kv.view(torch.uint8), b.kv.view(torch.uint8))
        assert torch.equal(a.scales.view(torch.int32), b.scales.view(torch.int32))
        if ref:
            ref.advance(range(n), [1] * n)
            ref.write_last(1, k, v, range(n))
            live = ~torch.isnan(ref.scales)
            assert torch.equal(a.scales.cpu().double()[live], ref.scales[live]) and torch.equal(codes_of(a), bytes_of(ref.kv))
            check_attend(a, ref, got[0], got[1], 1, q, range(n), head_dim ** -0.5)
    before = a.kv.clone(), a.scales.clone()
    a.advance(counts=0)                   # no room was made: nothing is written
    again = a.attend(1, q, k=k * 8, v=v * 8)
    assert torch.equal(bits(again), bits(got[0])) and torch.equal(a.kv.view(torch.uint8), before[0].view(torch.uint8)) and torch.equal(a.scales.view(torch.int32), before[1].view(torch.int32))


def test_the_last_of_several_new_tokens_comes_with_the_attention():
    for heads in (2, 40):
        cache = filled([13, 0, 31], 1, 2, 64, 16, torch.bfloat16, width=6, spare=9)
        ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(heads)
        cache.advance(counts=4)
        ref.advance(range(3), [4] * 3)
        k, v = (new(g, torch.bfloat16, 3, 4, 2, 64) * torch.tensor([1, 1, 1, 9.0], device="cuda")[:, None, None] for _ in range(2))
        k, v = k.bfloat16(), v.bfloat16()
        cache.write(0, k[:, :3], v[:, :3])
        ref.write(0, k[:, :3], v[:, :3], range(3))
        q = new(g, torch.bfloat16, 3, heads, 64)
        out, lse = cache.attend(0, q, k=k[:, 3], v=v[:, 3], lse=True)
        ref.write_last(0, k[:, 3], v[:, 3], range(3))
        assert torch.equal(codes_of(cache), bytes_of(ref.kv))
        check_attend(cache, ref, out, lse, 0, q, range(3), 0.125)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_scales_that_lie_far_apart(dtype):
    """blocks of values 2^40 apart, scales that are no powers of two, and scores that rise, fall and alternate from tile to tile"""
    lengths, D = [160, 700, 33, 1], 64
    g = torch.Generator("cuda").manual_seed(3)
    for loud in (1, 12, 20):
        cache = filled(lengths, 1, 2, D, 16, dtype, seed=11, loud=loud, junk=False)
        cache.scales[:, :, 0] = torch.exp2(torch.randint(-9, -3, cache.scales[:, :, 0].shape, generator=g, device="cuda").float()) * 1.25
        cache.scales[:, :, 1] *= 1.5
        q = new(g, dtype, 4, 6, D, size=0.5)
        out, lse = cache.attend(0, q, lse=True)
        check_attend(cache, ref_of(cache), out, lse, 0, q, range(4), D ** -0.5)


def test_a_value_that_is_not_finite_counts_where_it_is():
    cache = filled([40, 40, 40], 1, 2, 64, 16, torch.bfloat16, seed=3, width=4, spare=9)
    g = torch.Generator("cuda").manual_seed(1)
    q, k, v = new(g, torch.bfloat16, 3, 4, 64), new(g, torch.bfloat16, 3, 2, 64), new(g, torch.bfloat16, 3, 2, 64)
    k[0, 0, 5], v[1, 1, 7] = float("nan"), float("inf")
    cache.advance()
    out = cache.attend(0, q, k=k, v=v)
    bad = torch.isnan(out.float())
    assert bad[0, :2].all() and not bad[0, 2:].any() and not bad[2].any()          # a key: its head's queries
    assert bad[1, 2:, 7].all() and int(bad[1].sum()) == 2                            # a value: its element


@pytest.mark.parametrize("n,head_dim,heads", [(6, 64, 4), (6, 256, 2), (600, 32, 6), (1300, 96, 2), (3, 128, 24)])
def test_a_pool_beyond_every_cache_gives_the_same(n, head_dim, heads):
    """pools of more than 256 MB are read with another hint"""
    r = random.Random(1)
    lengths = [r.choice(EDGES[:14] if n > 100 else [33, 722, 5000]) for _ in range(n)]
    small = filled(lengths, 1, 1, head_dim, 16, torch.bfloat16, seed=4)
    more = (300 << 20) // (2 * 16 * head_dim)
    kv = torch.cat([small.kv.view(torch.uint8), torch.full((more, *small.kv.shape[1:]), 0x7F, dtype=torch.uint8, device="cuda")]).view(E4M3)
    scales = torch.cat([small.scales, torch.zeros(more, *small.scales.shape[1:], device="cuda")])
    big = pg.PagedCache(kv, small.table, small.lengths, torch.cat([small.refs, torch.zeros(more, dtype=torch.int32, device="cuda")]), scales=scales, dtype=torch.bfloat16)
    g = torch.Generator("cuda").manual_seed(1)
    q, k, v = new(g, torch.bfloat16, n, heads, head_dim), new(g, torch.bfloat16, n, 1, head_dim, size=4.0), new(g, torch.bfloat16, n, 1, head_dim, size=4.0)
    a, b = small.attend(0, q, lse=True), big.attend(0, q, lse=True)
    assert torch.equal(bits(a[0]), bits(b[0])) and torch.equal(bits(a[1]), bits(b[1])) and torch.isfinite(a[0][torch.tensor(lengths) > 0].float()).all()
    room = ints([1 if 0 < m % 16 else 0 for m in lengths])        # (inside their last pages)
    small.lengths.copy_(ints(lengths)); big.lengths = small.lengths.clone()
    small = pg.PagedCache(small.kv, small.table, small.lengths, small.refs, scales=small.scales, dtype=torch.bfloat16)
    big = pg.PagedCache(big.kv, big.table.clone(), big.lengths, big.refs, scales=big.scales, dtype=torch.bfloat16)
    for cache in (small, big):
        cache.advance(counts=room)
    a, b = small.attend(0, q, k=k, v=v, lse=True), big.attend(0, q, k=k, v=v, lse=True)
    assert torch.equal(bits(a[0]), bits(b[0])) and torch.equal(bits(a[1]), bits(b[1]))
    used = small.kv.shape[0]
    assert torch.equal(small.kv.view(torch.uint8), big.kv.view(torch.uint8)[:used])


# ---- pages -----------------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("page_size,kv_heads,head_dim,layers,dtype", [(16, 2, 64, 2, torch.bfloat16), (32, 1, 32, 1, torch.float16), (64, 3, 96, 1, torch.float16), (16, 1, 256, 3, torch.bfloat16),
                                                                      (512, 1, 32, 1, torch.bfloat16)])
@pytest.mark.parametrize("seed", range(2))
def test_random_histories(page_size, kv_heads, head_dim, layers, dtype, seed):
    """Every call in random order on a pool that runs out now and then; everything compared after each."""
    r, g = random.Random(seed), torch.Generator("cuda").manual_seed(seed)
    slots, width = 19, 5
    cache = pg.PagedCache.empty(slots, 26, width * page_size, layers, kv_heads, head_dim, page_size, dtype, bits=8)
    cache.kv.view(torch.uint8).fill_(0x44)
    ref = ref_of(cache)
    said = set()
    for step in range(40):
        n = r.randint(0, slots)
        entries = r.sample(range(slots), n)
        entries = [r.choice([-1, -1, -5, slots, 2 ** 30]) if r.random() < 0.1 else s for s in entries]
        what = r.choice(["advance", "advance", "advance", "fork", "fork", "free", "compact"])
        if what == "advance":
            counts = [r.choice([0, 1, 1, 1, 2, page_size - 1, page_size, page_size + 1, 3 * page_size, -2]) for _ in entries]
            status = torch.full((n,), 99, dtype=torch.uint8, device="cuda")
            cache.advance(ints(entries), ints(counts), status)
            assert status.tolist() == ref.advance(entries, counts)
            said |= set(status.tolist())
            tokens = max([1] + ref.grown)
            k, v = ((torch.randn(n, tokens, kv_heads, head_dim, generator=g, device="cuda") * 2.0 ** r.randint(-3, 3)).to(dtype) for _ in range(2))
            for layer in range(layers):
                if n: cache.write(layer, k, v, ints(entries))
                ref.write(layer, k, v, entries)
        elif what == "fork":
            live = [s for s in entries if 0 <= s < slots]
            half = len(live) // 2
            src = [r.choice(live[:half]) if half else -1 for _ in live[half:]]
            pairs = [r.choice([(-1, d), (slots + 3, d), (s, -1), (s, -7)]) if r.random() < 0.1 else (s, d) for s, d in zip(src, live[half:])]
            status = torch.full((len(pairs),), 99, dtype=torch.uint8, device="cuda")
            cache.fork(ints([s for s, _ in pairs]), ints([d for _, d in pairs]), status)
            assert status.tolist() == ref.fork([s for s, _ in pairs], [d for _, d in pairs])
            said |= set(status.tolist())
        elif what == "free":
            entries = entries[: r.randint(0, 8)]
            cache.free(ints(entries))
            ref.free(entries)
        else:
            used = ints([0])
            cache.compact(used)
            assert int(used) == ref.compact()
        same(cache, ref)
    assert {0, 1} <= said


def test_offsets_beyond_32_bits():
    pages = 5 * 2 ** 30 // (2 * 8 * 64 * 128)               # 5 GB of pages
    kv = torch.zeros(pages, 1, 2, 8, 64, 128, dtype=torch.uint8, device="cuda").view(E4M3)
    scales = torch.ones(pages, 1, 2, 8, 4, device="cuda")
    g = torch.Generator("cuda").manual_seed(3)
    last = list(range(pages - 3, pages))
    refs = torch.ones(pages, dtype=torch.int32, device="cuda")
    refs[pages - 4:] = 0
    cache = pg.PagedCache(kv, torch.full((2, 4), -1, dtype=torch.int32, device="cuda"), ints([0, 0]), refs, scales=scales, dtype=torch.bfloat16)
    cache.refs[pages - 4] = 1
    cache.rescan()
    cache.advance(ints([0]), 130)
    assert cache.table[0].tolist() == last + [-1]
    k, v = new(g, torch.bfloat16, 1, 130, 8, 128), new(g, torch.bfloat16, 1, 130, 8, 128, size=3.0)
    cache.write(0, k, v, ints([0]))
    small = RefCache8(kv[last], scales[last], ints([[0, 1, 2, -1], [-1] * 4]), ints([130, 0]), ints([1, 1, 1]))
    plain = RefCache8(torch.zeros(3, 1, 2, 8, 64, 128).to(E4M3), torch.ones(3, 1, 2, 8, 4), ints([[0, 1, 2, -1], [-1] * 4]), ints([130, 0]), ints([1, 1, 1]))
    plain.grown = [130, 0]
    plain.write(0, k, v, [0])
    assert torch.equal(small.kv, plain.kv) and torch.equal(small.scales, plain.scales) and int((kv.view(torch.uint8)[: pages - 4: 97] != 0).sum()) == 0
    assert torch.equal(bits(cache.read(0, 130, ints([0]))[1]), bits(plain.read(0, 130, [0], [0], torch.bfloat16)[1]))
    q = new(g, torch.bfloat16, 2, 8, 128)
    out, lse = cache.attend(0, q, lse=True)
    check_attend(cache, small, out, lse, 0, q, [0, 1], 128 ** -0.5)
    cache.refs[pages - 4] = 0
    cache.rescan()
    cache.fork(ints([0]), ints([1]))
    assert cache.table[1].tolist() == last[:2] + [pages - 4, -1]
    assert torch.equal(bits(cache.attend(0, q[:1], ints([1]))), bits(out[:1]))
    cache.refs[5:9] = 0
    cache.rescan()
    cache.compact()
    assert cache.table[0].tolist() == [5 + [pages - 4, pages - 3, pages - 2, pages - 1].index(p) for p in last] + [-1]
    assert torch.equal(bits(cache.attend(0, q[:1], ints([0]))), bits(out[:1]))


def test_a_saved_cache_goes_on():
    cache = filled([40, 16, 3], 1, 1, 32, 16, torch.float16, seed=5, width=6, spare=9)
    ref, g = ref_of(cache), torch.Generator("cuda").manual_seed(1)
    again = pg.PagedCache(*(t.clone() for t in (cache.kv, cache.table, cache.lengths, cache.refs)), scales=cache.scales.clone(), dtype=torch.float16)
    again.advance(ints([2, 0]), ints([14, 9]))
    ref.advance([2, 0], [14, 9])
    k, v = new(g, torch.float16, 2, 14, 1, 32), new(g, torch.float16, 2, 14, 1, 32)
    again.write(0, k, v, ints([2, 0]))
    ref.write(0, k, v, [2, 0])
    live = torch.isfinite(ref.scales) & (ref.scales > 0)
    assert torch.equal(again.scales.cpu().double()[live], ref.scales[live]) and torch.equal(codes_of(again), bytes_of(ref.kv))


# ---- streams, graphs, refusals -----------------------------------------------------------------------------------------------------------


def test_two_captured_steps_are_replayed():
    """a search's step with turned queries and keys (one graph) and reading back (another) on one handle: each replay as the same calls made one by one"""
    lengths = [40, 16, 0, 99, 7, 64]
    a, b = (filled(lengths + [0] * 6, 2, 2, 64, 16, torch.bfloat16, seed=5, width=9, spare=40, junk=False) for _ in range(2))
    src, dst = ints(range(6)), ints(range(6, 12))
    g = torch.Generator("cuda").manual_seed(3)
    q, k, v = (new(g, torch.bfloat16, 6, h, 64) for h in (8, 2, 2))
    positions, frequencies = a.lengths[:6].clone(), pg.rotary_frequencies(64)
    made = lambda: ([torch.empty_like(q), torch.empty_like(k)], torch.empty_like(q), [torch.empty(6, 100, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)])  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = pg.PagedCache(a.kv, a.table, a.lengths, a.refs, scales=a.scales, dtype=torch.bfloat16)

    def step(cache, turned, out):
        cache.fork(src, dst)
        cache.advance(dst)
        for layer in (0, 1):
            qr, kr = pg.rotate((q, k), positions, frequencies, out=turned)
            cache.attend(layer, qr, dst, k=kr, v=v, out=out)

    first, second = made(), made()
    side.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0], stream=side):
        step(c, *first[:2])
    with torch.cuda.graph(graphs[1], stream=side):
        c.read(1, 100, dst, k=first[2][0], v=first[2][1])
    for t in range(5):
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        step(b, *second[:2])
        b.read(1, 100, dst, k=second[2][0], v=second[2][1])
        torch.cuda.synchronize()
        for x, y in zip((*first[0], first[1], *first[2]), (*second[0], second[1], *second[2])):
            assert torch.equal(bits(x), bits(y))
        for name in ("kv", "table", "lengths", "refs", "scales"):
            assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), name
        q.copy_(new(g, torch.bfloat16, 6, 8, 64))
        k.mul_(-1.5)
        positions.add_(1)


def test_new_outputs_belong_to_the_handles_stream():
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cache = filled([20, 5], 2, 2, 64, 16, torch.bfloat16)
    torch.cuda.synchronize()
    for t in cache.read(0, 7):
        at = t.data_ptr()
        assert [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]] == [side.cuda_stream]
    side.synchronize()


def cache_and_more():
    cache = filled([20, 5], 2, 2, 64, 16, torch.bfloat16)
    return cache, torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")


def with_(c, **k):
    return pg.PagedCache(**{**dict(kv=c.kv, table=c.table, lengths=c.lengths, refs=c.refs, scales=c.scales, dtype=c.dtype), **k})


REFUSED = [
    ("no scales", lambda c, q, k: with_(c, scales=None)),
    ("no type for the calls", lambda c, q, k: with_(c, dtype=None)),
    ("float32 for the calls", lambda c, q, k: with_(c, dtype=torch.float32)),
    ("scales of another size", lambda c, q, k: with_(c, scales=c.scales[:-1])),
    ("scales of another type", lambda c, q, k: with_(c, scales=c.scales.double())),
    ("scales on the host", lambda c, q, k: with_(c, scales=c.scales.cpu())),
    ("scales that are not dense", lambda c, q, k: with_(c, scales=torch.cat([c.scales, c.scales], -1)[..., ::2])),
    ("scales beside 16 bits", lambda c, q, k: with_(c, kv=c.kv.bfloat16())),
    ("another type beside 16 bits", lambda c, q, k: with_(c, kv=c.kv.bfloat16(), scales=None, dtype=torch.float16)),
    ("another 8-bit type", lambda c, q, k: with_(c, kv=c.kv.float().to(torch.float8_e5m2))),
    ("bits", lambda c, q, k: pg.PagedCache.empty(2, 4, 32, 1, 1, 64, bits=4)),
    ("page size", lambda c, q, k: pg.PagedCache.empty(2, 4, 32, 1, 1, 64, page_size=24, bits=8)),
    ("head size", lambda c, q, k: pg.PagedCache.empty(2, 4, 32, 1, 1, 48, bits=8)),
    ("keys in 8 bits", lambda c, q, k: c.write(0, k.to(E4M3), k.to(E4M3))),
    ("q in another type", lambda c, q, k: c.attend(0, q.half())),
    ("read: layer", lambda c, q, k: c.read(2, 3)),
    ("read: layer below 0", lambda c, q, k: c.read(-1, 3)),
    ("read: layer beyond 32 bits", lambda c, q, k: c.read(2 ** 32, 3)),
    ("read: tokens below 0", lambda c, q, k: c.read(0, -1)),
    ("read: tokens not whole", lambda c, q, k: c.read(0, 1.5)),
    ("read: first below 0", lambda c, q, k: c.read(0, 1, first=-1)),
    ("read: first of long", lambda c, q, k: c.read(0, 1, first=torch.zeros(2, dtype=torch.int64, device="cuda"))),
    ("read: first of other size", lambda c, q, k: c.read(0, 1, first=ints([0]))),
    ("read: slots of long", lambda c, q, k: c.read(0, 1, torch.zeros(1, dtype=torch.int64, device="cuda"))),
    ("read: k of other tokens", lambda c, q, k: c.read(0, 2, k=torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda"))),
    ("read: k of another type", lambda c, q, k: c.read(0, 1, k=torch.zeros(2, 1, 2, 64, dtype=torch.float16, device="cuda"))),
    ("read: k that overlaps", lambda c, q, k: c.read(0, 3, k=torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda").expand(2, 3, 2, 64))),
    ("read: v that overlaps", lambda c, q, k: c.read(0, 3, v=torch.zeros(4000, dtype=torch.bfloat16, device="cuda").as_strided((2, 3, 2, 64), (384, 128, 63, 1)))),
    ("read: keys and values into one tensor", lambda c, q, k: (lambda t: c.read(0, 3, k=t, v=t))(torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device="cuda"))),
    ("read: entries that overlap", lambda c, q, k: c.read(0, 3, v=torch.zeros(4000, dtype=torch.bfloat16, device="cuda").as_strided((2, 3, 2, 64), (256, 128, 64, 1)))),
]


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("what", [n for n, _ in REFUSED])
def test_refusals(what, native, monkeypatch):
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    with pytest.raises(pg.PgxGoError):
        dict(REFUSED)[what](*cache_and_more())


def test_native_and_python_checks_make_the_same_calls(monkeypatch):
    def history():
        g = torch.Generator("cuda").manual_seed(1)
        cache = filled([20, 5, 0, 33], 2, 2, 64, 16, torch.bfloat16, width=6, spare=20, junk=False)
        out = []
        cache.advance()
        cache.write(0, new(g, torch.bfloat16, 4, 2, 64), new(g, torch.bfloat16, 4, 2, 64))
        cache.advance(ints([3, -1, 1]), ints([2, 1, 9]))
        many = new(g, torch.bfloat16, 3, 11, 2, 64)
        cache.write(1, many, many.flip(1), ints([3, -1, 1]))
        out += [*cache.attend(1, new(g, torch.bfloat16, 2, 6, 64), ints([3, 0]), lse=True), cache.attend(0, new(g, torch.bfloat16, 2, 4, 64), ints([1, 0]), k=many[:2, 0], v=many[:2, 1])]
        out += [*cache.read(1, 7), *cache.read(0, 3, ints([2, 3, 3]), ints([0, 30, -1])), *cache.read(0, 9, first=4), *cache.read(1, 0)]
        wide = torch.zeros(2, 4, 2, 6, 64, dtype=torch.bfloat16, device="cuda")
        out += list(cache.read(1, 6, None, 2, wide[0].transpose(1, 2), wide[1].transpose(1, 2)))
        cache.fork(ints([3, 0]), ints([2, 1]))
        return out + [cache.kv.view(torch.uint8), cache.scales, cache.table, cache.lengths, cache.refs]

    assert pg.cache_binding._fast is not None
    native = history()
    monkeypatch.setattr(pg.cache_binding, "_fast", None)
    for a, b in zip(native, history()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_numbers_are_whole(native, monkeypatch):
    cache, q, k = cache_and_more()
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    for call in (lambda: cache.read(0.5, 1), lambda: cache.read("0", 1), lambda: cache.read(0, None), lambda: cache.read(0, 2 ** 31), lambda: cache.read(0, 1, first=0.5), lambda: cache.read(0, 1, first=2 ** 31),
                 lambda: cache.read(0, 1, first=[0, 0]), lambda: cache.read(0, 1, slots=[0]), lambda: cache.read(0, 1, k=3), lambda: cache.read(0, 1, v=q)):
        with pytest.raises(pg.PgxGoError):
            call()
    one = torch.ones(1, dtype=torch.int64).numpy()[0]
    assert torch.equal(cache.read(one, one, first=one)[0], cache.read(1, 1, first=1)[0])


def test_lists_on_another_device_are_left_alone():
    """A handle that says it is on another device stands for tensors on another device: neither the native checks nor Python's pass them on."""
    cache, q, k = cache_and_more()
    before = cache.kv.view(torch.uint8).clone()
    one = ints([0])
    cache._shape = cache._shape[:4] + (1,) + cache._shape[5:]
    cache.device = torch.device("cuda:1")
    out = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: cache.read(0, 1, one, k=out, v=out.clone()), lambda: cache.read(0, 1, None, ints([0, 0]), k=out, v=out.clone()), lambda: cache.write(0, k[:1], k[:1], one)):
        with pytest.raises(pg.PgxGoError):
            call()
    assert torch.equal(cache.kv.view(torch.uint8), before)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,head_dim,most", [(150, 64, 5280), (150, 128, 4400), (100, 64, 9600), (520, 256, 2400), (150, 256, 4400)])
def test_a_new_token_far_behind_the_first_tiles(n, head_dim, most, dtype):
    """more than 32 tiles for a wavefront, four or two to a row, in one block or two: the last one's pages and scales are looked up after the token was written"""
    lengths = [most - 1, most - 16, most - 17, most - 250, 4100 % most, 0, 1] + [0] * (n - 7)
    g = torch.Generator("cuda").manual_seed(n)
    a, b = (filled(lengths, 1, 2, head_dim, 16, dtype, seed=2, width=-(-most // 16), spare=2 * n) for _ in range(2))
    ref = ref_of(a)
    for step in range(2):
        q = new(g, dtype, n, 4, head_dim)
        k, v = ((torch.randn(n, 2, head_dim, generator=g, device="cuda") * (8.0 if step else 0.5)).to(dtype) for _ in range(2))
        room = ints([1 if m + step < most else 0 for m in lengths])
        for cache in (a, b):
            cache.advance(counts=room)
        ref.advance(range(n), room.tolist())
        b.write(0, k, v)
        got, want = a.attend(0, q, k=k, v=v, lse=True), b.attend(0, q, lse=True)
        assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
        assert torch.equal(a.kv.view(torch.uint8), b.kv.view(torch.uint8)) and torch.equal(a.scales.view(torch.int32), b.scales.view(torch.int32))
        ref.write_last(0, k, v, range(n))
        assert torch.equal(codes_of(a), bytes_of(ref.kv))
        check_attend(a, ref, got[0][:7], got[1][:7], 0, q[:7], range(7), head_dim ** -0.5)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_finite_values_near_the_types_end_stay_finite(dtype):
    """The code nearest to a value above 63488 (bfloat16: 2^127.95) at its scale is 256, beyond the type's largest number: what is read back is that number, 2^-4 of
    the value away at most, and attention over float16's stays finite too, in the row of one wavefront, of several, and of several blocks.  Every block's scale s is the
    one for the largest number, 448 s / 2 < most <= 448 s; values below 2^-6 s are held in steps of 2^-9 s, half a step 2^-10 s = 2^-4 2^-6 s."""
    D, most, s = 64, torch.finfo(dtype).max, 2.0 ** (8 if dtype is torch.float16 else 120)
    ends = [most, -most, most * 0.97, -most * 0.9698, most * 0.95, most / 2, 1.0]
    x = torch.tensor(ends, dtype=torch.float64).repeat(-(-D * 5 // len(ends)))[: D * 5].reshape(5, 1, D).to(dtype).cuda()      # every end in every token
    cache = pg.PagedCache.empty(5, 10, 32, 1, 1, D, dtype=dtype, bits=8)
    x[1, 0, 3], x[2, 0, 5] = float("nan"), float("-inf")
    odd = ~torch.isfinite(x)
    cache.advance()
    cache.write(0, x, x)
    for held in cache.read(0, 1):
        assert torch.equal(torch.isnan(held[:, 0]), odd)
        held, want = held[:, 0][~odd].double(), x[~odd].double()
        assert torch.isfinite(held).all() and ((held - want).abs() <= 2.0 ** -4 * want.abs().clamp(min=s / 64)).all()
    if dtype is torch.float16:   # (sums of the largest bfloat16 numbers go beyond 32 bits)
        for tokens, pages in ((1, 1), (16, 1), (300, 19), (2100, 132)):
            cache = pg.PagedCache.empty(2, 2 * pages, pages * 16, 1, 1, D, dtype=dtype, bits=8)
            cache.advance(counts=tokens)
            loud = torch.full((2, tokens, 1, D), most, dtype=dtype, device="cuda")
            loud[1, :, 0, 1::2], loud[1, :, 0, ::4] = -most, 63500.0
            cache.write(0, torch.zeros_like(loud), loud)
            out = cache.attend(0, torch.ones(2, 3, D, dtype=dtype, device="cuda")).double()
            want = loud[:, 0].double()                                   # (all tokens are alike)
            assert torch.isfinite(out).all() and ((out - want).abs() <= 2.0 ** -4 * want.abs()).all(), tokens


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("bits_", [8, 16])
def test_keys_and_values_read_into_memory_that_they_share(bits_, native, monkeypatch):
    if not native:
        monkeypatch.setattr(pg.cache_binding, "_fast", None)
    cache = pg.PagedCache.empty(2, 6, 48, 1, 2, 64, bits=bits_)
    g = torch.Generator("cuda").manual_seed(1)
    k, v = new(g, torch.bfloat16, 2, 40, 2, 64), new(g, torch.bfloat16, 2, 40, 2, 64)
    cache.advance(counts=40)
    cache.write(0, k, v)
    want = cache.read(0, 5, first=30)
    memory = torch.zeros(2, 11, 5, 64, dtype=torch.bfloat16, device="cuda")
    for a, b in ((memory[:, :5, :2], memory[:, 4:9, :2]), (memory[:, :5, :2], memory[:, :5, 1:3]), (memory[:, 0:10:2, :2], memory[:, 2:11:2, :2][:, :5]),
                 (memory[:1].expand(2, 11, 5, 64)[:, :5, :2], memory[:, 6:, :2]), (memory.flatten()[:1280].view(2, 5, 2, 64), memory.flatten()[1279:2559].view(2, 5, 2, 64))):
        with pytest.raises(pg.PgxGoError):
            cache.read(0, 5, first=30, k=a, v=b)
    assert (memory == 0).all()
    for a, b in ((memory[:, :5, :2], memory[:, :5, 2:4]), (memory[:, 0:10:2, :2], memory[:, 1:11:2, :2]), (memory[:, :5, 0:4:2], memory[:, :5, 1:4:2])):   # rows between each other's
        got = cache.read(0, 5, first=30, k=a, v=b)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("how", ["one", "several", "attend", "attend by a launch of its own"])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
def test_tokens_into_blocks_whose_scales_are_no_powers_of_two(head_dim, how):
    """The product with a reciprocal is off by what the reciprocal (2^-23) and the product (2^-24) are, less than 2^-22 together; half a step of the code on top.  The step is that
    of the exact quotient, 2^-3 of its power of two, or the next one's where 2^-22 takes it there."""
    g = torch.Generator("cuda").manual_seed(head_dim)
    filled_, new_ = 5, 3 if how == "several" else 1
    scales = torch.tensor([1.25, 1.1, 0.7, 1 / 3, 3e-3, 0.0179, 2.0 ** -20 * 1.9, 3e3], device="cuda")
    n, D = len(scales), head_dim
    cache = filled([filled_] * n, 1, 2, D, 16, torch.bfloat16, seed=1, width=1, spare=0)
    held = cache.table[:, 0].long()
    cache.scales[held] = scales[:, None, None, None, None].expand(n, 1, 2, 2, 1).contiguous()
    before = cache.kv.float()[held][:, 0, :, :, :filled_].double()
    cache.advance(counts=new_)
    k, v = new(g, torch.bfloat16, n, new_, 2, D), new(g, torch.bfloat16, n, new_, 2, D, size=0.3)
    if how == "several": cache.write(0, k, v)
    elif how == "one": cache.write(0, k[:, 0], v[:, 0])
    else: cache.attend(0, torch.zeros(n, 2 if how == "attend" else 40, D, dtype=torch.bfloat16, device="cuda"), k=k[:, 0], v=v[:, 0])
    now = cache.scales[held][:, 0, :, :, 0].double()                                               # [n][2][2]
    x = torch.stack((k, v), 1).transpose(2, 3).double()                                            # [n][2][2][tokens][D]
    own = torch.tensor([[[scale_for(m) for m in heads] for heads in which] for which in x.abs().amax((3, 4)).tolist()], dtype=torch.float64, device="cuda")
    was = scales.double()[:, None, None].expand_as(own)
    raised = own > was
    assert torch.equal(now, torch.where(raised, own, was)) and raised.any() and not raised.all()
    codes = cache.kv.float()[held][:, 0].double()

    def near(code, exact):
        _, e = torch.frexp(exact.abs() * (1 + 2.0 ** -22))
        return ((code - exact).abs() <= torch.exp2((e.double() - 1).clamp(min=-6) - 4) + 2.0 ** -22 * exact.abs()).all()

    now, was, raised = (t[..., None, None] for t in (now, was, raised))
    assert near(codes[:, :, :, filled_: filled_ + new_], x / now) and near(codes[:, :, :, :filled_], before * was / now)
    assert torch.equal(torch.where(raised, 0.0, codes[:, :, :, :filled_]), torch.where(raised, 0.0, before))
    got = cache.read(0, new_, first=filled_)[0].transpose(1, 2).double()
    want = codes[:, 0, :, filled_: filled_ + new_] * now[:, 0]
    assert ((got - want).abs() <= 2.0 ** -8 * 1.01 * want.abs()).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("tokens", [2, 17, 33, 40])
def test_many_short_prompts(tokens, head_dim, dtype):
    """thousands of entries of one to four blocks, which a wavefront writes one after the other: the same as in calls of fewer entries, a wavefront to each block, and some as in the
    plain model; beginning anywhere in a block, with and without earlier tokens that are louder or quieter, entries without room, left out and no slots"""
    n, kv_heads, layers = 2100, 2, 2
    r, g = random.Random(tokens + head_dim), torch.Generator("cuda").manual_seed(head_dim)
    lengths = [r.choice([0, 0, 1, 7, 15, 16, 17, 30, 31]) for _ in range(n)]
    a, b = (filled(lengths, layers, kv_heads, head_dim, 16, dtype, seed=2, width=5, spare=4 * n, junk=False) for _ in range(2))
    counts = [r.choice([0, 1, tokens // 2, tokens - 1, tokens, tokens, tokens + 3]) for _ in range(n)]
    order = r.sample(range(n), n)
    entries = [r.choice([-1, n, 2 ** 30]) if r.random() < 0.05 else s for s in order]
    size = torch.exp2(torch.randint(-4, 5, (n, tokens, 1, 1), generator=g, device="cuda").float())
    k, v = ((torch.randn(n, tokens, kv_heads, head_dim, generator=g, device="cuda") * size).to(dtype) for _ in range(2))
    plain = [i for i in range(n) if 0 <= entries[i] < n][:12]
    ref = ref_of(b)
    for cache in (a, b):
        cache.advance(ints(order), ints([counts[s] for s in order]))
    ref.table, ref.lengths = b.table.cpu(), b.lengths.cpu()
    ref.grown = [max(c, 0) for c in counts]
    a.write(1, k, v, ints(entries))
    assert n * 2 * kv_heads * ((tokens + 14) // 16 + 1) >= 16384
    for i in range(0, n, 150):                 # (fewer than 16384 blocks in a call)
        b.write(1, k[i: i + 150], v[i: i + 150], ints(entries[i: i + 150]))
    assert torch.equal(a.kv.view(torch.uint8), b.kv.view(torch.uint8)) and torch.equal(a.scales.view(torch.int32), b.scales.view(torch.int32))
    ref.write(1, k[plain].cpu(), v[plain].cpu(), [entries[i] for i in plain])
    pages = [p for i in plain for p in ref.table[entries[i]].tolist() if p >= 0]
    assert torch.equal(codes_of(a)[pages], bytes_of(ref.kv[pages])) and torch.equal(a.scales.cpu().double()[pages], ref.scales[pages])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("head_dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("n,width,kv_heads,heads", [(2050, 24, 2, 4), (2050, 64, 2, 2), (1030, 24, 4, 4)])
def test_a_new_token_with_two_wavefronts_to_a_row(n, width, kv_heads, heads, head_dim, dtype):
    """4096 rows and more of 11 to 32 tiles: what attention writes and gives is what write and attention give"""
    r, g = random.Random(width), torch.Generator("cuda").manual_seed(head_dim)
    most = width * 16
    lengths = [r.choice([0, 1, 15, 16, 31, 32, 33, 63, 64, most // 2, most - 17, most - 3]) if i < 40 else r.choice([0, 5, 31, 33, 70]) for i in range(n)]
    a, b = (filled(lengths, 1, kv_heads, head_dim, 16, dtype, seed=2, width=width, spare=3 * n) for _ in range(2))
    assert n * kv_heads >= 4096 and 10 < (most + 31) // 32 <= 32
    for step in range(3):
        q = new(g, dtype, n, heads, head_dim)
        size = torch.exp2(torch.randint(-3, 4, (n, 1, 1), generator=g, device="cuda").float())
        k, v = ((torch.randn(n, kv_heads, head_dim, generator=g, device="cuda") * size).to(dtype) for _ in range(2))
        for cache in (a, b):
            cache.advance()
        b.write(0, k, v)
        got, want = a.attend(0, q, k=k, v=v, lse=True), b.attend(0, q, lse=True)
        assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
        assert torch.equal(a.kv.view(torch.uint8), b.kv.view(torch.uint8)) and torch.equal(a.scales.view(torch.int32), b.scales.view(torch.int32))
    few = list(range(12))
    check_attend(a, ref_of(a), got[0][:12], got[1][:12], 0, q[:12], few, head_dim ** -0.5)
