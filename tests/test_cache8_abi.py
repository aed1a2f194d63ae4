"""CPU-only checks of the paged cache held in 8 bits: exported symbols, refused arguments, and the plain model's own rounding."""
import ctypes as C
import math
import random

import pytest
import torch

import paper_2303_17503_amd as pg
from cache8_ref import RefCache8, e4m3, scale_for
from paper_2303_17503_amd import cache_binding
from test_cache_abi import opts
from test_host_and_abi import declared_functions


def test_library_exports_what_is_declared():
    names = declared_functions("pgxcache.h", "pgxcache_")
    assert {"pgxcache_init_e4m3", "pgxcache_read"} <= set(names)
    L = C.CDLL(pg.LIB_PATH)
    assert all(hasattr(L, n) for n in names)


def test_argument_errors_need_no_gpu():
    L = cache_binding.lib()
    h, p, n = C.c_void_p(), C.c_void_p(4096), L.pgxcache_work_bytes(C.byref(opts()))
    init = lambda o=None, kv=p, scales=p, table=p, work=p, nbytes=n, out=C.byref(h): L.pgxcache_init_e4m3(  # noqa: E731
        out, C.byref(o or opts()), kv, scales, table, p, p, work, nbytes)
    for bad in (dict(scales=None), dict(scales=C.c_void_p(4098)), dict(o=opts(head_dim=48)), dict(kv=None), dict(kv=C.c_void_p(4104)), dict(table=None), dict(work=None),
                dict(nbytes=n - 1), dict(out=None), dict(o=opts(type=0))):
        assert init(**bad) == -1, bad
    assert L.pgxcache_read(None, 0, 1, None, None, 0, 1, p, 64, 64, 64, p, 64, 64, 64) == -1


def test_the_plain_model_rounds_as_torch_does():
    g = torch.Generator().manual_seed(0)
    x = torch.cat([torch.randn(20000, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-12, 8, (20000,), generator=g).double()), torch.tensor([0.0, -0.0, 448.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -10 * 1.01, 0.4375])])
    x = x.clamp(-448, 448).float()
    assert torch.equal(e4m3(x.double()), x.to(torch.float8_e4m3fn).double())
    assert math.isnan(float(e4m3(torch.tensor(math.inf, dtype=torch.float64)))) and math.isnan(float(e4m3(torch.tensor(math.nan, dtype=torch.float64))))
    for m, want in ((0.0, 2.0 ** -100), (448.0, 1.0), (448.5, 2.0), (447.0, 1.0), (224.0, 0.5), (224.1, 1.0), (2.0 ** -130, 2.0 ** -100)):
        assert scale_for(m) == want, m


@pytest.mark.parametrize("page", [16, 64])
def test_the_plain_model_keeps_its_own_rules(page):
    """what is held is within 2^-4 of the value (2^-10 of the scale below 2^-6 of it), and once more where a later token raised the scale; forks and moved pages hold the same"""
    r, g = random.Random(page), torch.Generator().manual_seed(page)
    kv = torch.zeros(20, 1, 2, 1, page, 32).to(torch.float8_e4m3fn)
    c = RefCache8(kv, torch.ones(20, 1, 2, 1, page // 16), torch.full((4, 8), -1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(20, dtype=torch.int32))
    said = torch.zeros(2, 0, 32, dtype=torch.float64)
    while said.shape[1] < 90:
        n = r.choice([1, 1, 1, 5, 17])
        assert c.advance([2], [n]) == [0]
        x = torch.randn(2, n, 32, generator=g, dtype=torch.float64) * 2.0 ** r.randint(-3, 3)
        c.write(0, x[0][None, :, None], x[1][None, :, None], [2])
        said = torch.cat([said, x], 1)
        held = c.sequence(2, 0)[:, 0]
        scale = c.scales[c.table[2, : c._pages(said.shape[1])].long(), 0, :, 0].permute(1, 0, 2).reshape(2, -1).repeat_interleave(16, 1)[:, : said.shape[1], None]
        bound = 2 * torch.maximum(said.abs() * 2.0 ** -4, scale * 2.0 ** -10)
        assert ((held - said).abs() <= bound * 1.0001).all()
    assert c.fork([2], [0]) == [0] and torch.equal(c.sequence(0, 0), c.sequence(2, 0))
    before = c.sequence(0, 0)
    c.free([2])
    c.compact()
    assert torch.equal(c.sequence(0, 0), before)
    k, v = c.read(0, 5, [0, 3, -1], [88, 0, 0], torch.float64)
    n = int(c.lengths[0])
    assert torch.equal(k[0, : n - 88, 0], before[0, 0, 88:93][: 5]) and (k[1:] == 0).all() and (v[0, n - 88:] == 0).all()


def test_what_is_held_after_the_scale_was_raised():
    """Each raise rounds to half a step, 2^-10 of the new scale, what is below 2^-6 of it; the scales before it add up to less than the last: 2^-9 of that in all.
    What is larger moves without rounding and stays within 2^-4 of itself."""
    g = torch.Generator().manual_seed(3)

    def after(x, scales):
        s = scales[0]
        code = e4m3(x / s)
        for now in scales[1:]:
            code, s = e4m3(code * s / now), now
        return code * s

    one = torch.tensor([0.65626], dtype=torch.float64)
    assert float((after(one, [1.0, 64.0]) - one).abs()) > 2.0 ** -10 * 64      # 0.6875 at first, then 0.75
    for _ in range(60):
        raises = torch.randint(1, 5, (int(torch.randint(0, 7, (1,), generator=g)),), generator=g).cumsum(0)
        scales = [2.0 ** -3] + [2.0 ** (-3 + int(e)) for e in raises]
        x = (torch.rand(4000, generator=g, dtype=torch.float64) * 2 - 1) * 448 * scales[0] * torch.exp2(-torch.rand(4000, generator=g, dtype=torch.float64) * 20)
        bound = torch.where(x.abs() >= scales[-1] * 2.0 ** -6, x.abs() * 2.0 ** -4, torch.tensor(scales[-1] * 2.0 ** -9))
        assert ((after(x, scales) - x).abs() <= bound).all()
        first = after(x, scales[:1])
        assert ((first - x).abs() <= torch.where(x.abs() >= scales[0] * 2.0 ** -6, x.abs() * 2.0 ** -4, torch.tensor(scales[0] * 2.0 ** -10))).all()
