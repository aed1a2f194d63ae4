"""CPU-only checks of the paged cache's boundary: exported symbols, sizes, refused arguments; and the plain model against itself."""
import ctypes as C

import torch

import paper_2303_17503_amd as pg
from cache_ref import RefCache
from paper_2303_17503_amd import cache_binding
from test_host_and_abi import declared_functions


def test_library_exports_every_declared_cache_symbol():
    names = declared_functions("pgxcache.h", "pgxcache_")
    assert {"pgxcache_init", "pgxcache_advance", "pgxcache_write", "pgxcache_attend", "pgxcache_fork", "pgxcache_free", "pgxcache_compact"} <= set(names)
    L = C.CDLL(pg.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n


def opts(**k):
    o = dict(slots=8, pages=100, width=10, page_size=16, layers=2, kv_heads=2, head_dim=64, type=2)
    o.update(k)
    return cache_binding._Opts(*[o[n] for n, _ in cache_binding._Opts._fields_[:-1]], None)


def test_sizes_and_argument_errors_need_no_gpu():
    L = cache_binding.lib()
    size = lambda **k: L.pgxcache_work_bytes(C.byref(opts(**k)))  # noqa: E731
    assert size() >= 100 // 8 + 8 * 8 + 100 * 12 and size() % 256 == 0 and size(pages=200000) > size() + 199000 * 12
    for bad in (dict(slots=0), dict(pages=0), dict(width=0), dict(width=2 ** 20 + 1), dict(layers=0), dict(kv_heads=0), dict(page_size=8), dict(page_size=24),
                dict(page_size=2048), dict(head_dim=48), dict(head_dim=0), dict(type=0), dict(type=3), dict(pages=2 ** 31 - 1)):
        assert size(**bad) == 0, bad
    assert size(width=2 ** 20, page_size=1024) > 0 and size(width=2 ** 20, page_size=1024, layers=4096, kv_heads=8) == 0   # pages of 16 GB
    assert L.pgxcache_work_bytes(None) == 0
    h, p, n = C.c_void_p(), C.c_void_p(4096), size()
    init = lambda o=None, kv=p, table=p, lengths=p, refs=p, work=p, nbytes=n, out=C.byref(h): L.pgxcache_init(  # noqa: E731
        out, C.byref(o or opts()), kv, table, lengths, refs, work, nbytes)
    for bad in (dict(o=opts(head_dim=48)), dict(kv=None), dict(kv=C.c_void_p(4104)), dict(table=None), dict(table=C.c_void_p(4098)), dict(lengths=None),
                dict(refs=None), dict(work=None), dict(work=C.c_void_p(4096 + 64)), dict(nbytes=n - 1), dict(out=None)):
        assert init(**bad) == -1, bad
    assert L.pgxcache_destroy(None) == -1 and L.pgxcache_rescan(None) == -1 and L.pgxcache_compact(None, None) == -1 and L.pgxcache_free(None, 1, None) == -1
    assert L.pgxcache_advance(None, 1, None, None, 1, None) == -1 and L.pgxcache_fork(None, 1, p, p, None) == -1
    assert L.pgxcache_strerror(-1) == b"invalid argument" and L.pgxcache_strerror(-3) == b"out of host memory"


def test_the_plain_model_keeps_its_own_rules():
    kv = torch.zeros(12, 1, 2, 1, 16, 32)
    c = RefCache(kv, torch.full((5, 4), -1, dtype=torch.int32), torch.zeros(5, dtype=torch.int32), torch.zeros(12, dtype=torch.int32))
    assert c.advance([3, 1, 0], [17, 16, 65]) == [0, 0, 2]
    assert c.table[3].tolist() == [0, 1, -1, -1] and c.table[1].tolist() == [2, -1, -1, -1]
    k = torch.arange(3 * 17.0).reshape(3, 17, 1, 1).expand(3, 17, 1, 32)
    c.write(0, k, -k, [3, 1, 0])
    assert c.fork([3, 1], [0, 2]) == [0, 0] and c.table[0].tolist() == [0, 3, -1, -1] and c.refs[:4].tolist() == [2, 1, 2, 1]
    assert torch.equal(c.sequence(0, 0), c.sequence(3, 0)) and torch.equal(c.sequence(2, 0), c.sequence(1, 0))
    c.free([3])
    assert c.refs[:4].tolist() == [1, 0, 2, 1] and c.compact() == 3 and c.table[0].tolist() == [0, 1, -1, -1]
    assert c.sequence(0, 0)[0, 0, :, 0].tolist() == list(range(17))
