"""CPU-only checks of the rotary positions' boundary: exported symbols, refused arguments, frequencies, and the plain form's own gradient."""
import ctypes as C
import math

import pytest
import torch

import paper_2303_17503_amd as pg
from paper_2303_17503_amd import rotary_binding
from rotary_ref import turned
from test_host_and_abi import declared_functions


def test_library_exports_every_declared_symbol():
    names = declared_functions("pgxrotary.h", "pgxrotary_")
    assert "pgxrotary_turn" in names
    L = C.CDLL(pg.LIB_PATH)
    assert all(hasattr(L, n) for n in names)


def test_argument_errors_need_no_gpu():
    L = rotary_binding.lib()
    P = rotary_binding._Part
    p, far = 4096, 1 << 30

    def call(entries=2, tokens=3, D=64, R=64, kind=0, positions=p, frequencies=p, magnitude=1.0, parts=1, part=None, **k):
        a = dict(in_=p, in_entry=3 * 64, in_token=64, in_head=64, out=far, out_entry=3 * 64, out_token=64, out_head=64, heads=1)
        a.update(k)
        array = (P * 2)(P(**a), P(**{**a, "out": far * 2}))
        return L.pgxrotary_turn(entries, tokens, D, R, kind, positions, 3, 1, frequencies, magnitude, 0, 0, parts, array if part is None else part, None)

    assert call(entries=0) == 0 and call(tokens=0, in_=None, out=None) == 0 and call(heads=0) == 0            # nothing to do
    for bad in (dict(entries=-1), dict(tokens=-1), dict(D=1, R=2), dict(D=1025), dict(R=0), dict(R=63), dict(R=66), dict(kind=3), dict(kind=-1), dict(positions=None),
                dict(positions=p + 2), dict(frequencies=None), dict(frequencies=p + 4), dict(magnitude=math.nan), dict(magnitude=math.inf), dict(parts=0), dict(parts=3),
                dict(in_=None), dict(out=None), dict(in_=p + 2), dict(out=far + 2), dict(heads=-1), dict(heads=65537), dict(entries=65536, tokens=32768),
                dict(out_entry=128), dict(out_token=63), dict(heads=2, out_head=63), dict(heads=2), dict(out_token=0), dict(out=p, out_entry=256)):
        assert call(**bad) == -1, bad
    same = (P * 2)(*[P(p, 192, 64, 64, far, 192, 64, 64, 1)] * 2)
    assert L.pgxrotary_turn(2, 3, 64, 64, 0, p, 3, 1, p, 1.0, 0, 0, 2, same, None) == -1
    assert L.pgxrotary_turn(2, 3, 64, 64, 0, p, 3, 1, p, 1.0, 0, 0, 1, None, None) == -1
    assert L.pgxrotary_strerror(-1) == b"invalid argument" and L.pgxrotary_strerror(0) == b"ok"


def test_frequencies():
    f = pg.rotary_frequencies(64, device="cpu")
    assert f.dtype is torch.float64 and f.shape == (32,) and float(f[0]) == 1.0 and math.isclose(float(f[16]), 0.01, rel_tol=1e-15)
    assert torch.equal(pg.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu"), f / 4)
    slow = pg.rotary_frequencies(64, scaling="base", factor=8.0, device="cpu")
    assert float(slow[0]) == 1.0 and math.isclose(float(slow[-1]), float(f[-1]) / 8, rel_tol=1e-12) and (slow[1:] < f[1:]).all()
    parts = pg.rotary_frequencies(64, scaling="parts", factor=8.0, original=4096, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], f[turns >= 32]) and torch.equal(parts[turns <= 1], f[turns <= 1] / 8) and (parts >= f / 8).all() and (parts <= f).all()
    assert (parts[1:] < parts[:-1]).all()


@pytest.mark.parametrize("bad", [dict(rotary_dim=63), dict(rotary_dim=0), dict(rotary_dim=1026), dict(rotary_dim=8.0), dict(base=0.0), dict(base=math.inf), dict(scaling="some"),
                                 dict(factor=2.0), dict(scaling="linear", factor=-1.0), dict(scaling="parts", factor=2.0), dict(scaling="parts", factor=2.0, original=0),
                                 dict(scaling="parts", factor=2.0, original=8, low=3.0, high=3.0), dict(scaling="base", factor=2.0, rotary_dim=2)])
def test_frequencies_that_are_refused(bad):
    with pytest.raises(pg.PgxGoError):
        pg.rotary_frequencies(**{**dict(rotary_dim=64, device="cpu"), **bad})


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_plain_form_turns_back_and_is_its_own_gradient(interleaved):
    g = torch.Generator().manual_seed(0)
    f = pg.rotary_frequencies(10, device="cpu")
    x = torch.randn(3, 2, 13, generator=g, dtype=torch.float64, requires_grad=True)
    p = torch.tensor([0, 7, -100000])
    y = turned(x, p, f, interleaved, 1.5)
    assert torch.equal(y[0, :, 10:], x[0, :, 10:]) and torch.allclose(y[0, :, :10], x[0, :, :10] * 1.5)
    assert torch.allclose(turned(y, p, f, interleaved, 1 / 1.5, True), x, rtol=1e-12)
    w = torch.randn(3, 2, 13, generator=g, dtype=torch.float64)
    (y * w).sum().backward()
    assert torch.allclose(x.grad, turned(w, p, f, interleaved, 1.5, True), rtol=1e-12)
    # products depend on the distance alone
    q, k = torch.randn(2, 1, 1, 10, generator=g, dtype=torch.float64)
    at = lambda v, n: turned(v, torch.tensor([n]), f, interleaved)  # noqa: E731
    assert torch.allclose((at(q, 50) * at(k, 43)).sum(), (at(q, 1007) * at(k, 1000)).sum())
