"""CPU-only checks of the rotary positions' boundary: exported symbols, refused arguments, frequencies, and the plain form's own gradient."""
import ctypes as C
import math
import os
import subprocess

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


def test_outputs_that_share_memory_with_other_tensors():
    """each refused before anything is launched"""
    L, P, base = rotary_binding.lib(), rotary_binding._Part, 1 << 20
    row, size = 64 * 4, 2 * 3 * 2 * 64 * 4            # bytes of a row and of a whole tensor [2][3][2][64]

    def call(*parts):
        array = (P * 2)(*[P(i, *a, o, *b, h) for i, a, o, b, h in parts])
        return L.pgxrotary_turn(2, 3, 64, 64, 0, 4096, 3, 1, 4096, 1.0, 0, 0, len(parts), array, None)

    dense, a, b, far, more = (384, 128, 64), base, base + size, base + 8 * size, base + 12 * size
    wide = (3 * 2 * 128, 2 * 128, 128)                # rows with as much room behind each
    for bad in ([(a, dense, b, dense, 2), (b, dense, a, dense, 2)],                        # two tensors exchanged
                [(a, dense, b, dense, 2), (b, dense, far, dense, 2)],                      # one's output is the other's input
                [(a, dense, far, dense, 2), (b, dense, a, dense, 2)],
                [(a, dense, far, dense, 2), (b, dense, far, dense, 2)],                    # one output twice
                [(a, dense, far, dense, 2), (b, dense, far + size - row, dense, 2)],       # outputs that share a row
                [(a, dense, far, dense, 2), (b, dense, far + size - 4, dense, 2)],         # or an element
                [(a, dense, far, dense, 2), (b, dense, a + row, dense, 1)],
                [(a, dense, a + row, dense, 2)], [(a, dense, a + 4, dense, 2)], [(a, dense, a - size + 4, dense, 2)],      # an output that begins inside its own input
                [(a, dense, a, (384, 64, 192), 2)],                                        # or is it in another order
                [(a, wide, a + 32 * 4, wide, 2)],                                          # between the rows, but for half of them
                [(a, (0, 0, 0), a, dense, 2)],                                             # over an input whose rows repeat
                [(a, dense, far, dense, 2), (a, dense, a, dense, 2)]):                     # an input that both read, in place
        assert call(*bad) == -1, bad
    assert call((a, dense, far, dense, 0), (b, dense, far, dense, 0)) == 0                 # nothing in either


PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "rows_apart.hpp"
static uint32_t x = 1;
static int below(int n) { x = x * 1664525u + 1013904223u; return (int)((x >> 8) % (uint32_t)n); }
static void rows(const Rows& r, int64_t row, std::vector<char>& at, int bit, bool& meets) {
  for (int64_t i = 0; i < r.sizes[0]; ++i)
    for (int64_t t = 0; t < r.sizes[1]; ++t)
      for (int64_t h = 0; h < r.sizes[2]; ++h)
        for (int64_t e = 0; e < row; ++e) {
          char& c = at[(size_t)(((intptr_t)r.p >> 1) + i * r.strides[0] + t * r.strides[1] + h * r.strides[2] + e)];
          if (c & ~bit) meets = true;
          c |= (char)bit;
        }
}
int main() {
  int wrong = 0, meeting = 0, looked = 400000;
  std::vector<char> at(16384);
  for (int k = 0; k < looked; ++k) {
    const int row = 1 + below(5);
    Rows r[2];
    const bool alike = below(2);     // the same strides but for some
    for (int j = 0; j < 2; ++j) {
      r[j].p = (const void*)(intptr_t)(2 * (8000 + below(below(3) ? 40 : 300)));
      for (int d = 0; d < 3; ++d) {
        r[j].sizes[d] = below(20) ? 1 + below(4) : 0;
        r[j].strides[d] = j && alike && below(8) ? r[0].strides[d] : below(4) ? below(41) - 10 : below(301) - 150;
      }
    }
    std::fill(at.begin(), at.end(), 0);
    bool before = false, meets = false;
    rows(r[0], row, at, 1, before);
    rows(r[1], row, at, 2, meets);
    wrong += rows_meet(r[0], r[1], row, 2) != meets || rows_meet(r[1], r[0], row, 2) != meets;
    meeting += meets;
  }
  // sizes that outgrow 64 bits as bytes, and layouts that do not nest
  const int64_t big = (int64_t)1 << 62;
  wrong += rows_meet(Rows{(void*)4096, {1 << 30, 1, 1}, {big, 1, 1}}, Rows{(void*)(4096 + 64), {1 << 30, 1, 1}, {big, 1, 1}}, 32, 2);
  wrong += !rows_meet(Rows{(void*)4096, {1 << 30, 1, 1}, {big, 1, 1}}, Rows{(void*)(4096 + 62), {1 << 30, 1, 1}, {big, 1, 1}}, 32, 2);
  wrong += !rows_meet(Rows{(void*)4096, {1 << 20, 1 << 20, 1}, {1000003, 1009, 1}}, Rows{(void*)5001, {1 << 20, 1 << 20, 1}, {1000033, 1013, 1}}, 1, 2);
  printf("%d wrong of %d, %d meeting\n", wrong, looked, meeting);
  return wrong != 0 || meeting < looked / 10 || meeting > looked - looked / 10;
}
"""


def test_whether_rows_meet_against_every_element(tmp_path):
    src, exe = tmp_path / "meet.cpp", tmp_path / "meet"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(os.path.dirname(rotary_binding.__file__), "csrc"), "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.startswith("0 wrong of "), r.stdout


@pytest.mark.parametrize("bad", [dict(scaling="parts", factor=2.0, original=8192, low=-math.inf),
                                 dict(scaling="parts", factor=2.0, original=8192, low=-math.inf, high=math.inf),
                                 dict(scaling="parts", factor=2.0, original=8192, high=math.nan), dict(scaling="parts", factor=2.0, original=math.nan),
                                 dict(scaling="base", factor=1e200, rotary_dim=4), dict(scaling="base", factor=1e10, base=1e300), dict(base=math.nan), dict(scaling="linear", factor=math.nan),
                                 dict(base=1e-300, scaling="linear", factor=1e-200), dict(rotary_dim=True)])
def test_frequencies_that_would_not_be_finite(bad):
    with pytest.raises(pg.PgxGoError):
        pg.rotary_frequencies(**{**dict(rotary_dim=64, device="cpu"), **bad})


def test_frequencies_at_the_ends():
    """ends that leave every number finite are no reason to refuse"""
    f = pg.rotary_frequencies(64, device="cpu")
    assert torch.equal(pg.rotary_frequencies(64, scaling="parts", factor=2.0, original=8192, high=math.inf, device="cpu"), f / 2)
    assert torch.equal(pg.rotary_frequencies(64, scaling="parts", factor=2.0, original=math.inf, device="cpu"), f)
