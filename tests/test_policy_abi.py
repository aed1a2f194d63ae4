"""CPU-only checks of the policy operators' boundary: exported symbols, refused arguments, and the plain form's own gradient."""
import ctypes as C

import torch

import paper_2303_17503_amd as pg
import policy_ref as ref
from paper_2303_17503_amd import policy_binding
from test_host_and_abi import declared_functions


def test_library_exports_every_declared_policy_symbol():
    names = declared_functions("pgxpolicy.h", "pgxpolicy_")
    assert {"pgxpolicy_logits", "pgxpolicy_sample", "pgxpolicy_loss"} <= set(names)
    L = C.CDLL(pg.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n


def test_argument_errors_need_no_gpu():
    L = policy_binding.lib()
    p = C.c_void_p(4096)
    ok = lambda **k: policy_binding._Adjust(**k)  # noqa: E731
    logits = lambda rows=4, actions=82, x=p, kind=0, pitch=82, adjust=None, out=p, out_pitch=82: L.pgxpolicy_logits(  # noqa: E731
        rows, actions, x, kind, pitch, None if adjust is None else C.byref(adjust), 0, out, out_pitch, None)
    assert logits(rows=0) == 0 and logits(rows=0, x=None, out=None) == 0         # nothing to do
    for bad in (dict(rows=-1), dict(actions=0), dict(actions=8193), dict(x=None), dict(x=C.c_void_p(4098)), dict(kind=3), dict(kind=-1), dict(pitch=-1),
                dict(out=None), dict(out_pitch=81), dict(adjust=ok(repetition=-1.0)), dict(adjust=ok(repetition=float("nan"))),
                dict(adjust=ok(repetition=float("inf"))), dict(adjust=ok(temperature=-0.5)), dict(adjust=ok(temperature=float("nan"))),
                dict(adjust=ok(record=4096, record_len=65536)), dict(adjust=ok(record=4096, record_len=-1)), dict(adjust=ok(mask=4096, mask_pitch=-3)),
                dict(adjust=ok(bias=4096, bias_pitch=-1))):
        assert logits(**bad) == -1, bad
    assert L.pgxpolicy_sample(4, 82, p, 0, 82, None, None, 0, None, None, None) == -1                          # no actions
    assert L.pgxpolicy_sample(4, 82, p, 0, 82, None, p, -1, p, None, None) == -1                               # noise pitch
    loss = lambda target, taken, grad, pitch=82: L.pgxpolicy_loss(4, 82, p, 0, 82, None, target, 82, taken, None, 0.0, 1.0, None, None, grad, pitch, None)  # noqa: E731
    assert loss(None, None, p) == -1 and loss(p, p, p) == -1 and loss(p, None, None) == -1 and loss(p, None, p, 80) == -1
    assert L.pgxpolicy_strerror(-1) == b"invalid argument" and L.pgxpolicy_strerror(0) == b"ok"


def test_plain_form_against_the_written_out_gradient():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(6, 11, generator=g)
    mask = (torch.rand(6, 11, generator=g) < 0.6).to(torch.uint8)
    mask[2] = 0
    y, w, beta, T = torch.rand(6, 11, generator=g), torch.randn(6, generator=g), 0.25, 0.5
    loss, entropy, grad = ref.loss(x, y, weight=w, entropy=beta, mask=mask, temperature=T)
    z, live = ref.adjusted(x, mask=mask, temperature=T)
    logp = ref.log_probabilities(z, live)
    flat, p = torch.where(live, logp, 0.0), logp.exp()
    y = torch.where(live, y.double(), 0.0)
    h = -(p * flat).sum(1)
    want = (w.double()[:, None] * (y.sum(1, keepdim=True) * p - y) + beta * p * (flat + h[:, None])) / T
    assert torch.allclose(grad, torch.where(live, want, 0.0), atol=1e-12) and torch.allclose(entropy, h, atol=1e-12)
    assert loss[2] == 0 and (grad[2] == 0).all()
