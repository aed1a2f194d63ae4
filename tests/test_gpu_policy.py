"""adjust_logits, sample_actions and policy_loss against plain forms in 64 bits (and, where the header fixes every rounding, in 32).

Tolerances.  u = 2^-24.  An adjusted logit is the 32-bit one to the bit.  A log-probability z - top - log(total): two subtractions,
each off by at most u times its operands (at most 2 Z each, Z the largest |z|), and a logarithm of a sum of up to 8192 terms,
added in runs of at most 32 and then pairwise, each term an exponential with a relative error of at most (Z + 4) u from its argument's
scaling and the instruction: 4 Z u + (2 Z + 64) u, doubled: (12 Z + 128) u.  Gradients: p has that error relatively, as has y
through the sums; |w| (sum y + 1) and the entropy's term bound what it multiplies; then the rounding to the logits' type."""
import math

import pytest
import torch

import paper_2303_17503_amd as pg
import policy_ref as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUNDING = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -24, "bf16": 2.0 ** -126}
SIZES = [1, 2, 7, 8, 9, 15, 82, 122, 128, 129, 200, 362, 384, 385, 1000, 2048, 2049, 8192]


def bits(t):
    return t.view(torch.int32)


def error_of_logp(z):
    big = float(z[torch.isfinite(z)].abs().max()) if torch.isfinite(z).any() else 0.0
    return (12 * big + 128) * U


def inputs(rows, actions, dtype, seed, padded=False, record=0, time_major=False):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, actions, generator=g) * 3).to(TYPES[dtype]).cuda()
    width = actions + (37 if padded else 0)
    mask = (torch.rand(rows, width, generator=g) < torch.rand(rows, 1, generator=g)).to(torch.uint8)
    mask[::5] = 0                                   # rows in which nothing can be played
    if rows > 1:
        mask[1] = 0
        mask[1, actions - 1] = 1                    # and one with a single action
    how = {"mask": mask.cuda(), "bias": torch.randn(actions, generator=g).cuda()}
    if record:
        moves = torch.randint(-1, actions + 1, (rows, record), generator=g, dtype=torch.int32) % max(2, actions // 2 + 1)
        moves[:, ::7] = -1
        moves = moves.cuda()
        how["record"] = moves.t().contiguous().t() if time_major else moves
        how["begin"] = torch.randint(-2, record, (rows,), generator=g, dtype=torch.int32).cuda()
        how["end"] = torch.randint(0, record + 3, (rows,), generator=g, dtype=torch.int32).cuda()
        how.update(repetition=1.3, frequency=0.15, presence=0.4)
    t = torch.rand(rows, generator=g) + 0.1
    t[2::4] = 0.0
    how["temperature"] = t.cuda()
    return x, how, g


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("actions", SIZES)
def test_adjusted_logits_to_the_bit_and_log_probabilities(actions, dtype):
    rows = 23
    x, how, _ = inputs(rows, actions, dtype, actions, padded=actions % 2 == 0, record=40, time_major=actions % 3 == 0)
    z, _ = ref.adjusted(x.float(), dtype=torch.float32, **how)
    got = pg.adjust_logits(x, **how).cpu()
    assert torch.equal(bits(got + 0.0), bits(z + 0.0))
    z64, possible = ref.adjusted(x, **how)
    want = ref.log_probabilities(z64, possible)
    got = pg.adjust_logits(x, normalize=True, **how).cpu().double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)) and torch.equal(torch.isfinite(got), possible)
    # the adjustment itself is rounded at up to six places
    live = torch.isfinite(want)
    assert not live.any() or (got - want)[live].abs().max() <= error_of_logp(z64) + 12 * U * (float(z64[live].abs().max()) + 16)


@pytest.mark.parametrize("part", ["mask", "bias", "bias rows", "record", "temperature", "number", "nothing"])
@pytest.mark.parametrize("actions", [5, 82, 362, 700])
def test_each_part_of_the_adjustment_by_itself(actions, part):
    x, how, g = inputs(9, actions, "f32", 3, record=30)
    only = {"mask": ["mask"], "bias": ["bias"], "record": ["record", "begin", "end", "repetition", "frequency", "presence"], "temperature": ["temperature"]}.get(part, [])
    how = {k: v for k, v in how.items() if k in only}
    if part == "bias rows": how = {"bias": torch.randn(9, actions + 3, generator=g).cuda()[:, :actions]}
    if part == "number": how = {"temperature": 0.7}
    z, possible = ref.adjusted(x, dtype=torch.float32, **how)
    assert torch.equal(bits(pg.adjust_logits(x, **how).cpu() + 0.0), bits(z + 0.0))
    a, logp = pg.sample_actions(x, **how)
    assert torch.equal(a.cpu(), ref.sampled(z, possible, None, how.get("temperature")))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("actions", SIZES)
def test_sampled_actions_are_the_definitions(actions, dtype):
    rows = 33
    x, how, g = inputs(rows, actions, dtype, 100 + actions, padded=actions % 2 == 1, record=25, time_major=actions % 2 == 0)
    noise = -torch.log(-torch.log(torch.rand(rows, actions, generator=g).clamp(1e-6, 1 - 1e-6)))
    if actions > 3:
        x[3:6] = x[3:6, :1].clone()                # equal logits: the lowest index
        noise[3:6] = 0.5
        how["bias"][:] = 0.25
    z, possible = ref.adjusted(x.float(), dtype=torch.float32, **how)
    for n in (noise, None):
        a, logp = pg.sample_actions(x, noise=None if n is None else n.cuda(), **how)
        want = ref.sampled(z, possible, n, how["temperature"])
        assert torch.equal(a.cpu(), want)
        z64, live = ref.adjusted(x, **how)
        lp = ref.log_probabilities(z64, live)
        lp = torch.where(want >= 0, lp.gather(1, want.clamp(min=0).long()[:, None])[:, 0], 0.0)
        assert (logp.cpu().double() - lp).abs().max() <= error_of_logp(z64) + 12 * U * (float(z64[live].abs().max()) + 16)
        assert (logp.cpu()[want < 0] == 0).all()


def test_draws_follow_the_distribution():
    rows, actions = 40000, 9
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.tensor([[0.0, 1.0, -1.0, 0.5, 2.0, -2.0, 0.3, 0.7, 1.5]], device="cuda").expand(rows, actions).contiguous()
    mask = torch.tensor([[1, 1, 0, 1, 1, 1, 1, 0, 1]], dtype=torch.uint8, device="cuda").expand(rows, actions)   # one row for all
    noise = -torch.log(-torch.log(torch.rand(rows, actions, generator=g, device="cuda").clamp(1e-7, 1 - 1e-7)))
    a, _ = pg.sample_actions(x, noise=noise, mask=mask, temperature=0.8)
    p = torch.softmax(torch.where(mask[0] != 0, x[0] / 0.8, float("-inf")).double(), 0).cpu()
    share = torch.bincount(a.long(), minlength=actions).cpu().double() / rows
    assert ((share - p).abs() <= 5 * (p * (1 - p) / rows).sqrt() + 1e-12).all()   # five standard deviations


@pytest.mark.parametrize("op", ["adjust", "sample", "loss"])
@pytest.mark.parametrize("actions", [6, 82, 362])
def test_what_masked_places_hold_does_not_matter(actions, op):
    rows = 16
    x, how, g = inputs(rows, actions, "f32", 5, record=10)
    dead = how["mask"][:, :actions] == 0
    noise = torch.randn(rows, actions, generator=g).cuda()
    target = torch.rand(rows, actions, generator=g).cuda()
    outs = []
    for junk in (0.0, float("nan"), float("inf"), float("-inf"), torch.finfo(torch.float32).min, torch.finfo(torch.float32).max):
        y, n, t = (torch.where(dead, torch.full_like(v, junk), v) for v in (x, noise, target))
        if op == "adjust":
            outs.append([pg.adjust_logits(y, **how), pg.adjust_logits(y, normalize=True, **how)])
        elif op == "sample":
            outs.append(list(pg.sample_actions(y, noise=n, **how)))
        else:
            outs.append(list(pg.policy_loss(y, t, entropy=0.1, **how)))
    for o in outs[1:]:
        for a, b in zip(o, outs[0]):
            assert torch.equal(a.view(torch.int32), b.view(torch.int32))
    assert all(not torch.isnan(v.float()).any() for v in outs[0])


def test_masks_of_the_lowest_value_and_of_minus_infinity_in_the_bias():
    lowest = torch.finfo(torch.float32).min
    x = torch.tensor([[1.0, 2.0, 3.0, 4.0]], device="cuda").repeat(4, 1)
    bias = torch.tensor([[0.0, 0.0, lowest, lowest], [float("-inf"), 0.0, 0.0, float("-inf")],
                         [lowest, lowest, lowest, lowest], [float("-inf")] * 4], device="cuda")
    a, logp = pg.sample_actions(x, bias=bias)
    assert a.tolist() == [1, 2, 0, -1]
    want = [torch.log_softmax(torch.tensor([1.0, 2.0]), 0)[1], torch.log_softmax(torch.tensor([2.0, 3.0]), 0)[1], -math.log(4.0), 0.0]
    assert (logp.cpu() - torch.tensor(want)).abs().max() <= 200 * U
    loss, entropy, grad = pg.policy_loss(x, torch.full((4,), 1, dtype=torch.int32, device="cuda"), bias=bias)
    assert torch.isfinite(loss).all() and torch.isfinite(grad).all() and (grad[3] == 0).all() and loss[3] == 0 and entropy[3] == 0
    assert abs(float(entropy[2]) - math.log(4.0)) <= 200 * U


@pytest.mark.parametrize("actions", [5, 82, 362, 700])
def test_nan_logits_are_not_possible_and_nan_noise_counts_as_minus_infinity(actions):
    rows, nan, inf = 12, float("nan"), float("inf")
    x, how, g = inputs(rows, actions, "f32", 31, record=15)
    how["mask"][:] = 1
    hurt = torch.rand(rows, actions, generator=g).cuda() < 0.3
    hurt[:, actions // 2] = False
    y = torch.where(hurt, torch.full_like(x, nan), x)
    without = {**how, "mask": (~hurt).to(torch.uint8)}                 # the same with those actions masked
    raw = pg.adjust_logits(y, **how)
    assert torch.isnan(raw[hurt]).all() and torch.equal(raw[~hurt], pg.adjust_logits(x, **how)[~hurt])
    noise = torch.randn(rows, actions, generator=g).cuda()
    target, moves = torch.rand(rows, actions, generator=g).cuda(), torch.randint(0, actions, (rows,), generator=g, dtype=torch.int32).cuda()
    for f in (lambda l, h: [pg.adjust_logits(l, normalize=True, **h)], lambda l, h: pg.sample_actions(l, noise=noise, **h),
              lambda l, h: pg.policy_loss(l, target, entropy=0.1, **h), lambda l, h: pg.policy_loss(l, moves, entropy=0.1, **h)):
        for a, b in zip(f(y, how), f(x, without)):
            assert torch.equal(a + 0, b + 0)
    odd = noise.clone()
    odd[:, ::2] = nan
    odd[:, 1::2] = -inf
    odd[0, actions - 1] = -1e30
    odd[1] = nan
    how["temperature"] = torch.ones(rows, device="cuda")
    a, logp = pg.sample_actions(y, noise=odd, **how)
    first = [int((~hurt[b]).nonzero()[0]) for b in range(rows)]
    if not hurt[0, actions - 1]:
        first[0] = actions - 1
    assert a.tolist() == first and torch.isfinite(logp).all()
    odd[2, actions // 2] = inf
    assert pg.sample_actions(y, noise=odd, **how)[0][2] == actions // 2


@pytest.mark.parametrize("target", ["visits", "moves"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("actions", [1, 3, 8, 13, 82, 122, 362, 385, 2048, 5000])
def test_loss_and_gradient(actions, dtype, target):
    rows, bonus, scale = 21, 0.05, 0.5
    x, how, g = inputs(rows, actions, dtype, 7 + actions, padded=True, record=20 if actions % 2 == 0 else 0, time_major=True)
    weight = torch.randn(rows, generator=g).cuda()
    if target == "visits":
        y = torch.rand(rows, actions, generator=g).pow(6)
        y = (y / y.sum(1, keepdim=True)).cuda()
        most = y.sum(1).cpu().double()
    else:
        y = torch.randint(-1, actions + 1, (rows,), generator=g, dtype=torch.int32).cuda()   # -1 and one beyond the last: no move
        most = torch.ones(rows, dtype=torch.float64)
    loss, entropy, grad = pg.policy_loss(x, y, weight=weight, entropy=bonus, grad_scale=scale, **how)
    want, h, dx = ref.loss(x, y, weight=weight, entropy=bonus, **how)
    z, live = ref.adjusted(x, **how)
    eps = error_of_logp(z) + 12 * U * (float(z[live].abs().max()) + 16) if live.any() else U
    big = float(z[live].max() - z[live].min()) if live.any() else 0.0
    w = weight.cpu().double().abs()
    assert ((loss.cpu().double() - want).abs() <= eps * (w * (most + 1) * (1 + big) + bonus * (2 + big)) * 2).all()
    assert (entropy.cpu().double() - h).abs().max() <= eps * (2 + big) * 2
    slope = 1.3 / torch.where(how["temperature"] > 0, how["temperature"], 1.0).cpu().double()
    bound = scale * slope * eps * (w * (most + 1) + bonus * (2 + big)) * 4
    dx = dx * scale
    assert grad.dtype == TYPES[dtype]
    assert ((grad.cpu().double() - dx).abs() <= bound[:, None] + ROUNDING[dtype] * 1.01 * dx.abs() + TINY[dtype]).all()
    assert (grad.cpu()[~live] == 0).all()


@pytest.mark.parametrize("actions", [2, 9, 82])
def test_gradient_against_differences(actions):
    """(L(x + h) - L(x - h)) / 2h of the kernel's own loss, h = 1/32: off by h^2 / 6 times a third derivative, which for a log-sum-exp of
    sharpness s = 1/T <= 2 is at most 0.1 s^3 per unit of weight and, with p (log p)^2 <= 1, 4 s^3 per unit of entropy bonus, and by the losses' rounding
    over h."""
    rows, h = 6, 1.0 / 32
    g = torch.Generator().manual_seed(11)
    x = torch.randn(rows, actions, generator=g).cuda()
    how = {"mask": (torch.rand(rows, actions, generator=g) < 0.7).to(torch.uint8).cuda(), "temperature": 0.5}
    weight = (torch.rand(rows, generator=g) + 0.5).cuda()
    y = torch.softmax(torch.randn(rows, actions, generator=g), 1).cuda()
    bonus = 0.1
    of = lambda v: pg.policy_loss(v, y, weight=weight, entropy=bonus, **how)[0].double()  # noqa: E731
    grad = pg.policy_loss(x, y, weight=weight, entropy=bonus, **how)[2].double()
    for a in range(actions):
        step = torch.zeros_like(x)
        step[:, a] = h
        slope = (of(x + step) - of(x - step)) / (2 * h)
        assert ((slope - grad[:, a]).abs() <= h * h / 6 * 8 * (0.1 * 1.5 + 4 * bonus) + 400 * U * 8 / h).all()


def test_strides_broadcasts_and_given_outputs():
    rows, actions = 19, 82
    x, how, g = inputs(rows, actions, "bf16", 9)
    wide = torch.zeros(rows, 2 * actions + 5, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + actions] = x
    odd = wide[:, 3:3 + actions]                    # rows of 169 elements, from an odd one on
    assert torch.equal(bits(pg.adjust_logits(odd, **how)), bits(pg.adjust_logits(x, **how)))
    out = torch.full((rows, 100), 7.0, device="cuda")
    pg.adjust_logits(odd, out=out[:, 9:91], **how)
    assert torch.equal(bits(out[:, 9:91].contiguous()), bits(pg.adjust_logits(x, **how))) and (out[:, :9] == 7).all() and (out[:, 91:] == 7).all()
    y = torch.softmax(torch.randn(rows, actions, generator=g), 1).cuda()
    gradient = torch.full((rows, 99), 7.0, dtype=torch.bfloat16, device="cuda")
    _, _, into = pg.policy_loss(odd, y, grad=gradient[:, 1:83], **how)
    assert into.data_ptr() == gradient[:, 1:83].data_ptr()
    assert torch.equal(gradient[:, 1:83], pg.policy_loss(x, y, **how)[2]) and (gradient[:, :1] == 7).all() and (gradient[:, 83:] == 7).all()
    every = how["mask"][:1].expand(rows, actions)
    assert torch.equal(bits(pg.adjust_logits(x, mask=every)), bits(pg.adjust_logits(x, mask=every.contiguous())))
    assert torch.equal(bits(pg.adjust_logits(x, mask=every != 0)), bits(pg.adjust_logits(x, mask=every)))
    a = torch.empty(rows, dtype=torch.int32, device="cuda")
    logp = torch.empty(rows, device="cuda")
    got = pg.sample_actions(x, out=a, logp=logp, **how)
    assert got[0] is a and got[1] is logp and torch.equal(a, pg.sample_actions(x, **how)[0])
    empty = pg.sample_actions(x[:0], mask=how["mask"][:0])
    assert empty[0].shape == (0,) and pg.adjust_logits(x[:0]).shape == (0, actions)


def test_record_orders_and_bounds():
    rows, actions, plies = 70, 362, 500
    g = torch.Generator().manual_seed(2)
    x = torch.randn(rows, actions, generator=g).cuda()
    moves = torch.randint(0, 20, (rows, plies), generator=g, dtype=torch.int32).cuda()
    how = dict(repetition=2.0, frequency=0.125, presence=1.0)
    want = pg.adjust_logits(x, record=moves, **how)
    assert torch.equal(bits(want.cpu()), bits(ref.adjusted(x, record=moves, dtype=torch.float32, **how)[0]))
    for other in (moves.t().contiguous().t(), torch.stack([moves, moves * 0 + 400], 2)[:, :, 0], moves.flip(1)):
        assert torch.equal(bits(pg.adjust_logits(x, record=other, **how)), bits(want))
    same = pg.adjust_logits(x, record=torch.full((rows, 65535), 5, dtype=torch.int32, device="cuda"), frequency=1.0)
    assert (same[:, 5] == x[:, 5] - 65535.0).all() and torch.equal(same[:, 6:], x[:, 6:])
    none = pg.adjust_logits(x, record=moves, begin=torch.full((rows,), 600, dtype=torch.int32, device="cuda"), **how)
    assert torch.equal(none, x) and torch.equal(pg.adjust_logits(x, record=moves[:, :0], **how), x)


def test_another_stream_and_a_captured_graph():
    rows, actions = 64, 362
    x, how, g = inputs(rows, actions, "bf16", 21, record=50, time_major=True)
    noise = torch.randn(rows, actions, generator=g).cuda()
    want = pg.sample_actions(x, noise=noise, **how)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = x.clone()
        got = pg.sample_actions(y, noise=noise, **how)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    a, logp = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pg.sample_actions(x, noise=noise, out=a, logp=logp, **how)
    for k in range(4):
        noise.copy_(torch.randn(rows, actions, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        eager = pg.sample_actions(x, noise=noise, **how)
        assert torch.equal(a, eager[0]) and torch.equal(logp, eager[1])


def test_moves_from_the_environments_own_mask():
    env = pg.GoEnv(50, 9, seed=1, auto_reset=True, line_padded=True)
    mask = env.new_mask()
    env.bind_outputs(mask)
    g = torch.Generator("cuda").manual_seed(3)
    for t in range(60):
        x = torch.randn(50, env.A, generator=g, device="cuda")
        a, _ = pg.sample_actions(x, noise=torch.randn(50, env.A, generator=g, device="cuda"), mask=mask)
        assert (mask.gather(1, a.long()[:, None]) == 1).all()
        env.step(a)
    assert int(env.export_state()["illegal"].sum()) == 0


REFUSED = [
    ("logits of another type", lambda x, k: pg.adjust_logits(x.double())),
    ("logits on the host", lambda x, k: pg.adjust_logits(x.cpu())),
    ("one dimension", lambda x, k: pg.adjust_logits(x[0])),
    ("strided rows", lambda x, k: pg.adjust_logits(x[:, ::2])),
    ("too many actions", lambda x, k: pg.adjust_logits(torch.zeros(2, 8193, device="cuda"))),
    ("no actions", lambda x, k: pg.adjust_logits(x[:, :0])),
    ("narrow mask", lambda x, k: pg.sample_actions(x, mask=k["mask"][:, :50])),
    ("mask of floats", lambda x, k: pg.sample_actions(x, mask=k["mask"].float())),
    ("mask of other rows", lambda x, k: pg.sample_actions(x, mask=k["mask"][:3])),
    ("bias in bf16", lambda x, k: pg.adjust_logits(x, bias=k["bias"].bfloat16())),
    ("bias too short", lambda x, k: pg.adjust_logits(x, bias=k["bias"][:9])),
    ("record of long", lambda x, k: pg.adjust_logits(x, record=torch.zeros(8, 5, dtype=torch.int64, device="cuda"))),
    ("record too long", lambda x, k: pg.adjust_logits(x, record=torch.zeros(8, 65536, dtype=torch.int32, device="cuda"))),
    ("record of other rows", lambda x, k: pg.adjust_logits(x, record=torch.zeros(5, 8, dtype=torch.int32, device="cuda"))),
    ("penalty without record", lambda x, k: pg.adjust_logits(x, repetition=1.5)),
    ("repetition 0", lambda x, k: pg.adjust_logits(x, record=torch.zeros(8, 5, dtype=torch.int32, device="cuda"), repetition=0.0)),
    ("temperature 0", lambda x, k: pg.adjust_logits(x, temperature=0.0)),
    ("temperature nan", lambda x, k: pg.adjust_logits(x, temperature=float("nan"))),
    ("temperatures of other rows", lambda x, k: pg.adjust_logits(x, temperature=torch.ones(7, device="cuda"))),
    ("noise of other size", lambda x, k: pg.sample_actions(x, noise=torch.zeros(8, 5, device="cuda"))),
    ("out of other type", lambda x, k: pg.sample_actions(x, out=torch.zeros(8, dtype=torch.int64, device="cuda"))),
    ("target of long", lambda x, k: pg.policy_loss(x, torch.zeros(8, dtype=torch.int64, device="cuda"))),
    ("target of other size", lambda x, k: pg.policy_loss(x, torch.zeros(8, 5, device="cuda"))),
    ("no target", lambda x, k: pg.policy_loss(x, None)),
    ("gradient in another type", lambda x, k: pg.policy_loss(x, torch.zeros(8, dtype=torch.int32, device="cuda"), grad=torch.zeros(8, 82, device="cuda", dtype=torch.float16))),
    ("overlapping gradient", lambda x, k: pg.policy_loss(x, torch.zeros(8, dtype=torch.int32, device="cuda"), grad=torch.zeros(1, 82, device="cuda").expand(8, 82))),
]


@pytest.mark.parametrize("what", [n for n, _ in REFUSED])
def test_refusals(what):
    x = torch.zeros(8, 82, device="cuda")
    k = {"mask": torch.ones(8, 82, dtype=torch.uint8, device="cuda"), "bias": torch.zeros(82, device="cuda")}
    with pytest.raises(pg.PgxGoError):
        dict(REFUSED)[what](x, k)


@pytest.mark.parametrize("what", [n for n, _ in REFUSED])
def test_refusals_without_the_native_checks(what, monkeypatch):
    monkeypatch.setattr(pg.policy_binding, "_fast", None)
    test_refusals(what)


@pytest.mark.parametrize("actions", [5, 82, 362])
def test_native_and_python_checks_make_the_same_calls(actions, monkeypatch):
    x, how, g = inputs(12, actions, "bf16", 4, padded=True, record=9, time_major=True)
    noise, y, w = torch.randn(12, actions, generator=g).cuda(), torch.rand(12, actions, generator=g).cuda(), torch.randn(12, generator=g).cuda()
    moves = torch.randint(-1, actions, (12,), generator=g, dtype=torch.int32).cuda()
    plain = {k: v for k, v in how.items() if k == "mask"}

    def every():
        out = []
        for h in (how, plain, {**plain, "temperature": 2}, {**plain, "bias": noise}):
            out += [pg.adjust_logits(x, **h), pg.adjust_logits(x, normalize=True, **h), *pg.sample_actions(x, noise=noise, **h), *pg.sample_actions(x, **h),
                    *pg.policy_loss(x, y, weight=w, entropy=0.1, grad_scale=0.5, **h), *pg.policy_loss(x, moves, **h)]
        return out

    calls = []
    real = pg.policy_binding._fast

    class Counting:
        def __getattr__(self, name):
            def call(*a):
                got = getattr(real, name)(*a)
                calls.append(got)
                return got
            return call

    assert real is not None
    monkeypatch.setattr(pg.policy_binding, "_fast", Counting())
    native = every()
    assert len(calls) == 24 and all(type(c) is tuple for c in calls)   # none was left to Python
    monkeypatch.setattr(pg.policy_binding, "_fast", None)
    for a, b in zip(native, every()):
        assert a.dtype == b.dtype and torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32), b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


@pytest.mark.parametrize("layout", ["plies", "games", "far"])
@pytest.mark.parametrize("actions", [82, 700, 3000])
def test_begins_and_ends_at_the_limits_of_their_type(actions, layout):
    """max(begin, 0) <= t < min(end, plies) for every int32; with 16, 64 and 256 lanes to a row; "far": moves beyond 32-bit offsets in bytes"""
    low, high = -2 ** 31, 2 ** 31 - 1
    ranges = [(high, high), (high, low), (low, high), (low, low), (high - 3, high), (high - 15, 7), (high - 254, high), (0, high), (6, high), (7, high), (8, 8), (high, 7), (-1, 1)]
    rows, plies = 2 if layout == "far" else len(ranges), 9
    g = torch.Generator().manual_seed(actions)
    moves = torch.randint(0, 5, (len(ranges), plies), generator=g, dtype=torch.int32).cuda()
    x = torch.randn(len(ranges), actions, generator=g).cuda()
    begin, end = (torch.tensor([r[i] for r in ranges], dtype=torch.int64).int().cuda() for i in (0, 1))
    how = dict(repetition=1.5, frequency=0.25, presence=0.5)
    if layout == "far":
        memory = torch.full((2 ** 29 + plies,), -1, dtype=torch.int32, device="cuda")
    for first in range(0, len(ranges), rows):
        part = slice(first, min(first + rows, len(ranges)))
        record = moves[part]
        n = record.shape[0]
        if layout == "games": record = record.t().contiguous().t()
        if layout == "far":
            far = memory.as_strided((n, plies), (2 ** 29, 1))
            record = far.copy_(record)
        now = dict(how, record=record, begin=begin[part], end=end[part])
        want, _ = ref.adjusted(x[part], dtype=torch.float32, **dict(now, record=moves[part]))
        assert torch.equal(bits(pg.adjust_logits(x[part], **now).cpu()), bits(want))


@pytest.mark.parametrize("target", ["visits", "moves"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("actions", [5, 82, 362, 700, 3000])
def test_the_gradient_is_0_where_an_action_is_not_possible(actions, dtype, target):
    """whatever the temperature, the scale and the bonus multiply to, and beside a logit of +infinity, which makes the possible ones NaN"""
    rows = 14
    x, how, g = inputs(rows, actions, "f32", 50 + actions, record=12)
    how["mask"][:, actions // 2] = 1
    x, dead = x.to(TYPES[dtype]), how["mask"][:, :actions] == 0
    y = torch.rand(rows, actions, generator=g).cuda() if target == "visits" else torch.randint(-1, actions, (rows,), generator=g, dtype=torch.int32).cuda()
    for t, scale, bonus in ((1e-4, 65536.0, 1.0), (1e-6, 65536.0, 0.01), (1e-30, 1.0, 0.5), (1e-36, 1e9, 0.5), (1.0, 3e38, 3e38), (0.5, -65536.0, 1e30)):
        how["temperature"] = torch.full((rows,), t, device="cuda")
        grad = pg.policy_loss(x, y, entropy=bonus, grad_scale=scale, **how)[2]
        assert (grad[dead] == 0).all() and (scale / t > 1e12 or not torch.isnan(grad).any()), (t, scale, bonus)
    how["temperature"] = torch.ones(rows, device="cuda")
    x[:, actions // 2] = float("inf")
    for bonus in (0.0, 0.1):
        loss, entropy, grad = pg.policy_loss(x, y, entropy=bonus, **how)
        assert (grad[dead] == 0).all() and torch.isnan(grad[~dead]).all() and torch.isnan(loss).all() and torch.isnan(entropy).all()


@pytest.mark.parametrize("actions", [4, 82, 700])
def test_the_loss_at_logits_of_the_lowest_value(actions):
    """A mask of the type's lowest value leaves the action possible, with a log-probability of about that value: the loss for a target there is as large,
    to one rounding each of the difference, its product with the share and the weight (4 u), and beside the highest value it is capped there."""
    low, high = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    x = torch.randn(6, actions, generator=torch.Generator().manual_seed(1))
    x[:, 1] = torch.tensor([low, low, -3.1e38, -2.9e38, low, low])
    x[4, 2] = x[5, 2] = high
    share = torch.zeros(6, actions)
    share[:, 1], share[:, 0] = 0.25, 0.5
    want = -x[:, 1].double() + torch.tensor([0, 0, 0, 0, high, high]).double()   # (what lies beside it is below its rounding)
    want = torch.minimum(want, torch.full_like(want, high))
    loss = pg.policy_loss(x.cuda(), torch.full((6,), 1, dtype=torch.int32, device="cuda"))[0].cpu().double()
    assert ((loss - want).abs() <= 4 * U * want).all()
    loss, _, grad = pg.policy_loss(x.cuda(), share.cuda(), entropy=0.25)
    loss = loss[:4].cpu().double()
    assert ((loss - 0.25 * want[:4]).abs() <= 4 * U * want[:4]).all()
    assert torch.isfinite(grad).all() and (grad[:, 1] == -0.25).all()


@pytest.mark.parametrize("divisor", ["temperature", "repetition", "both"])
def test_the_sign_of_zero_is_kept(divisor):
    """every operation rounded by itself: -0 / T is -0; to the bit, zeros of both signs beside numbers of all sizes"""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(9, 82, generator=g) * 2.0 ** torch.randint(-60, 60, (9, 82), generator=g)
    x[:, ::3], x[:, 1::6] = -0.0, 0.0
    x = x.cuda()
    how = {} if divisor == "repetition" else {"temperature": torch.rand(9, generator=g).cuda() + 0.3}
    if divisor != "temperature":
        how.update(record=torch.randint(0, 82, (9, 60), generator=g, dtype=torch.int32).cuda(), repetition=1.3)
    want = ref.adjusted(x, dtype=torch.float32, **how)[0]
    assert torch.equal(bits(pg.adjust_logits(x, **how).cpu()), bits(want)) and torch.signbit(want[want == 0]).any()


@pytest.mark.parametrize("actions", [5, 82, 362, 383, 513, 1030, 2049, 2561, 2567, 3075, 4099, 8191])
def test_outputs_in_the_place_of_the_logits(actions):
    """sizes whose last chunk, moved back, shares actions with one of the same wavefront and of another"""
    x, how, g = inputs(300, actions, "f32", 8, record=0)
    moves = torch.randint(0, actions, (300,), generator=g, dtype=torch.int32).cuda()
    for h in (how, {k: how[k] for k in ("bias", "temperature")}):
        for normalize in (False, True):
            want, y = pg.adjust_logits(x, normalize=normalize, **h), x.clone()
            assert torch.equal(bits(pg.adjust_logits(y, normalize=normalize, out=y, **h)), bits(want))
        want, y = pg.policy_loss(x, moves, entropy=0.1, **h), x.clone()
        got = pg.policy_loss(y, moves, entropy=0.1, grad=y, **h)
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want)) and torch.equal(bits(y), bits(want[2]))


@pytest.mark.parametrize("actions", [82, 700, 3000])
def test_rows_beyond_32_bit_offsets(actions):
    """pitches of more than 2^31 elements, and of 2^32 bytes for the mask: the second row as in dense memory"""
    x, how, g = inputs(7, actions, "bf16", 3, record=0)
    x, how = x[1:3].clone(), {"mask": how["mask"][1:3].clone(), "bias": torch.randn(2, actions, generator=g).cuda(), "temperature": how["temperature"][:2].clone()}
    noise, y = torch.randn(2, actions, generator=g).cuda(), torch.rand(2, actions, generator=g).cuda()

    def far(t, pitch=2 ** 31 + 9):
        return torch.empty(pitch + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (pitch, 1)).copy_(t)

    fx, fhow, fnoise, fy = far(x), dict(how, mask=far(how["mask"], 2 ** 32 + 9), bias=far(how["bias"])), far(noise), far(y)
    assert torch.equal(bits(pg.adjust_logits(fx, out=far(noise), **fhow).contiguous()), bits(pg.adjust_logits(x, **how)))
    for a, b in zip(pg.sample_actions(fx, noise=fnoise, **fhow), pg.sample_actions(x, noise=noise, **how)):
        assert torch.equal(a, b)
    for a, b in zip(pg.policy_loss(fx, fy, entropy=0.1, grad=far(x), **fhow), pg.policy_loss(x, y, entropy=0.1, **how)):
        assert torch.equal(a, b)
