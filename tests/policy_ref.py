"""Plain 64-bit forms of the policy operators (include/pgxpolicy.h), on the CPU, row by row where that is plainer."""
import torch

NEG = float("-inf")


def counts_of(record, begin, end, rows, actions):
    c = torch.zeros(rows, actions, dtype=torch.float64)
    for b in range(rows):
        lo = 0 if begin is None else max(int(begin[b]), 0)
        hi = record.shape[1] if end is None else min(int(end[b]), record.shape[1])
        for t in range(lo, hi):
            a = int(record[b, t])
            if 0 <= a < actions:
                c[b, a] += 1
    return c


def adjusted(logits, mask=None, bias=None, record=None, begin=None, end=None, repetition=1.0, frequency=0.0, presence=0.0, temperature=None, dtype=torch.float64):
    """(z, possible); every operation in `dtype`, so with float32 it is the header's definition to the bit"""
    z = logits.detach().cpu().to(dtype) if not logits.requires_grad else logits
    rows, actions = z.shape
    one = lambda v: torch.tensor(v, dtype=torch.float32).to(dtype)  # noqa: E731   parameters are 32-bit numbers
    if record is not None:
        c = counts_of(record.cpu(), begin, end, rows, actions).to(dtype)
        z = torch.where(c > 0, torch.where(z > 0, z / one(repetition), z * one(repetition)), z)
        z = z - one(frequency) * c
        z = torch.where(c > 0, z - one(presence), z)
    if bias is not None:
        z = z + bias.cpu().to(dtype)
    if temperature is not None:
        t = temperature.cpu().to(dtype) if isinstance(temperature, torch.Tensor) else torch.full((rows,), float(temperature)).to(dtype)
        z = z / torch.where(t > 0, t, torch.ones_like(t))[:, None]
    if mask is not None:
        z = torch.where(mask.cpu()[:, :actions] != 0, z, torch.full_like(z, NEG))
    return z, z > NEG


def log_probabilities(z, possible):
    out = torch.full_like(z, NEG)
    for b in range(z.shape[0]):
        if possible[b].any():
            out[b, possible[b]] = torch.log_softmax(z[b, possible[b]], 0)
    return out


def sampled(z32, possible, noise=None, temperature=None):
    """the header's draw, from z in 32 bits"""
    out = []
    for b in range(z32.shape[0]):
        t = 1.0 if temperature is None else float(temperature[b]) if isinstance(temperature, torch.Tensor) else temperature
        score = z32[b] if noise is None or not t > 0 else z32[b] + noise[b].cpu()
        score = torch.where(torch.isnan(score), torch.full_like(score, NEG), score)
        where = possible[b].nonzero()[:, 0]
        out.append(int(where[(score[where] == score[where].max()).nonzero()[0, 0]]) if len(where) else -1)
    return torch.tensor(out, dtype=torch.int32)


def loss(logits, target, weight=None, entropy=0.0, **how):
    """(loss [rows], entropies [rows], gradient of the losses' sum), by automatic differentiation in 64 bits"""
    x = logits.detach().cpu().double().requires_grad_()
    z, possible = adjusted(x, **how)
    rows = x.shape[0]
    losses, entropies = [], []
    for b in range(rows):
        live = possible[b].nonzero()[:, 0]
        if not len(live):
            losses.append(x[b].sum() * 0)
            entropies.append(x[b].sum() * 0)
            continue
        logp = torch.log_softmax(z[b, live], 0)
        if target.dtype == torch.int32:
            y = (live == int(target[b])).double()
        else:
            y = target[b].cpu().double()[live]
        h = -(logp.exp() * logp).sum()
        w = 1.0 if weight is None else float(weight[b])
        losses.append(-w * (y * logp).sum() - float(torch.tensor(entropy, dtype=torch.float32)) * h)
        entropies.append(h)
    losses, entropies = torch.stack(losses), torch.stack(entropies)
    losses.sum().backward()
    return losses.detach(), entropies.detach(), x.grad
