"""Plain 64-bit form of rotary positions (include/pgxrotary.h), on the CPU, pair by pair."""
import torch


def turned(x, positions, frequencies, interleaved=False, magnitude=1.0, inverse=False):
    """x [..., heads, head_dim], positions [...]; float64"""
    x, f = x.detach().cpu().double() if not x.requires_grad else x, frequencies.cpu().double()
    R = 2 * f.numel()
    angle = positions.cpu().double()[..., None, None] * f
    c, s = torch.cos(angle) * magnitude, torch.sin(angle) * (-magnitude if inverse else magnitude)
    out = [None] * x.shape[-1]
    for j in range(R // 2):
        u, w = (2 * j, 2 * j + 1) if interleaved else (j, j + R // 2)
        out[u] = x[..., u] * c[..., j] - x[..., w] * s[..., j]
        out[w] = x[..., w] * c[..., j] + x[..., u] * s[..., j]
    for e in range(R, x.shape[-1]):
        out[e] = x[..., e]
    return torch.stack(out, -1)
