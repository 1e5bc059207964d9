"""Plain 64-bit forms of the decoder's attention operators, for their tests."""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half a step, relative


def to_bf16(x, up):
    """x (float64) to the nearest bfloat16 that is not below (up) or not above it."""
    b = x.float().bfloat16()
    toward = torch.full_like(b, math.inf if up else -math.inf)
    wrong = b.double() < x if up else b.double() > x
    return torch.where(wrong, torch.nextafter(b, toward), b).double()


def held(x):
    """(codes, lowest value, step, tie): the cache's row quantizer; tie marks codes within 2^-18 of halfway between two."""
    x = x.double()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    low = to_bf16(lo, False)
    step = to_bf16((hi - low) / torch.full_like(low, 15.0), True)
    step = torch.where(hi == low, torch.zeros_like(step), step.clamp(min=2.0 ** -126))
    t = torch.where(step > 0, (x - low) / torch.where(step > 0, step, torch.ones_like(step)), torch.zeros_like(x))
    frac = t - t.floor()
    return torch.round(t), low, step, ((frac - 0.5).abs() < 2.0 ** -18) & (frac != 0.5)


def rotated(x, weight, positions, inv_freq, interleaved, eps):
    """(result, size): norm and rotation in float64, and the largest each output's two parts are."""
    x = x.double()
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    r = 0 if inv_freq is None else 2 * inv_freq.numel()
    if r == 0:
        return x, x.abs()
    # whole turns leave exactly, in integers: angle / 2 pi as a fraction of 2^-60 a turn
    f = [round(float(v) / (2 * math.pi) * 2 ** 60) for v in inv_freq.double().tolist()]
    turn = torch.tensor([[int(p) * v % 2 ** 60 / 2 ** 60 for v in f] for p in positions.tolist()], dtype=torch.float64, device=x.device)
    c, s = torch.cos(2 * math.pi * turn)[:, None], torch.sin(2 * math.pi * turn)[:, None]
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    y, size = x.clone(), x.abs()
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = x[..., i].abs() + x[..., j].abs()
    return y, size


def attended(q, k, v, see, scale):
    """(o, lse, sum_t p |v|, sum |q| per row) of q [n, heads, d] over k, v [m, kv, d] in float64; query i sees the first see[i] keys."""
    n, heads, d = q.shape
    g = heads // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    o = torch.zeros_like(q)
    mass = torch.zeros_like(q)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device=q.device)
    for i in range(n):
        m = max(0, min(int(see[i]), k.shape[0]))
        if m == 0:
            continue
        s = torch.einsum("hd,mhd->hm", q[i], k[:m]) * scale
        lse[i] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[i][:, None])
        o[i] = torch.einsum("hm,mhd->hd", p, v[:m])
        mass[i] = torch.einsum("hm,mhd->hd", p, v[:m].abs())
    return o, lse, mass, q.abs().sum(-1)


def close(got, want, tol):
    """got within tol of want; the same infinities, no NaN."""
    got = got.double()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    bad = ~((got - want).abs() <= tol) & ~inf
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values off, by up to {((got - want).abs() / tol)[bad].max().item():.3g} times their bound"
