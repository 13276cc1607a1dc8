"""The operators around the quantised layer in 64 bits, with the bound of each
output's error (test infrastructure).

Every value travels as a pair (y, err): err bounds |computed - y| for a kernel
that rounds as the interface says.  With u = 2^-24 (half a step of fp32):

* the quantised product: its int32 sum is exact; its conversion to float and
  the two scalings round once each: 3 u of its magnitude.
* a compensation u L2: sums of n terms in any order are off by at most n u of
  the sum of magnitudes; with bf16 factors each row enters as hi + lo, two bf16
  roundings of 2^-8 each in turn: 2^-16 of each term, once for the smoothed row
  and once for u.
* bias, product and residual: u of the result each.
* activations: |act'| <= 1.13 for the three of them, and 16 u of the result for
  exp, erfc and the quotient (a few units in the last place each), plus, for an
  exponent of size a, a u of the result.
* the output's rounding: eps / 2 of the result.

32-bit results below 2^-126 may be flushed: 1e-37 is added.
"""
import math

import torch

U = 2.0 ** -24


def smoothed(x, mod, inv):
    """Smoothed rows, codes and steps as the rounding contract defines them, from
    32-bit products and quotients formed in 64 bits and rounded once."""
    xs = (x.double() * inv.double()[mod.long()]).float()
    amax = xs.abs().amax(1).double()
    safe = torch.where(amax > 0, amax, torch.ones_like(amax))
    dx = (amax / 127.0).float()
    q = torch.round((xs.double() * (127.0 / safe).float().double()[:, None]).float())
    return xs.double(), q.clamp(-127, 127).double(), dx.double()


def layer(x, mod, inv, codes, scale, l_down, r_up, bias=None):
    """(z, err) of the layer and its bias, before the activation.  codes [N][K]
    as integers, factors [M-1][r][K] and [M-1][N][r] or None."""
    xs, q, dx = smoothed(x, mod, inv)
    z = (q @ codes.double().T) * dx[:, None] * scale.double()
    err = 3 * U * z.abs()
    if l_down is not None:
        split = 2.0 ** -16 if l_down.dtype == torch.bfloat16 else 0.0
        K, r = xs.shape[1], l_down.shape[1]
        ld, ru = l_down.double(), r_up.double()
        for m in range(1, inv.shape[0]):
            i = torch.nonzero((mod == m).cpu()).flatten().to(x.device)
            if not i.numel():
                continue
            u, ua = xs[i] @ ld[m - 1].T, xs[i].abs() @ ld[m - 1].abs().T
            ue = ua * (split + (K + 2) * U)
            c = u @ ru[m - 1].T
            ca = (u.abs() + ue) @ ru[m - 1].abs().T
            z[i] += c
            err[i] += ue @ ru[m - 1].abs().T + ca * (split + (r + 2) * U) + U * (z[i].abs() + ca) * (r + 1)
    if bias is not None:
        z = z + bias.double()
        err = err + U * z.abs()
    return z, err


def act(z, err, kind):
    if kind == "none":
        return z, err
    if kind == "silu":
        a, h = z, z * torch.sigmoid(z)
    elif kind == "gelu":
        a, h = z * z / 2, 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    else:
        a = math.sqrt(8.0 / math.pi) * (z + 0.044715 * z ** 3)
        h = z * torch.sigmoid(a)
    return h, 1.13 * err + U * (16 + 4 * a.abs()) * h.abs()


def finish(z, err, kind, gated, residual, dtype):
    """(y, err) past the activation, with the output's rounding."""
    if gated:
        h, e = act(z[:, 0::2], err[:, 0::2], kind)
        up, ue = z[:, 1::2], err[:, 1::2]
        y = h * up
        e = e * (up.abs() + ue) + h.abs() * ue + U * y.abs()
    else:
        y, e = act(z, err, kind)
    if residual is not None:
        y = y + residual.double()
        e = e + U * y.abs()
    return y, e + torch.finfo(dtype).eps / 2 * (y.abs() + e) + 1e-37


def assert_close(got, want, err):
    got = got.double()
    bad = ~((got - want).abs() <= err)
    if bad.any():
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{int(bad.sum())} of {bad.numel()} off; first at {i}: got {got[i].item()!r}, "
                             f"want {want[i].item()!r} +- {err[i].item():.3e}")


def route(logits, k, renorm):
    """experts, weights, offsets, rows, slots by plain loops (lists)."""
    T, E = logits.shape
    experts, weights = [], []
    for row in logits.double().tolist():
        live = [e for e in range(E) if row[e] > -math.inf]             # (NaN compares false)
        pick = sorted(live, key=lambda e: (-row[e], e))[:k]
        top = row[pick[0]] if pick else 0.0
        p = {e: 1.0 if row[e] == top else math.exp(row[e] - top) for e in live}
        total = sum(p[e] for e in (pick if renorm else live))
        experts.append(pick + [-1] * (k - len(pick)))
        weights.append([p[e] / total for e in pick] + [0.0] * (k - len(pick)))
    offsets, rows, slots = [0], [], [[-1] * k for _ in range(T)]
    for e in range(E):
        for t in range(T):
            if e in experts[t]:
                slots[t][experts[t].index(e)] = len(rows)
                rows.append(t)
        offsets.append(len(rows))
    rows += [-1] * (T * k - len(rows))
    return experts, weights, offsets, rows, slots
