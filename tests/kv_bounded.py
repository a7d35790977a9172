"""Plain forms in 64 bits of the calls that keep a key/value cache bounded (sinks beside a window, accumulated
attention, the choice of what stays), one sequence and one head at a time, with what the bounds on errors need."""
import math

import torch


def visible(m, L, window=0, sinks=0, spans=None, tree=None):
    """see [m, L] of a sequence's m new tokens, their positions, and its slots' positions."""
    ctx, j = L - m, torch.arange(L)
    pos, kpos = torch.arange(ctx, L), torch.arange(L)
    if tree is not None:
        bits = torch.tensor([[(int(w) >> b) & 1 for b in range(m)] for w in tree], dtype=torch.bool).view(m, m)
        pos = ctx + bits.sum(1) - 1
        kpos = torch.cat([torch.arange(ctx), pos])
        see = torch.cat([torch.ones(m, ctx, dtype=torch.bool), bits], 1)
    elif spans is not None:
        see = (j >= spans[:, :1]) & (j < spans[:, 1:])
    else:
        see = j <= pos[:, None]
    if window:
        see = see & ((kpos > pos[:, None] - window) | (kpos < sinks))
    return see, pos, kpos


def scores64(q, key, h, see, pos, kpos, scale, softcap=0.0, slopes=None):
    """Scores of head h [m, L], -inf where masked, and the largest magnitude of each row's products."""
    m, H, _ = q.shape
    x = q[:, h].double() @ key[:, h // (H // key.shape[1])].double().T * scale
    big = x.masked_fill(~see, 0).abs().amax(-1) if key.shape[0] else torch.zeros(m).double()
    if softcap:
        x = softcap * torch.tanh(x / softcap)
    if slopes is not None:
        x = x - float(slopes[h]) * (pos[:, None] - kpos).abs()
    return x.masked_fill(~see, -math.inf), big


def attend64(q, key, val, scale, softcap=0.0, slopes=None, window=0, sinks=0, tree=None):
    """out, lse, and what kv_plain.near_attend's bounds need: sum of p|v| and the largest |product|."""
    m, H, D = q.shape
    L, K = key.shape[0], key.shape[1]
    see, pos, kpos = visible(m, L, window, sinks, None, tree)
    out, lse = torch.zeros(m, H, D, dtype=torch.float64), torch.zeros(m, H, dtype=torch.float64)
    spread, big = torch.zeros_like(out), torch.zeros_like(lse)
    for h in range(H):
        x, big[:, h] = scores64(q, key, h, see, pos, kpos, scale, softcap, slopes)
        lse[:, h] = torch.logsumexp(x, -1)
        p = torch.exp(x - torch.where(lse[:, h] == -math.inf, torch.zeros(()).double(), lse[:, h])[:, None])
        v = val[:, h // (H // K)].double()
        out[:, h], spread[:, h] = p @ v, p @ v.abs()
    return out, lse, spread, big


def weigh64(q, key, lse, scale, softcap=0.0, slopes=None, window=0, sinks=0, spans=None):
    """What each slot gets [kv_heads, L], and how far a kernel may be from it: a score, in fp32 from exact products, is
    within 2^-20 of its row's largest magnitude; a few units of exp2, of the scaled argument and of the distance's bias
    are 1e-5 in all (arguments that matter are below 32); a weight below 2^-126 may be 0."""
    m, H, _ = q.shape
    L, K = key.shape[0], key.shape[1]
    see, pos, kpos = visible(m, L, window, sinks, spans)
    got, off = torch.zeros(K, L, dtype=torch.float64), torch.zeros(K, L, dtype=torch.float64)
    for h in range(H):
        x, big = scores64(q, key, h, see, pos, kpos, scale, softcap, slopes)
        some = lse[:, h] > -math.inf
        p = torch.exp(x[some] - lse[some, h].double()[:, None])
        got[h // (H // K)] += p.sum(0)
        off[h // (H // K)] += ((1e-5 + 2.0 ** -20 * big[some])[:, None] * p).sum(0) + m * 2.0 ** -126
    return got, 1.01 * off


def near_weights(got, held, want, off, ctx, decay, what=""):
    """A row's weights [kv_heads, L] after the call: decay * held + want before the new tokens, want from there on; a few
    roundings of the whole sum (each below 2^-24 of it, in pieces that are added up apart) are 2^-20 of it."""
    old = torch.where(torch.arange(want.shape[1]) < ctx, held.double() * decay if decay else 0.0, 0.0)
    err = (got.double() - (old + want)).abs()
    bound = off + 2.0 ** -20 * (old.abs() + want)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    assert (err <= bound).all(), f"{what}: {float((err / bound).nan_to_num().max()):.3f} of the bound"


def select_plain(w, n, sinks, recent):
    """Slots of a row w [L] that stay, ascending, n of them: an order by numbers, of equals by slot."""
    L = len(w)
    a = min(sinks, n)
    b = min(recent, n - a)
    middle = [j for j in range(a, L - b)]
    middle.sort(key=lambda j: (1, 0.0) if math.isnan(w[j]) else (0, -w[j]))  # (sort keeps the order of equals)
    return sorted([*range(a), *middle[:n - a - b], *range(L - b, L)])
