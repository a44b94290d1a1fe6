"""Plain references of the latent-cache calls, in 64 bits on the host, request by request."""
from __future__ import annotations

import math

import torch

from tests.draft_ref import tree_tolerances


def attend(q, k, v, limit, scale):
    """q [N, H, W], k [L, H or 1, W], v [L, H or 1, E], all float64; query i sees the keys j < limit[i].  Returns out
    [N, H, E], lse [N, H] and what their tolerances are made of (see tree_tolerances)."""
    n, h, _ = q.shape
    length = k.shape[0]
    k, v = k.expand(length, h, -1), v.expand(length, h, -1)
    seen = (torch.arange(length)[None, :] < torch.as_tensor(limit)[:, None])[:, None, :]          # [N, 1, L]
    x = torch.einsum("nhw,lhw->nhl", q, k) * scale
    x = torch.where(seen, x, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.where(seen, torch.exp(x - lse[..., None]), 0.0).nan_to_num(0.0)
    size = (torch.einsum("nhw,lhw->nhl", q.abs(), k.abs()) * scale * seen).amax(-1) if length else torch.zeros((n, h), dtype=torch.float64)
    return (torch.einsum("nhl,lhe->nhe", p, v), lse, torch.einsum("nhl,lhe->nhe", p, v.abs()), size,
            torch.as_tensor(limit).clamp(min=0).double())


def step_expected(q, rows, c_new, n, latent, scale, bf16):
    """One request of dsa_latent_step: q [N, H, W], cached rows [S, W], c_new [N, W], float64; n new tokens exist.  Returns
    out [N, H, R], lse [N, H] and their tolerances; tokens that do not exist: zeros, -inf, exactly."""
    big_n, h, w = q.shape
    out, lse = torch.zeros((big_n, h, latent), dtype=torch.float64), torch.full((big_n, h), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    if n > 0:
        k = torch.cat([rows, c_new[:n]])[:, None]
        out[:n], lse[:n], weight, size, count = attend(q[:n], k, k[..., :latent], [len(rows) + i + 1 for i in range(n)], scale)
        tol[:n], ltol[:n] = tree_tolerances(out[:n], lse[:n], weight, size, count, w, bf16)
    return out, lse, tol, ltol


def prompt_expected(q, k_nope, k_rope, v, causal, scale, bf16):
    """One request of dsa_latent_prompt: q [Lq, H, W], k_nope [Lk, H, .], k_rope [Lk, P], v [Lk, H, E], float64."""
    nq, h, w = q.shape
    nk = v.shape[0]
    k = torch.cat([k_nope, k_rope[:, None].expand(nk, h, -1)], -1)
    limit = [min(nk, max(0, i + 1 + nk - nq)) if causal else nk for i in range(nq)]
    o, l, weight, size, count = attend(q, k, v, limit, scale)
    tol, ltol = tree_tolerances(o, l, weight, size, count, w, bf16)
    none = (count == 0)[:, None]
    return o, l, torch.where(none[..., None], 0.0, tol), torch.where(none, 0.0, ltol)


def assert_near(got, want, tol, what):
    got = got.detach().cpu().double()
    same = (got == want) | ((got - want).abs() <= tol)
    if not bool(same.all()):
        off = torch.where(same, 0.0, (got - want).abs() / tol.clamp(min=1e-300)).nan_to_num(nan=math.inf)
        at = int(off.argmax())
        raise AssertionError("%s: %d of %d beyond the tolerance, worst at %d: %r, wanted %r +- %r" % (
            what, int((~same).sum()), same.numel(), at, got.reshape(-1)[at].item(), want.reshape(-1)[at].item(), tol.reshape(-1)[at].item()))


def map_expected(count, base, table, page, blocks, room, n):
    """dsa_map_tokens by hand: start, slot, position, request."""
    start, slot, position, request = [0], [], [], []
    for b, c in enumerate(count):
        for k in range(max(c, 0)):
            if len(slot) == n:
                break
            at = (base[b] if base is not None else 0) + k
            s = -1
            if 0 <= at < room:
                if table is None:
                    s = b * room + at
                elif at // page < len(table[b]) and 0 <= table[b][at // page] < blocks:
                    s = table[b][at // page] * page + at % page
            slot.append(s), position.append(at), request.append(b)
        start.append(len(slot))
    pad = [-1] * (n - len(slot))
    return start, slot + pad, position + pad, request + pad
