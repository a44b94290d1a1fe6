"""Plain references of the drafted-token calls, in 64 bits on the host, request by request."""
from __future__ import annotations

import math

import numpy as np
import torch

BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2      # a rounding is off by at most this, relative to the value
F32_HALF_STEP = torch.finfo(torch.float32).eps / 2


def lines_of(parent, n):
    """The nodes of every node's line, roots first."""
    lines = []
    for i in range(n):
        p = int(parent[i])
        lines.append((lines[p] if 0 <= p < i else []) + [i])
    return lines


def tree_reference(q, rows_k, rows_v, k_new, v_new, parent, seq, prompt, n, scale, window=0, sinks=0):
    """One request: q [N, Hq, D], cached rows [S, Hkv, D], new rows [N, Hkv, D], all float64; n nodes exist.
    Returns out [N, Hq, D], lse [N, Hq] and what their tolerances are made of: sum p |v|, the largest
    sum |q k| scale, the number of tokens seen."""
    N, hq, d = q.shape
    g = hq // k_new.shape[1]
    out, lse = torch.zeros_like(q), torch.full((N, hq), -math.inf, dtype=torch.float64)
    weight, size, count = torch.zeros_like(q), torch.zeros((N, hq), dtype=torch.float64), torch.zeros((N,))
    prompt = min(prompt, seq)
    lines = lines_of(parent, n)
    for i in range(n):
        at = seq + len(lines[i]) - 1
        cached = [s for s in range(seq) if not window or s < prompt + sinks or at - s < window]
        own = [j for e, j in enumerate(lines[i]) if not window or seq + e < prompt + sinks or at - (seq + e) < window]
        count[i] = len(cached) + len(own)
        k = torch.cat([rows_k[cached], k_new[own]])
        v = torch.cat([rows_v[cached], v_new[own]])
        for h in range(hq):
            kh, vh = k[:, h // g], v[:, h // g]
            x = kh @ q[i, h] * scale
            p = torch.softmax(x, 0)
            lse[i, h] = torch.logsumexp(x, 0)
            out[i, h] = p @ vh
            weight[i, h] = p @ vh.abs()
            size[i, h] = (kh.abs() @ q[i, h].abs()).max() * scale
    return out, lse, weight, size, count


def tree_tolerances(out, lse, weight, size, count, d, bf16):
    """Bounds of what the kernel may be off by.  A logit is a sum of d products in fp32 (d + 4 roundings, the scale
    among them) and one rounding of x log2 e; the exponential adds 2^-21 (2 units of ex2.approx, and the
    subtraction of the maximum); a weight is off by twice a logit's error, relative, and sums of `count` terms by as
    many roundings.  bf16: every weight is rounded to bf16 before the product, and the result once."""
    dx = (d + 4) * F32_HALF_STEP * size + 2.0 ** -21 + 4 * F32_HALF_STEP * size
    n = count[:, None].double() + 8
    rel = 2 * dx + 2 * n * F32_HALF_STEP
    tol = (rel[..., None] + (BF16_HALF_STEP if bf16 else 0.0)) * weight * (1 + 2.0 ** -7)
    tol = tol + (BF16_HALF_STEP if bf16 else F32_HALF_STEP) * (out.abs() + tol)
    ltol = dx + n * F32_HALF_STEP + 4 * F32_HALF_STEP * lse.abs().nan_to_num(posinf=0.0)
    return tol + 1e-30, ltol


def verify_reference(tokens, p, q, u, parent, n, mode):
    """One request: p, q float64 [N, V] (q None: points), u [N]; the walk of dsa_verify_tree."""
    v_all = p.shape[1]
    if n == 0:
        return [], -1
    path, cur = [0], 0
    left, weight = p[0].copy(), 1.0
    for i in range(1, n):
        up = parent[i] if 0 <= parent[i] < i else -1
        if up != cur:
            continue
        x = int(tokens[i])
        if mode == "greedy":
            stands = x == int(np.argmax(p[cur]))
        else:
            if not 0 <= x < v_all:
                continue
            qx = q[cur, x] if mode == "sample" else 1.0
            stands = float(u[i]) * weight * qx < left[x]
            if not stands:
                if mode == "sample":
                    left = np.maximum(left - weight * q[cur], 0.0)
                    weight = math.fsum(left)
                else:
                    weight -= left[x]
                    left[x] = 0.0
        if stands:
            path.append(i)
            cur, left, weight = i, p[i].copy(), 1.0
    if mode == "greedy":
        return path, int(np.argmax(p[cur]))
    if not math.fsum(left) > 0:
        left = p[cur].copy()
    total = math.fsum(left)
    if not total > 0:
        return path, -1
    return path, int(np.argmax(np.cumsum(left) > float(u[0]) * total))


class Pool:
    """The page calls, entry by entry."""

    def __init__(self, refs, table, page):
        self.refs, self.table, self.page = [int(x) for x in refs], [[int(x) for x in r] for r in table], page

    def free(self):
        return [i for i, r in enumerate(self.refs) if r == 0]

    def reserve(self, lens, extra):
        status, stopped = [], False
        for row, length in zip(self.table, lens):
            need = 0 if length < 0 else -(-(length + extra) // self.page)
            lacks = [e for e in range(min(need, len(row))) if row[e] < 0]
            if need > len(row):
                status.append(len(lacks) + need - len(row))
                continue
            if not lacks:
                status.append(0)
                continue
            free = self.free()
            stopped = stopped or len(lacks) > len(free)
            if stopped:
                status.append(len(lacks))
                continue
            for e, page in zip(lacks, free):
                row[e] = page
                self.refs[page] = 1
            status.append(0)
        return status

    def release(self, keep):
        for b, row in enumerate(self.table):
            k = 0 if keep is None else keep[b]
            if k < 0:
                continue
            for e in range(-(-k // self.page), len(row)):
                if row[e] >= 0:
                    self.refs[row[e]] -= 1
                    row[e] = -1

    def fork(self, src, dst, lens, prompts, caches):
        """caches: numpy arrays [layers, pages, page, ...] that are changed like the table."""
        rows = len(self.table)
        status, free = [], self.free()
        for i, (s, d) in enumerate(zip(src, dst)):
            if not (0 <= s < rows and 0 <= d < rows) or d in src or d in dst[:i]:
                status.append(2)
                continue
            full, part = divmod(lens[s], self.page)
            if part and not free:
                status.append(1)
                continue
            row = self.table[s][:full]
            for page in row:
                self.refs[page] += 1
            if part:
                fresh = free.pop(0)
                self.refs[fresh] = 1
                for c in caches:
                    c[:, fresh, :part] = c[:, self.table[s][full], :part]
                row = row + [fresh]
            self.table[d] = row + [-1] * (len(self.table[d]) - len(row))
            lens[d], prompts[d] = lens[s], prompts[s]
            status.append(0)
        return status
