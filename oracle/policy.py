"""Plain checker for the learned-policy operators: numpy, 64 bits, one row at a time, written from the formulas.

  distill   loss = T^2 sum_k q_k (ln q_k - ln p_k), d loss / d x = T (p - q)
  balance   f_h = count_h / sum count, P = mean softmax over live rows, loss = n sum f P,
            d loss / d x = n / live * p (f - f . p)
  sample    whole-numbered weights floor(2^31 2^((x - m) c)), filters, draws in index order; sums are Python integers
"""
from __future__ import annotations

import math

import numpy as np


def _softmax(z):
    """(p, ln p) of one row; -inf entries have p = 0, a row of -inf has p = 0 everywhere."""
    z = np.asarray(z, dtype=np.float64)
    m = z.max() if z.size else -np.inf
    if m == -np.inf:
        return np.zeros_like(z), np.full_like(z, -np.inf)
    e = np.exp(z - m)
    return e / e.sum(), (z - m) - math.log(e.sum())


def distill(logits, hosts, teacher, temperature=1.0):
    """logits [R, n], hosts [R, k], teacher [R, k] (float64 in): loss [R], d loss / d logits [R, n]."""
    rows, n = logits.shape
    loss, grad = np.zeros(rows), np.zeros((rows, n))
    for r in range(rows):
        p, log_p = _softmax(logits[r] / temperature)
        entries = [(int(h), float(t)) for h, t in zip(hosts[r], teacher[r])
                   if 0 <= h < n and t > -np.inf and logits[r, h] != -np.inf]
        if not entries:
            continue
        q, log_q = _softmax(np.array([t for _, t in entries]) / temperature)
        for (h, _), qk, lk in zip(entries, q, log_q):
            if qk > 0:
                loss[r] += temperature ** 2 * qk * (lk - log_p[h])
            grad[r, h] -= temperature * qk
        grad[r] += temperature * p
    return loss, grad


def balance(logits, hosts):
    """One group: logits [B, n], hosts [B, k]: loss, counts [n], shares [n], d loss / d logits [B, n]."""
    rows, n = logits.shape
    counts, live = np.zeros(n, dtype=np.int64), np.zeros(rows, dtype=bool)
    for r in range(rows):
        for h in hosts[r]:
            if 0 <= h < n:
                counts[h] += 1
                live[r] = True
    shares, grad = np.zeros(n), np.zeros((rows, n))
    if not live.any():
        return 0.0, counts, shares, grad
    f = counts / counts.sum()
    for r in np.flatnonzero(live):
        p, _ = _softmax(logits[r])
        shares += p / live.sum()
        grad[r] = n / live.sum() * p * (f - f @ p)
    return n * float(f @ shares), counts, shares, grad


ONE = 2 ** 31
STEPS = 2 ** 24


def sample_weights(x, temperature):
    """Whole-numbered weights of one row of 32-bit logits. The steps are rounded to 32 bits as defined; the power is
    taken in 64 bits, so the weights are the library's wherever the power is exact (whole exponents)."""
    x = np.asarray(x, dtype=np.float32)
    x = np.where(np.isnan(x), np.float32(-np.inf), np.minimum(x, np.finfo(np.float32).max)).astype(np.float32)
    m = x.max()
    if m == -np.inf:
        return x, [0] * x.size
    c = np.float32(1.4426950408889634) / np.float32(temperature)
    with np.errstate(invalid="ignore", over="ignore"):
        y = ((x - m).astype(np.float32) * c).astype(np.float32).astype(np.float64)
    return x, [int(math.floor(math.ldexp(2.0 ** v, 31))) if v > -64 else 0 for v in y]


def sample_kept(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weights of one row after the filters."""
    n = len(x)
    greedy = not temperature > 2.0 ** -20
    x, w = sample_weights(x, 1.0 if greedy else temperature)
    order = sorted(range(n), key=lambda h: (-x[h], h))
    kept = order[:1] if greedy else (order[:top_k] if top_k > 0 else order)
    if not greedy and top_p < 1.0:
        share = int(math.floor(max(float(np.float32(top_p)), 0.0) * STEPS))
        limit = max(1, sum(w[h] for h in kept) * share // STEPS)
        before, inside = 0, []
        for h in kept:
            if before < limit:
                inside.append(h)
            before += w[h]
        kept = inside
    if min_p > 0:
        least = int(math.floor(min(float(np.float32(min_p)), 1.0) * ONE))
        kept = [h for h in kept if w[h] >= least]
    out = [0] * n
    for h in kept:
        out[h] = w[h]
    return out


def draw(weights, uniforms):
    """Distinct hosts drawn from whole-numbered weights: hosts (-1 padded), how many."""
    w, hosts = list(weights), []
    for u in uniforms:
        left = sum(w)
        if left == 0:
            hosts.append(-1)
            continue
        u = 0.0 if math.isnan(u) else min(max(float(u), 0.0), 1.0)
        t = left * min(int(math.floor(u * STEPS)), STEPS - 1) // STEPS
        run = 0
        for h, v in enumerate(w):
            run += v
            if run > t:
                break
        hosts.append(h)
        w[h] = 0
    return hosts, sum(h >= 0 for h in hosts)


def sample(logits, uniforms, temperature=None, top_k=None, top_p=None, min_p=None):
    """logits [R, n] 32-bit, uniforms [R, draws], one setting per row or None: hosts [R, draws], found [R]."""
    hosts, found = [], []
    for r in range(logits.shape[0]):
        kept = sample_kept(logits[r], 1.0 if temperature is None else temperature[r], 0 if top_k is None else int(top_k[r]),
                           1.0 if top_p is None else top_p[r], 0.0 if min_p is None else min_p[r])
        h, f = draw(kept, uniforms[r])
        hosts.append(h)
        found.append(f)
    return np.array(hosts, dtype=np.int32).reshape(logits.shape[0], -1), np.array(found, dtype=np.int32)
