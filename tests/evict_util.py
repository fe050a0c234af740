"""What the operators for trees of drafted tokens and for evictions compute, in 64 bits and by plain loops over the sequences of a paged_util.Cache."""
import math

import torch

from paged_util import BF16_STEP, F32_STEP


def tree_of(parents):
    """[n, n]: token i sees itself and what is above it; parents[i] < i, -1: it follows the text."""
    sees = torch.zeros(len(parents), len(parents), dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def packed(sees, words):
    """[n, words] int32 of bits [n, m]."""
    n, m = sees.shape
    x = torch.zeros(n, words * 32, dtype=torch.int64)
    x[:, :m] = sees[:, :words * 32]
    x = (x.view(n, words, 32) << torch.arange(32)).sum(-1)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def seen_in_tree(cache, b, sees, pos=None):
    """[n, keys]: which keys the new tokens of sequence b see; sees: [n, bits] of its tree."""
    n, kv = cache.q[b], cache.kv[b]
    p0 = kv - n if pos is None else pos[b]
    j = torch.arange(kv) - p0
    bits = torch.zeros(n, max(n, 1), dtype=torch.bool)
    bits[:, :min(n, sees.shape[1])] = sees[:n, :n]
    return (j < 0) | ((j < n) & bits[:, j.clamp(0, max(n - 1, 0))])


def attention_on(cache, q, scale, seen_of):
    """As paged_util.attention for any mask: seen_of(b) [n, keys].  The bounds are derived there."""
    found = []
    gq = q.shape[1] // cache.Hkv
    for b, n in enumerate(cache.q):
        if n == 0:
            continue
        lo, kv = cache.starts[b], cache.kv[b]
        K, ok = cache.rows("k", b)
        V, _ = cache.rows("v", b)
        seen = seen_of(b).to(q.device) & ok
        qs = q[0, :, lo:lo + n].double().view(cache.Hkv, gq, n, cache.D)
        any_row = seen.any(0) if n else ok
        K = torch.where(any_row[:, None, None], K, 0.0).permute(1, 0, 2)[:, None]
        V = V.permute(1, 0, 2)[:, None]
        x = (qs @ K.transpose(2, 3) * scale).masked_fill(~seen, -math.inf)
        size = (qs.abs() @ K.abs().transpose(2, 3) * scale).masked_fill(~seen, 0.0).amax(-1) if kv else torch.zeros_like(qs[..., 0])
        lse = torch.logsumexp(x, -1) if kv else torch.full_like(qs[..., 0], -math.inf)
        p = torch.exp(x - lse.clamp(min=-1e300).unsqueeze(-1))
        clean = torch.where(V.isfinite(), V, 0.0).expand(cache.Hkv, gq, kv, cache.D)
        out, mean = p @ clean, p @ clean.abs()
        for h, j, d in (~V.isfinite())[:, 0].nonzero().tolist():
            out[h, :, :, d] += torch.where(p[h, :, :, j] > 0, V[h, 0, j, d], 0.0)
        d_lse = (cache.D + 16) * F32_STEP * size + (kv + 16) * F32_STEP + 2.0 ** -20 + 2 * F32_STEP * lse.abs().nan_to_num(0, 0, 0)
        d_out = (BF16_STEP + 2 * d_lse.unsqueeze(-1)) * mean + 2.0 ** -126
        shape = (1, q.shape[1], n)
        found.append((slice(lo, lo + n), out.reshape(*shape, cache.D), lse.reshape(shape), d_out.reshape(*shape, cache.D), d_lse.reshape(shape)))
    return found


def causal_mask(cache, b, pos=None):
    n, kv = cache.q[b], cache.kv[b]
    p0 = kv - n if pos is None else pos[b]
    return torch.arange(kv) <= (p0 + torch.arange(n))[:, None]


def lse_of(cache, q, scale, seen_of):
    """[1, Hq, S] fp32, -inf for tokens without a sequence: what an attention on the same keys would have given."""
    lse = torch.full((1, q.shape[1], q.shape[2]), -math.inf, device=q.device)
    for rows, _, ref, _, _ in attention_on(cache, q, scale, seen_of):
        lse[:, :, rows] = ref.float()
    return lse


def weigh(cache, q, lse, scale, weights, fresh, seen_of, pos=None):
    """(weights after the call, bounds on what rounding may add), in 64 bits.

    Rounding, for a term exp(x - lse): the score to (D + 16) half steps of sum |q| |k| scale, x in units of 2 and what is taken off it each to a half step of themselves (four of
    them in all with the subtraction's), the exponential to 2 steps; sums of n terms to n half steps of their size; what is smaller than 2^-126 may be 0."""
    new, err = weights.double().clone(), torch.zeros_like(weights, dtype=torch.float64)
    gq = q.shape[1] // cache.Hkv
    for b, n in enumerate(cache.q):
        if n == 0 or cache.kv[b] == 0:
            continue
        lo, kv = cache.starts[b], cache.kv[b]
        K, ok = cache.rows("k", b)
        seen = (seen_of(b).to(q.device) & ok).expand(cache.Hkv, gq, n, kv)
        z = lse[0, :, lo:lo + n].double().view(cache.Hkv, gq, n, 1)
        seen = seen & z.isfinite()
        qs = q[0, :, lo:lo + n].double().view(cache.Hkv, gq, n, cache.D)
        clean = torch.where((qs.isfinite() | seen.any(-1, keepdim=True)), qs, 0.0)
        Kc = torch.where(seen.any(0).any(0).any(0)[:, None, None], K, 0.0).permute(1, 0, 2)[:, None]
        x = clean @ Kc.transpose(2, 3) * scale
        size = clean.abs() @ Kc.abs().transpose(2, 3) * scale
        z = torch.where(z.isfinite(), z, 0.0)
        e = torch.where(seen, torch.exp(x - z), 0.0)
        rel = F32_STEP * ((cache.D + 16) * size + 4 * (x.abs() + z.abs()) + 4 + gq * n + 16)
        added, off = e.sum((1, 2)), torch.where(seen, e * rel, 0.0).sum((1, 2)) + gq * n * 2.0 ** -126    # [Hkv, kv]
        p0 = kv - n if pos is None else pos[b]
        c = torch.arange(kv, device=q.device)
        own = (c >= p0) & (c < p0 + n)
        page = cache.table[b].long()[c // cache.page]
        touched = ok & (seen_of(b).to(q.device).any(0) | own)
        page, slot = page[touched], (c % cache.page)[touched]
        old = weights[page, :, slot].double()        # [keys, Hkv]
        if fresh:
            old = torch.where(own[touched][:, None], 0.0, old)
        new[page, :, slot] = old + added.T[touched]
        err[page, :, slot] = off.T[touched] + F32_STEP * (old + added.T[touched]).abs()
    return new, err


def select(cache, weights, first, last, most):
    """Lists by (sequence, head): the definition, by sorting."""
    lists = []
    for b, kv in enumerate(cache.kv):
        lists.append([])
        for h in range(weights.shape[1]):
            w = []
            for c in range(kv):
                page = int(cache.table[b, c // cache.page])
                w.append(None if not 0 <= page < cache.n_pages else float(weights[page, h, c % cache.page]))
            if kv <= most:
                lists[b].append(list(range(kv)))
                continue
            between = range(first, kv - last)
            rank = lambda c: (-2 if w[c] is None else 1 if math.isnan(w[c]) else 0, 0.0 if w[c] is None or math.isnan(w[c]) else w[c])   # noqa: E731,B023
            best = sorted(between, key=rank, reverse=True)[:most - first - last]      # (sorted keeps the order of equal ones, reversed or not)
            lists[b].append(sorted([*range(first), *best, *range(kv - last, kv)]))
    return lists


def keep(cache, tensors, keys, count, start):
    """The tensors (by name: [n_pages, Hkv, page_size, ...]) after the call: all reads in front of all writes."""
    old = {k: t.clone() for k, t in tensors.items()}
    new = {k: t.clone() for k, t in tensors.items()}
    table = cache.table.tolist()
    for b, kv in enumerate(cache.kv):
        for h in range(cache.Hkv):
            row = keys[b][min(h, len(keys[b]) - 1)]
            for i in range(max(0, min(count[b], len(row)))):
                c, to = row[i], (start[b] if start else 0) + i
                if not (0 <= to <= c < kv):
                    continue
                a, d = table[b][c // cache.page], table[b][to // cache.page]
                if not (0 <= a < cache.n_pages and 0 <= d < cache.n_pages):
                    continue
                for k in old:
                    new[k][d, h, to % cache.page] = old[k][a, h, c % cache.page]
    return new
