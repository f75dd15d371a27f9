"""The operators beside the products in 64 bits, by loops over their definitions, with the bounds their results are held to."""
import math

import numpy as np

H = 2.0 ** -11            # half a step of FP16, relative
F = 2.0 ** -24            # half a step of FP32, relative
TINY = 2.0 ** -25         # half a step of FP16 below its normal range


def kv_slots(lens, counts, table, page, blocks, free, head, n_slots):
    table, slots, cu, new = table.copy(), np.full(n_slots, -1, np.int32), [0], []
    left = max(len(free) - head, 0) if head >= 0 else 0
    asked = taken = 0
    for r, (n, c) in enumerate(zip(lens.tolist(), counts.tolist())):
        begin, end = cu[-1], cu[-1] + max(c, 0)
        cu.append(end)
        if n < 0 or c < 0 or n + c > table.shape[1] * page or end > n_slots:
            new.append(n)
            continue
        have, all_ = -(-n // page), -(-(n + c) // page)
        need, first = all_ - have, asked
        asked += need
        if need and asked > left:
            new.append(n)
            continue
        for p in range(have, all_):
            table[r, p] = free[head + first + p - have]
        taken = max(taken, asked if need else 0)
        new.append(n + c)
        for j in range(c):
            b = int(table[r, (n + j) // page])
            slots[begin + j] = b * page + (n + j) % page if 0 <= b < blocks else -1
    return slots, np.minimum(cu, n_slots).astype(np.int32), np.array(new, np.int32), np.array([head + taken], np.int32), table


def tree_attention(q, k, v, k_cache, v_cache, table, lens, cu, mask, scale):
    """(result, bound), NaN in rows nobody owns.  q, k, v: (N, heads, dim) float64; caches (blocks, heads, page, dim)."""
    n, heads, dim = q.shape
    page, group = k_cache.shape[2], heads // k.shape[1]
    out, bound = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for r, length in enumerate(lens.tolist()):
        pages = table[r, :-(-length // page)]
        for h in range(heads):
            kh = h // group
            old_k, old_v = (c[pages, kh].reshape(-1, dim)[:length] for c in (k_cache, v_cache))
            for i in range(cu[r], cu[r + 1]):
                see = [cu[r] + j for j in range(cu[r + 1] - cu[r]) if int(mask[i]) >> j & 1]
                keys, values = np.concatenate([old_k, k[see, kh]]), np.concatenate([old_v, v[see, kh]])
                if not len(keys):
                    out[i, h], bound[i, h] = 0, 0
                    continue
                s = keys @ q[i, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[i, h] = w @ values
                # a weight: half a step of FP16, and what the sum of `dim` products in FP32 (rounded once more by the scale,
                # by the difference to the maximum and by exp) does to its exponent; numerator and denominator have it each.
                # The weighted sum: a step of FP32 an addition.
                wrong = (dim + 6) * F * (np.abs(keys) @ np.abs(q[i, h]) * abs(scale)).max() + 8 * F
                size = w @ np.abs(values)
                bound[i, h] = H * np.abs(out[i, h]) + (H + 2 * wrong + (len(keys) + 64) * F) * (size + np.abs(out[i, h])) + TINY
    return out, bound


def lora(X, A, B, index, base, scale):
    """(result, bound); NaN where the index is past the adapters."""
    out = base.copy()
    bound = (H + F) * np.abs(out) + TINY
    for m, a in enumerate(index.tolist()):
        if a >= len(A):
            out[m] = np.nan
        elif a >= 0:
            h, size = A[a] @ X[m], np.abs(A[a]) @ np.abs(X[m])
            out[m] += scale[a] * (B[a] @ h)
            # FP32 sums of cols and of rank products; h is passed on in 22 bits; three roundings to FP32 around them
            bound[m] = H * np.abs(out[m]) + (len(X[m]) + A.shape[1] + 16) * F * abs(scale[a]) * (np.abs(B[a]) @ size) + 3 * F * np.abs(out[m]) + F * np.abs(base[m]) + TINY
    return out, bound


def rules(logits, cu, half, history=None, history_len=None, prompt_len=None, draft=None, mask=None, repetition=None, frequency=None, presence=None,
          bias_ids=None, bias=None, allowed=None, allowed_row=None):
    """(result, bound), rows nobody owns as they are with a bound of zero."""
    out, bound = logits.astype(np.float64), np.zeros(logits.shape)
    vocab = logits.shape[1]
    for r in range(len(cu) - 1):
        for i in range(cu[r], cu[r + 1]):
            told, count, add = set(), {}, {}
            if history is not None:
                n = min(max(int(history_len[r]), 0), history.shape[1])
                p = 0 if prompt_len is None else min(max(int(prompt_len[r]), 0), n)
                told = set(history[r, :p].tolist())
                for t in history[r, p:n].tolist():
                    count[t] = count.get(t, 0) + 1
            if draft is not None:
                for j in range(min(cu[r + 1] - cu[r], 64)):
                    if int(mask[i]) >> j & 1:
                        t = int(draft[cu[r] + j])
                        count[t] = count.get(t, 0) + 1
            if bias_ids is not None:
                add = dict(zip(bias_ids[r].tolist(), bias[r].astype(np.float64).tolist()))
            x = out[i]
            size = np.abs(x)
            for t in told | set(count):
                if not 0 <= t < vocab:
                    continue
                if repetition is not None:
                    x[t] = x[t] / float(repetition[r]) if x[t] > 0 else x[t] * float(repetition[r])
                    size[t] = max(size[t], abs(x[t]))
                if count.get(t):
                    f = (0 if frequency is None else float(frequency[r])) * count[t]
                    p = 0 if presence is None else float(presence[r])
                    x[t] = x[t] - f - p
                    size[t] += abs(f) + abs(p)
            for t, a in add.items():
                if 0 <= t < vocab:
                    x[t] += a
                    size[t] += abs(a)
            # up to six roundings to FP32, of numbers no larger than `size`; one to FP16
            bound[i] = 6 * F * size + ((H * np.abs(x) + TINY) if half else 0)
            if allowed is not None and int(allowed_row[i]) >= 0:
                if allowed_row[i] >= len(allowed):
                    x[:] = np.nan
                    continue
                t = np.arange(vocab)
                x[(allowed[allowed_row[i]].view(np.uint32)[t // 32] >> (t % 32) & 1) == 0] = -math.inf
    return out, bound


def close(got, want, bound, what=""):
    got = np.asarray(got, dtype=np.float64)
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True), f"{what}: infinities or NaN differ"
    err = np.abs(got[~odd] - want[~odd])
    bad = ~(err <= bound[~odd])
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} out of bounds, worst {float(np.nanmax(err / np.maximum(bound[~odd], 1e-300)))} times the bound"


def trees(rng, counts, total=None):
    """Masks of random trees, one a request: a token sees itself and its ancestors."""
    words = []
    for c in counts:
        seen = []
        for j in range(c):
            parent = int(rng.integers(-1, j)) if j else -1
            seen.append((seen[parent] if parent >= 0 else 0) | 1 << j)
        words += seen
    out = np.zeros(len(words) if total is None else total, dtype=np.uint64)
    out[:len(words)] = words
    return out
