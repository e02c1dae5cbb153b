"""Plain 64-bit reference of the choice of experts from logits, row by row (numpy only)."""
import numpy as np


def exp_of(a):
    """e^a, a <= 0; what is below e^-690 counts as zero (64 bits do not hold all digits of what is below 2^-1022, and 1 / (1 + e^-x) is zero from x = -709.8 on)"""
    return np.where(a < -690.0, 0.0, np.exp(np.maximum(a, -690.0)))


def choose(logits, top_k, sigmoid=False, bias=None, groups=1, top_groups=1, pair=False, renormalise=True, scale=1.0, gate_bits=8, valid=None):
    """logits float64 [n][E] -> (experts, gates, weights float64) [n][top_k]"""
    n, E = logits.shape
    l = np.where(np.isnan(logits), -np.inf, np.minimum(logits, 3.4028234663852886e38))
    experts, weights = np.full((n, top_k), -1, np.int32), np.zeros((n, top_k))
    for t in range(n):
        if valid is not None and not valid[t]:
            continue
        x = l[t]
        with np.errstate(over="ignore"):
            if sigmoid:
                y = exp_of(-np.abs(x))
                s = np.where(x >= 0, 1, y) / (1 + y)
            else:
                e = exp_of(x - x.max()) if x.max() > -np.inf else np.zeros(E)
                s = e / e.sum() if e.sum() > 0 else e
        c = x if bias is None else s + bias.astype(np.float64)
        able = (x > -np.inf) & ~np.isnan(c) & (c > -np.inf)
        value = s if bias is None and pair else c
        if top_groups < groups:
            size, rank = E // groups, []
            for g in range(groups):
                inside = [i for i in range(g * size, (g + 1) * size) if able[i]]
                inside.sort(key=lambda i: (-c[i], i))
                if inside:
                    rank.append((-sum(value[i] for i in inside[:2 if pair else 1]), g))
            kept = {g for _, g in sorted(rank)[:top_groups]}
            able &= np.array([i // size in kept for i in range(E)])
        chosen = sorted(np.nonzero(able)[0].tolist(), key=lambda i: (-c[i], i))[:top_k]
        w = s[chosen]
        if renormalise:
            total = w.sum()
            w = w / total if total > 0 else 0 * w
        experts[t, :len(chosen)], weights[t, :len(chosen)] = chosen, w * np.float64(np.float32(scale))
    return experts, np.rint(weights * 2.0 ** gate_bits).astype(np.int64), weights
