"""The definition of fef_draw_logits for one row in numpy, 64 bits."""
import numpy as np


def law(x, tau=1.0, greedy=False):
    """float32 logits times 1 / tau in float32, and which tokens exist (None: the row has no law)."""
    with np.errstate(over="ignore", invalid="ignore"):
        y = x.astype(np.float32) * (np.float32(1) if greedy else np.float32(1) / np.float32(tau))
    if not (y < np.inf).all():
        return None
    ids = np.nonzero(y >= np.float32(-2e38))[0]
    return (y, ids) if len(ids) else None


def truncate(x, u, tau=1.0, k=0, p=1.0, min_p=0.0, greedy=False):
    """(truncated logits, log-sum-exp, kept, token, confidence); `x` a row of logits as float32 holds them."""
    V = len(x)
    none = (np.full(V, -np.inf, np.float32), -np.inf, 0, -1, 0.0)
    got = law(x, tau, greedy)
    if got is None:
        return none
    y, ids = got
    order = ids[np.lexsort((ids, -y[ids].astype(np.float64)))]
    w = np.exp(y[order].astype(np.float64) - float(y[order[0]]))
    n = len(order)
    if greedy:
        k = 1
    length = min(n, k) if k > 0 else n
    kept = length
    if p < 1:
        before = np.concatenate(([0.0], np.cumsum(w[:length])[:-1]))
        target = float(p) * w[:length].sum()
        assert not ((before != target) & (np.abs(before - target) < 1e-11 * target)).any(), "an input too near a border to be compared"
        kept = min(kept, max(1, int((before < target).sum())))
    if min_p > 0:
        kept = min(kept, max(1, int((w >= float(min_p)).sum())))
    chosen = np.sort(order[:kept])
    w_id = np.exp(y[chosen].astype(np.float64) - float(y[order[0]]))
    total = w_id.sum()
    sums = np.cumsum(w_id)
    target = min(max(float(u), 0.0), 1.0) * total
    token = chosen[np.nonzero((sums >= target * (1 - 1e-12)) & (w_id > 2.0 ** -60))[0][0]]
    out = np.full(V, -np.inf, np.float32)
    out[chosen] = y[chosen]
    return out, float(y[order[0]]) + np.log(total), kept, int(token), float(w_id[chosen == token][0] / total)
