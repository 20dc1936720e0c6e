"""Float64 references of the choice of blocks and of attention behind a shared
prefix: plain loops over requests and query rows."""
import numpy as np

from oracle import step as S


def means(keys):
    """[n, 64, 576] -> [n, 576]."""
    return np.asarray(keys, np.float64).sum(1) / 64.0


def end_block(pos, window):
    """The first block that a row at `pos` may not choose for its window."""
    return max(pos + 1 - window, 0) // 64


def scores(q, keys, ok, n, qn, window, n_sink, scale):
    """q [Mq, H, 576], block means keys [NB, 576], ok [NB] (the table entry names a
    block) -> (scores [Mq, NB], the largest sum |q| |k| |scale| of a row)."""
    Mq, H, _ = q.shape
    out, mag = np.full((Mq, len(keys)), -np.inf), np.zeros(Mq)
    j = np.arange(len(keys))
    for i in range(min(qn, Mq)):
        may = ok & (64 * j >= n_sink) & (j < end_block(n - qn + i, window))
        if not may.any():
            continue
        out[i, may] = 0.0
        for h in range(H):
            s = keys[may] @ q[i, h] * scale
            with np.errstate(invalid="ignore"):
                w = np.exp(s - s.max())
            out[i, may] += w / w.sum()
        mag[i] = (np.abs(keys[may]) @ np.abs(q[i]).T).max() * abs(scale)
    return out, mag


def topk(x, K):
    """One row of scores -> K places, by a sort of (value, place) pairs."""
    def rank(j):
        v = x[j]
        return (0, 0.0, j) if v != v else (1, -float(v), j)
    best = sorted((j for j in range(len(x)) if not x[j] == -np.inf), key=rank)[:K]
    return sorted(best) + [-1] * (K - len(best))


def prefix_row(q, prefix, own, n_own, pos, scale):
    """Attention of rows q [h, 576] over all of `prefix` = (keys, values) and the
    tokens up to `pos` of the first n_own of `own` (see step.attend)."""
    keys = np.concatenate([prefix[0], own[0][:n_own]])
    values = np.concatenate([prefix[1], own[1][:n_own]])
    see = np.concatenate([np.ones(len(prefix[0]), bool), np.arange(n_own) <= pos])
    return S.attend(q, keys, values, see, scale)
