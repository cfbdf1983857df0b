"""fp64 restatement (numpy) of the loss that trains classes from a teacher's top logits, and of its
gradient.  Shares no code with the library."""
import numpy as np


def _log_softmax(v):
    with np.errstate(invalid="ignore", divide="ignore"):
        v = v - v.max()
        return v - np.log(np.exp(v).sum())


def distill(z, index, teacher, dloss, T=1.0):
    """(loss, lse, dz, q, share) of logits z [rows, V], slots index and teacher [rows, top] and
    weights dloss [rows], row by row: q is softmax(z / T), share [rows, V] what the row's slots put on
    each class.  A slot whose class is outside [0, V) or whose logit is -inf is empty; a row of empty
    slots has loss 0 and gradient 0."""
    rows, V = z.shape
    loss, lse = np.zeros(rows), np.zeros(rows)
    dz, q, share = np.zeros((rows, V)), np.zeros((rows, V)), np.zeros((rows, V))
    for r in range(rows):
        v = z[r] / T
        with np.errstate(invalid="ignore", divide="ignore"):
            lse[r] = v.max() + np.log(np.exp(v - v.max()).sum())
            q[r] = np.exp(v - lse[r])
        slots = [k for k in range(index.shape[1])
                 if 0 <= index[r, k] < V and teacher[r, k] != -np.inf]
        if not slots:
            continue
        logp = _log_softmax(teacher[r, slots] / T)
        for k, lp in zip(slots, logp):
            p = np.exp(lp)
            share[r, index[r, k]] += p
            if p > 0:
                loss[r] += T * T * p * (lp - (v[index[r, k]] - lse[r]))
        if dloss[r] != 0:
            dz[r] = dloss[r] * T * (q[r] - share[r])
    return loss, lse, dz, q, share
