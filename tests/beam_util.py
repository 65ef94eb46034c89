"""beam_select from its definition, in 64 bits, on numpy arrays."""
import numpy as np

# Half of the distance from which beam_select compares sums in 64 bits (csrc/beams.hip derives it): what a sum in 32 bits, and so a
# score, may be off by.
LSE_ERROR = 5e-6


def select(logits, scores, beams, n_out, ended=None, eos=-1):
    """-> scores (64 bits), parent, token, ended, each [items, n_out], and whether something was not finite."""
    rows, vocab = logits.shape
    x = logits.astype(np.float64)
    bad = False
    got = [np.full((rows // beams, n_out), fill, dtype) for fill, dtype in ((-np.inf, np.float64), (-1, np.int64), (max(eos, 0), np.int64), (1, np.int64))]
    for item in range(rows // beams):
        s, b, t, done, logit = [], [], [], [], []
        for row in range(item * beams, (item + 1) * beams):
            c = float(scores[row])
            if np.isnan(c) or c == np.inf:
                bad = True
            elif c == -np.inf:
                pass
            elif ended is not None and ended[row]:
                s.append([c]), b.append([row]), t.append([eos]), done.append([1]), logit.append([0.0])
            elif np.isnan(x[row]).any() or (x[row] == np.inf).any():
                bad = True
            else:
                some = np.flatnonzero(x[row] > -np.inf)
                if len(some):
                    v = x[row][some]
                    top = v.max()
                    s.append(c + ((v - top) - np.log(np.exp(v - top).sum())))  # (a constant added to a row changes nothing)
                    b.append(np.full(len(some), row)), t.append(some), done.append((some == eos).astype(np.int64)), logit.append(v)
        if not s:
            continue
        s, b, t, done, logit = (np.concatenate(y) for y in (s, b, t, done, logit))
        best = np.lexsort((t, -logit, b, -s))[:n_out]
        for out, y in zip(got, (s, b, t, done)):
            out[item, :len(best)] = y[best]
    return got[0], got[1], got[2], got[3], bad
