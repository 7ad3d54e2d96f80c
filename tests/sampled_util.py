"""The acceptance walk in 64 bits that also says how far each of its comparisons is from its border."""
import numpy as np

# What a weight of rest_accept_sampled may be off by (largest weight 1): its 24-bit float is half a step,
# 2^-24 of itself; the exponential before that rounding is good to 5e-9 < 2^-27; it is a whole number of
# 2^-44, half a step of which is 2^-45, and what is below rounds to nothing.  The largest logit's weight
# is exactly 1, and equal logits have equal weights.
REL, ABS = 2.0 ** -24 + 2.0 ** -27, 2.0 ** -44


def walk(logits, tokens, parents, n_nodes, uniforms, temperature, top_p, max_depth):
    """One context (numpy; logits float64 [N+1,V]).  Returns (accepted nodes, emitted tokens, clear): clear is
    the smallest of |difference| / what the weights' errors may move it by over all comparisons that the walk
    makes (above 1: no comparison can fall the other way)."""
    N, V = tokens.shape[0], logits.shape[1]
    u = np.clip(np.nan_to_num(uniforms.astype(np.float64), nan=0.0), 0.0, np.float64(np.float32(0.99999994)))
    nodes, out, cur, clear = [], [], -1, np.inf

    def compare(a, b, err):                      # sums in double and the kernel's products in double: 2^-52
        nonlocal clear
        clear = min(clear, abs(a - b) / (err + 2.0 ** -50 * (abs(a) + abs(b)) + 1e-300))

    while True:
        x = logits[cur + 1].astype(np.float64).copy()
        x[np.isnan(x)] = -np.inf
        if not (x > -np.inf).any():
            out.append(-1)
            return nodes, out, clear
        order = np.lexsort((np.arange(V), -x))
        certain = x == x.max()
        if temperature > 0:
            with np.errstate(invalid="ignore", over="ignore"):
                w = np.where(certain, 1.0, np.exp((x - x.max()) / min(np.float64(temperature), np.float64(np.float32(1e30)))))
            w[w < 2.0 ** -46] = 0.0
            err = np.where(certain | (w == 0), 0.0, w * REL + ABS)
            w[w < 2.0 ** -44] = 0.0              # such a weight is nothing, or one step
            if top_p < 1:
                p, total = np.float64(top_p), w.sum()
                before = np.cumsum(w[order]) - w[order]
                off = np.cumsum(err[order]) - err[order] + max(p, 0.0) * err.sum() + 2.0 ** -43
                if p > 0:
                    # the first token is always in; nothing follows from where weights are 0
                    for r in np.nonzero(w[order] > 0)[0][1:]:
                        compare(before[r], p * total, off[r])
                drop = before >= p * total
                drop[0] = False
                w[order[drop]] = err[order[drop]] = 0.0
        else:
            w, err = np.zeros(V), np.zeros(V)
            w[order[0]] = 1.0
        child = -1
        for c in range(min(max(int(n_nodes), 0), N)):
            t = tokens[c]
            if len(nodes) < max_depth and parents[c] == cur and 0 <= t < V and w[t] > 0:
                compare(u[c + 1] * w.sum(), w[t], err[t] + u[c + 1] * err.sum())
                if u[c + 1] * w.sum() < w[t]:
                    child = c
                    break
                w[t] = err[t] = 0.0
        if child < 0:
            cdf, off = np.cumsum(w), np.cumsum(err) + u[0] * err.sum()
            if u[0] > 0:                         # (a draw at 0 takes the first token that is there)
                for v in np.nonzero(w > 0)[0]:
                    compare(cdf[v], u[0] * cdf[-1], off[v])
            out.append(int(np.argmax(cdf > u[0] * cdf[-1])))
            return nodes, out, clear
        nodes.append(child)
        out.append(int(tokens[child]))
        cur = child
