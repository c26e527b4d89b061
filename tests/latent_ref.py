"""The latent-cache operators in 64 bits on the CPU, written from their definition (include/taper_latent.h), seeded batches for them,
and the arithmetic behind their tests' tolerances."""
import numpy as np

PAGE, ROPE = 16, 64
U = 2.0 ** -8  # half a step of bf16, relative to the value: every rounding to bf16 is off by at most this


def to_bf16(x):
    """float32 values that bf16 holds exactly (round to nearest even)."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).view(np.float32)


def pages_of(n):
    return (n + PAGE - 1) // PAGE


class Batch:
    """requests: [(prefix tokens, [[private segments of a sequence], ...]), ...]; new: new tokens per sequence (prompts)."""

    def __init__(self, requests, seed, new=None, spare=3):
        rng = np.random.default_rng(seed)
        used = sum(pages_of(p) + sum(pages_of(n) for segs in seqs for n in segs) for p, seqs in requests)
        self.n_pages = used + spare
        free = rng.permutation(self.n_pages).astype(np.int32)
        cur, rows, self.group, self.prefix, self.seg_start, self.seg_len = 0, [], [], [], [0], []
        for g, (p, seqs) in enumerate(requests):
            shared = free[cur:cur + pages_of(p)]
            cur += len(shared)
            for segs in seqs:
                n = sum(pages_of(x) for x in segs)
                rows.append(np.concatenate([shared, free[cur:cur + n]]))
                cur += n
                self.group.append(g)
                self.prefix.append(p)
                self.seg_len += segs
                self.seg_start.append(len(self.seg_len))
        self.table = np.full((len(rows), max(1, max(map(len, rows)))), -1, np.int32)
        for s, r in enumerate(rows):
            self.table[s, :len(r)] = r
        self.S = len(rows)
        self.new = np.array(new if new is not None else [1] * self.S, np.int32)
        self.unreferenced = free[cur:]

    def slots(self, s):
        """Physical slots of sequence s's tokens in logical order."""
        out, entry = [], 0
        for n in [self.prefix[s]] + self.seg_len[self.seg_start[s]:self.seg_start[s + 1]]:
            t = np.arange(n)
            out.append(self.table[s, entry + t // PAGE].astype(np.int64) * PAGE + t % PAGE)
            entry += pages_of(n)
        return np.concatenate(out)


def values(batch, H, R, hd, seed, rows=None):
    """q, w_up and the tokens (a row a slot, those of no token NaN), bf16-exact float32."""
    rng = np.random.default_rng(seed)
    n = int(batch.new.sum()) if rows is None else rows
    q = to_bf16(rng.standard_normal((n, H, hd + ROPE)))
    w = to_bf16(rng.standard_normal((H, 2 * hd, R)) * R ** -0.5)
    tok = np.full((batch.n_pages * PAGE, R + ROPE), np.nan, np.float32)
    live = np.unique(np.concatenate([batch.slots(s) for s in range(batch.S)]))
    tok[live] = to_bf16(rng.standard_normal((len(live), R + ROPE)))
    return q, w, tok


def pool_of(tok):
    """Rows of slots as the pool lays them out: [page][value / 8][token][8]."""
    n, d = tok.shape
    return np.ascontiguousarray(tok.reshape(n // PAGE, PAGE, d // 8, 8).transpose(0, 2, 1, 3))


def rows_of(pool):
    n, d8 = pool.shape[:2]
    return np.ascontiguousarray(pool.transpose(0, 2, 1, 3)).reshape(n * PAGE, d8 * 8)


def attention(batch, q, w, tok, H, R, hd, scale, absorbed):
    """(out, lse, bound of |out - exact| per element, bound of |lse - exact|) in float64.

    Bounds.  Absorbed: q_lat = W_k^T q_n is rounded, which moves a score by at most d = scale U sum_r |q_lat_r c_r|; the weights are
    rounded (U) and, with scores off by up to D = max_t d_t, off by a factor of at most exp(2 D); the merged sum of latents is rounded
    before W_v (U sum_r |W_v| |o_lat|).  Expanded: keys and values are rounded, d = scale U sum_n |q_n k_n|, and U sum_t p_t |v_t|.  Both
    round the result.  What 32-bit sums add is below U / 100 of the same terms: the bounds get 2 % for it, and 1e-6 absolute."""
    q, w, tok = q.astype(np.float64), w.astype(np.float64), tok.astype(np.float64)
    out = np.zeros((q.shape[0], H, hd))
    lse = np.zeros((q.shape[0], H))
    tol, tol_lse = np.zeros_like(out), np.zeros_like(lse)
    r0 = 0
    for s in range(batch.S):
        n = int(batch.new[s])
        if n == 0:
            continue
        c = tok[batch.slots(s)]
        T = len(c)
        rows = slice(r0, r0 + n)
        r0 += n
        see = np.tril(np.ones((n, T), bool), T - n)
        for h in range(H):
            k, v = c[:, :R] @ w[h, :hd].T, c[:, :R] @ w[h, hd:].T
            sc = scale * (q[rows, h, :hd] @ k.T + q[rows, h, hd:] @ c[:, R:].T)
            if absorbed:
                d = scale * U * np.abs(q[rows, h, :hd] @ w[h, :hd]) @ np.abs(c[:, :R]).T
            else:
                d = scale * U * np.abs(q[rows, h, :hd]) @ np.abs(k).T
            sc, D = np.where(see, sc, -np.inf), np.where(see, d, 0).max(1, keepdims=True)
            m = sc.max(1, keepdims=True)
            p = np.exp(sc - m)
            z = p.sum(1, keepdims=True)
            p /= z
            out[rows, h], lse[rows, h] = p @ v, (m + np.log(z))[:, 0]
            D = np.minimum(D, 300)  # (the bound is without effect long before)
            off = np.expm1(2 * D) + U
            bound = off * (p @ np.abs(v))
            if absorbed:
                bound += U * np.abs(p @ c[:, :R]) @ np.abs(w[h, hd:]).T * np.exp(2 * D)
            else:
                bound += U * (p @ np.abs(v)) * np.exp(2 * D)
            tol[rows, h] = 1.02 * (bound + U * (np.abs(out[rows, h]) + bound)) + 1e-6
            tol_lse[rows, h] = 1.02 * D[:, 0] + 1e-5 * (1 + np.abs(lse[rows, h]))
    return out, lse, tol, tol_lse


# Independent roundings add up as squares.  Relative to the result's own size each of the four roundings above (weights, scores through
# the softmax, latents or values, result) contributes at most U / sqrt(3) where scores have a standard deviation of at most 1.5: together
# below U / sqrt(3) sqrt(3 + 1.5^2) < 1.4 U.  2 U over all elements of a test.
RMS = 2 * U
