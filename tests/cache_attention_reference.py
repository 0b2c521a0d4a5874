"""Plain forms, in 64 bits and one token at a time, of the attention steps on a key/value cache and of the eviction from one; and the tolerances of the
kernels that compute them."""
import numpy as np

# What a call may be off, from its roundings alone.  Logits: products of bf16 are exact in fp32, d_head of them are added with at most
# one rounding each of the running sum, which is no larger than sum |q_i k_i| (LOGIT_EPS below, times that sum and the scale).  A weight 2^(x - m)
# then carries that error of the exponent and the exponential's own 2^-21.  Weights may be rounded to bf16 before they multiply the values:
# at most 2^-8 of each, so at most 2^-8 sum w |v| in an output; the output is rounded once more, at most 2^-8 of it.
BF16_HALF_STEP = 2.0 ** -8


def attention(q, K, V, scale, seen):
    """q [g, d], K, V [n, d] and seen: the indices of the visible keys, in float64.  Returns out [g, d], lse [g], weights [g, len(seen)] and the
    weighted sum of |V| and of each row's sum |q_i k_i| maximum, for tolerances."""
    q, K, V = q.astype(np.float64), K[seen].astype(np.float64), V[seen].astype(np.float64)
    if len(seen) == 0:
        zero = np.zeros((q.shape[0], q.shape[1]))
        return zero, np.full(q.shape[0], -np.inf), np.zeros((q.shape[0], 0)), zero, np.zeros(q.shape[0])
    x = scale * (q @ K.T)
    top = x.max(1, keepdims=True)
    w = np.exp(x - top)
    total = w.sum(1, keepdims=True)
    p = w / total
    return p @ V, (top + np.log(total))[:, 0], p, p @ np.abs(V), abs(scale) * (np.abs(q) @ np.abs(K).T).max(1)


def visible(pos, window=None, sinks=0):
    """Positions that a token at `pos` sees."""
    return [l for l in range(pos + 1) if window is None or pos - l < window or l < sinks]


def logit_error(spread, d):
    """At most this is a logit off: d roundings of a running sum of at most `spread`, each of at most a step of fp32 (tensor cores cut instead of
    rounding), and two of the product with the scale."""
    return (d + 4) * 2.0 ** -23 * spread


def out_tolerance(out, absolute, spread, d):
    """`absolute`: the weighted sum of |V|.  Weights off by a factor exp(+-2 e) (the row's sum has the same error) and 2^-20, rounded to bf16; sums in
    fp32 whose chains are at most 2^8 additions long, a rounding of at most 2^-24 each; the output rounded to bf16."""
    e = np.expm1(2 * logit_error(spread, d))[..., None] + 2.0 ** -20
    return BF16_HALF_STEP * (np.abs(out) + absolute) * 1.01 + absolute * (e + 2.0 ** -16) + 1e-30


def lse_tolerance(lse, spread, d):
    return logit_error(spread, d) + 2.0 ** -18 + np.abs(np.where(np.isfinite(lse), lse, 0.0)) * 2.0 ** -22


def evict(tally, length, keep, sinks, recent):
    """Indices that stay, ascending."""
    n = int(length)
    if n <= keep:
        return list(range(n))
    t = np.where(np.isnan(tally[:n]), -np.inf, tally[:n]).astype(np.float64)
    nan = np.isnan(tally[:n])
    middle = sorted(range(sinks, n - recent), key=lambda i: (nan[i], -t[i], i))[: keep - sinks - recent]
    return sorted(list(range(sinks)) + middle + list(range(n - recent, n)))


def tally_tolerance(tally_in, added, error, rows):
    """`added`: the sum of the weights; `error`: the sum of each weight times its own relative error (two logits' errors and 2^-20); one rounding a row
    and the last addition's."""
    return error + (rows + 2) * 2.0 ** -24 * added + 2.0 ** -24 * np.abs(tally_in + added) + 1e-30


class Case:
    """Inputs of one call on the GPU and what it should return.  tokens: a list of (sequence, position)."""

    def __init__(self, tokens, n_head, group, d, n_seq, L, *, seed=0, P=0, gain=2.0, scale=None, by_token=False, members_first=False,
                 hide=None, device="cuda"):
        import torch
        rng = np.random.default_rng(seed)
        self.tokens, self.n_head, self.group, self.d, self.n_seq, self.L, self.P = tokens, n_head, group, d, n_seq, L, P
        self.scale = 1.0 / np.sqrt(d) if scale is None else scale
        T = len(tokens)

        def draw(*shape, by=1.0):
            x = torch.from_numpy((rng.standard_normal(shape) * by).astype(np.float32)).to(torch.bfloat16)
            return x, x.float().numpy()
        q, self.q_np = draw(T, n_head, group, d, by=gain)
        K, self.K_np = draw(n_seq, n_head, L, d)
        V, self.V_np = draw(n_seq, n_head, L, d)
        if hide is not None:                      # what no token sees may be anything: (sequence, slot) by hide(s, slot)
            for s in range(n_seq):
                for l in range(L):
                    if hide(s, l):
                        K[s, :, l] = [float("nan"), float("inf"), -float("inf"), 3e38][l % 4]
                        V[s, :, l] = [float("inf"), float("nan"), 3e38, -float("inf")][l % 4]
        if by_token:                              # a cache stored by position
            K, V = (x.transpose(1, 2).contiguous().to(device).transpose(1, 2) for x in (K, V))
        else:
            K, V = K.to(device), V.to(device)
        self.K, self.V = K, V
        self.q = q.to(device)
        if members_first:                         # the attention layer's order: experts before heads
            self.q = self.q.transpose(1, 2).contiguous().transpose(1, 2)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((T, n_head, group), 7.0, device=device)
        self.tok_seq = torch.tensor([s for s, _ in tokens], dtype=torch.int32, device=device)
        self.pos = torch.tensor([p for _, p in tokens], dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        if P:
            Kp, self.Kp_np = draw(n_head, P, d)
            Vp, self.Vp_np = draw(n_head, P, d)
            self.Kp, self.Vp = Kp.to(device), Vp.to(device)

    def desc(self):
        import paper_2404_05567_b200 as dm
        return dm.make_attention_desc(self.q, self.K, self.scale, self.out)

    def expected(self, window=None, sinks=0, rolling=False):
        """(out, lse, tolerance of out, tolerance of lse, weights by key and their relative error)"""
        T, d = len(self.tokens), self.d
        out, lse = np.zeros((T, self.n_head, self.group, d)), np.zeros((T, self.n_head, self.group))
        out_tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
        tally, tally_err = np.zeros((self.n_seq, self.n_head, self.L)), np.zeros((self.n_seq, self.n_head, self.L))
        ring = self.L - sinks
        for t, (s, p) in enumerate(self.tokens):
            seen = visible(p, window, sinks)
            slots = [l if not rolling or l < sinks else sinks + (l - sinks) % ring for l in seen]
            for j in range(self.n_head):
                K, V, at = self.K_np[s, j], self.V_np[s, j], np.array(slots, dtype=int)
                if self.P:
                    K, V = np.concatenate((self.Kp_np[j], K)), np.concatenate((self.Vp_np[j], V))
                    at = np.concatenate((np.arange(self.P), self.P + at))
                o, x, w, absolute, spread = attention(self.q_np[t, j], K, V, self.scale, at)
                out[t, j], lse[t, j] = o, x
                out_tol[t, j], lse_tol[t, j] = out_tolerance(o, absolute, spread, d), lse_tolerance(x, spread, d)
                if not self.P:
                    np.add.at(tally[s, j], at, w.sum(0))
                    np.add.at(tally_err[s, j], at, (w * (np.expm1(2 * logit_error(spread, d)) + 2.0 ** -20)[:, None]).sum(0))
        return out, lse, out_tol, lse_tol, tally, tally_err

    def check(self, want):
        got, lse = self.out.float().cpu().numpy().astype(np.float64), self.lse.cpu().numpy().astype(np.float64)
        out, x, out_tol, lse_tol = want[:4]
        assert np.isfinite(got).all()
        worst = np.abs(got - out) - out_tol
        assert worst.max(initial=-1) <= 0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
        none = ~np.isfinite(x)
        assert (lse[none] == -np.inf).all() and np.isfinite(lse[~none]).all()
        assert (np.abs(lse[~none] - x[~none]) <= lse_tol[~none]).all(), np.abs(lse[~none] - x[~none]).max()
        assert (got[none.any(-1) if none.ndim == 4 else none] == 0).all()
