"""Plain forms, in 64 bits, of the key/value cache in 4 bits and of the attention over it, and the tolerances of the kernels that compute them."""
import numpy as np

from cache_attention_reference import BF16_HALF_STEP, attention, logit_error, lse_tolerance, visible

GROUP = 32


def scales_of(d):
    """Places for scales in a row."""
    return 2 if d <= 64 else 4 if d <= 128 else 8


def quantise(x):
    """x [.., d] float64 -> integers [.., d] and scales [.., d / 32]: largest magnitude / 7 up to four significant bits (and a multiple of 2^-129), 2^122 at
    most; a group with a value that is no finite number: a scale that is none, integers 0."""
    x = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, GROUP)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    top = np.abs(x).max(-1)
    mantissa, exponent = np.frexp(top / 7)
    step = np.maximum(np.ldexp(1.0, exponent - 4), 2.0 ** -129)
    scale = np.minimum(np.ceil(top / 7 / step) * step, 2.0 ** 122)
    code = np.where(scale[..., None] > 0, np.rint(x / np.where(scale > 0, scale, 1.0)[..., None]), 0.0)
    code = np.clip(code, -7, 7)
    scale = np.where(bad, np.nan, scale)
    return code.reshape(*code.shape[:-2], -1).astype(int), scale


def values(code, scale):
    return code * np.repeat(scale, GROUP, -1)


def places(d):
    """(byte, bits to shift) of each value of a row."""
    G = d // GROUP
    return [(4 * (x % GROUP // 8 * G + x // GROUP) + x % 8 // 2, 4 * (x % 2)) for x in range(d)]


def pack(code):
    """Integers [.., d] -> bytes [.., d / 2]."""
    d = code.shape[-1]
    held = np.zeros((*code.shape[:-1], d // 2), dtype=np.uint8)
    for x, (byte, shift) in enumerate(places(d)):
        held[..., byte] |= ((code[..., x] + 8) << shift).astype(np.uint8)
    return held


def unpack(held):
    code = np.zeros((*held.shape[:-1], held.shape[-1] * 2), dtype=int)
    for x, (byte, shift) in enumerate(places(code.shape[-1])):
        code[..., x] = ((held[..., byte] >> shift) & 15).astype(int) - 8
    return code


def slot_of(p, L, sinks=0, rolling=False):
    return p if not rolling or p < sinks else sinks + (p - sinks) % (L - sinks)


def tensors(code, scale, by_token=False, device="cuda", fill=0.0):
    """Codes and scales of rows [n_seq, n_head, L, d] as a cache holds them; `fill`: what lies in the places for scales behind the last group."""
    import torch
    d = code.shape[-1]
    held = torch.from_numpy(pack(code))
    sc = torch.full((*scale.shape[:-1], scales_of(d)), fill, dtype=torch.bfloat16)
    sc[..., : d // GROUP] = torch.from_numpy(scale).to(torch.bfloat16)
    if by_token:
        return tuple(x.transpose(1, 2).contiguous().to(device).transpose(1, 2) for x in (held, sc))
    return held.to(device), sc.to(device)


# Logits: a row's queries are fp16 numbers scaled so that the largest is 2^14 or more, in half of the places 2^10: exact, or rounded by 2^-25 at most, 2^-35 of the
# largest.  Times |s c| <= 7 s that is what 32 values add to a group's sum.  The sum itself begins with -8 times the sum of the queries, which is off by 32 2^-24
# of sum |q|, and takes two tensor instructions of 16 products of at most 15 |q|, that may cut each of their 17 terms 2^-23 below the largest, at most
# 8 sum |q| + 15 max |q|.  Then the scales multiply and G sums are added, as the other attention kernels' d products are.
def quant_logit_error(q, scale, K_scale, spread, d):
    """q [g, d], K_scale [n, d / 32]: for every row of q."""
    q = np.abs(q)
    sums, top = q.reshape(q.shape[0], -1, GROUP).sum(-1), q.max(-1, keepdims=True)          # [g, d / 32], [g, 1]
    group = 7 * GROUP * 2.0 ** -35 * top + 8 * 32 * 2.0 ** -24 * sums + 2 * 17 * 2.0 ** -23 * (8 * sums + 15 * top)
    return abs(scale) * (group @ K_scale.T).max(1, initial=0.0) + logit_error(spread, d)


def quant_out_tolerance(out, absolute, error, prompt, n, V_scale):
    """`absolute`: the weighted sum of |V|; n keys; V_scale: the largest of their values' scales.  Weights are off by exp(+-2 error) and 2^-20.  Prompts: rounded to
    bf16, 2^-8.  Otherwise: rounded to fp16 before and behind the product with a scale, 2^-11 each; products of less than 2^-14 by 2^-25, in units in which the
    largest weight is 2^6 and the largest scale 1 / 2 or more, and their codes' magnitudes are 7 at most: n 2^-31 14 V_scale.  Sums in fp32: chains of at most 2^8
    additions, 2^-24 each.  The output is rounded to bf16."""
    e = np.expm1(2 * error)[..., None] + 2.0 ** -20
    if prompt:
        return BF16_HALF_STEP * (np.abs(out) + absolute) * 1.01 + absolute * (e + 2.0 ** -16) + 1e-30
    return BF16_HALF_STEP * np.abs(out) * 1.01 + absolute * (e + 2.0 ** -10 * 1.01 + 2.0 ** -16) + V_scale * n * 2.0 ** -31 * 14 + 1e-30


def taken_as_prompts(T, n_seq, n_head, group, L, d, scale):
    units = T * n_head * ((group + 15) // 16) * (L // 32 + 1) * (4 if group > 8 else 1)
    return (d in (64, 96, 128) and scale > 0 and T * group >= 64 and T >= 8 * n_seq
            and units >= (8192 if n_seq == 1 or T >= 48 * n_seq else 32768))


class QuantCase:
    """Inputs of one attention call on the GPU and what it should return.  tokens: a list of (sequence, position)."""

    def __init__(self, tokens, n_head, group, d, n_seq, L, *, seed=0, gain=2.0, scale=None, by_token=False, members_first=False, hide=None, device="cuda",
                 value_gain=1.0):
        import torch
        rng = np.random.default_rng(seed)
        self.tokens, self.n_head, self.group, self.d, self.n_seq, self.L = tokens, n_head, group, d, n_seq, L
        self.scale = 1.0 / np.sqrt(d) if scale is None else scale
        T = len(tokens)
        q = torch.from_numpy((rng.standard_normal((T, n_head, group, d)) * gain).astype(np.float32)).to(torch.bfloat16)
        self.q_np = q.double().numpy()
        held, self.scales_np, self.values_np = [], [], []
        for by in (1.0, value_gain):
            code, sc = quantise(rng.standard_normal((n_seq, n_head, L, d)) * by)
            self.scales_np.append(sc)
            self.values_np.append(values(code, sc))
            if hide is not None:                  # what no token sees may be anything: (sequence, slot) by hide(s, slot)
                code, sc = code.copy(), sc.copy()
                for s in range(n_seq):
                    for l in range(L):
                        if hide(s, l):
                            code[s, :, l], sc[s, :, l] = 7 - l % 16, [np.nan, np.inf, -np.inf, 3e38][l % 4]
            held.append(tensors(code, sc, by_token, device, fill=float("nan")))
        (self.K, self.K_scale), (self.V, self.V_scale) = held
        self.q = q.to(device)
        if members_first:
            self.q = self.q.transpose(1, 2).contiguous().transpose(1, 2)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((T, n_head, group), 7.0, device=device)
        self.tok_seq = torch.tensor([s for s, _ in tokens], dtype=torch.int32, device=device)
        self.pos = torch.tensor([p for _, p in tokens], dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def cache(self):
        import paper_2404_05567_b200 as dm
        return dm.make_quant_cache(self.K, self.V, self.K_scale, self.V_scale)

    def prompts(self):
        return taken_as_prompts(len(self.tokens), self.n_seq, self.n_head, self.group, self.L, self.d, self.scale)

    def expected(self, window=None, sinks=0, rolling=False, seen_at=visible):
        T, d, prompt = len(self.tokens), self.d, self.prompts()
        out, lse = np.zeros((T, self.n_head, self.group, d)), np.zeros((T, self.n_head, self.group))
        out_tol, lse_tol = np.zeros_like(out), np.zeros_like(lse)
        K, V = self.values_np
        for t, (s, p) in enumerate(self.tokens):
            at = np.array([slot_of(l, self.L, sinks, rolling) for l in seen_at(p, window, sinks)], dtype=int)
            for j in range(self.n_head):
                q = self.q_np[t, j]
                o, x, _, absolute, spread = attention(q, K[s, j], V[s, j], self.scale, at)
                error = quant_logit_error(q, self.scale, self.scales_np[0][s, j][at], spread, d)
                out[t, j], lse[t, j] = o, x
                largest = self.scales_np[1][s, j][at].max(initial=0.0)
                out_tol[t, j], lse_tol[t, j] = quant_out_tolerance(o, absolute, error, prompt, len(at), largest), error + lse_tolerance(x, spread, d)
        return out, lse, out_tol, lse_tol

    def check(self, want):
        got, lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        out, x, out_tol, lse_tol = want
        assert np.isfinite(got).all()
        worst = np.abs(got - out) - out_tol
        assert worst.max(initial=-1) <= 0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
        none = ~np.isfinite(x)
        assert (lse[none] == -np.inf).all() and np.isfinite(lse[~none]).all()
        assert (np.abs(lse[~none] - x[~none]) <= lse_tol[~none]).all(), np.abs(lse[~none] - x[~none]).max()
        assert (got[none] == 0).all()
