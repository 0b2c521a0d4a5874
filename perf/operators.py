"""The operators on a key/value cache that is bounded, shared or thinned out, as cases that can be timed and compared.

  window   dsmoe_window_attention: each token sees the last `window` keys and the first `sinks`; a cache of all positions or a rolling one
  prefix   dsmoe_prefix_attention: a batch whose sequences share one long prefix, each with a cache of its own behind it
  tally    dsmoe_tally_attention: causal attention that also adds up the weight that each key of the cache got
  evict    dsmoe_cache_evict: thins a cache out to the keys with the largest tally

Head shapes are those of the attention layer (4 heads of 128 with 5 experts a token, 4 of 96 and 2 of 64 with 6) and generic ones.  A case has
n_seq sequences with n neighbouring tokens each; `least` to 1 is the range, relative to the room there is, over which the sequences' lengths
are spread.
"""
import math

import torch

own = False


def _case(op, n_seq, n, n_head, group, d_head, L, **more):
    return {"op": op, "n_seq": n_seq, "n": n, "n_head": n_head, "group": group, "d_head": d_head, "L": L, "least": 0.5, **more}


def _window(n_seq, n, n_head, group, d_head, L, window, sinks, *, rolling=False, by_token=False, idle=0, **more):
    """rolling: the cache keeps its first `sinks` positions and the latest others; by_token: it is stored [n_seq][L][n_head][d_head];
    idle: that many sequences of the batch are padding (position -1)."""
    return _case("window", n_seq, n, n_head, group, d_head, L, window=window, sinks=sinks, rolling=rolling, by_token=by_token, idle=idle, **more)


def _prefix(n_seq, n, n_head, group, d_head, P, L, **more):
    return _case("prefix", n_seq, n, n_head, group, d_head, L, P=P, **more)


def _tally(n_seq, n, n_head, group, d_head, L, **more):
    return _case("tally", n_seq, n, n_head, group, d_head, L, **more)


def _evict(n_seq, n_head, d_head, L, keep, sinks, recent, **more):
    return _case("evict", n_seq, 0, n_head, 1, d_head, L, keep=keep, sinks=sinks, recent=recent, **more)


def listed():
    named = [
        # one conversation, one token, a rolling cache: what counts is latency
        ("window_one_token", _window(1, 1, 4, 5, 128, 516, 512, 4, rolling=True)),
        # a decoding batch with two padded entries, long contexts of ragged lengths
        ("window_decode", _window(64, 1, 4, 5, 128, 8192, 2048, 4, by_token=True, idle=2)),
        # prompts of ragged contexts, the odd head width, a window that ends inside tiles
        ("window_prompts", _window(3, 1111, 4, 6, 96, 2500, 700, 3)),
        # one long prompt
        ("window_long_prompt", _window(1, 8192, 4, 5, 128, 8192, 4096, 4, least=1.0)),
        # a few requests behind a system prompt
        ("prefix_few", _prefix(4, 1, 4, 5, 128, 1500, 200)),
        # a decoding batch behind a long document
        ("prefix_decode", _prefix(48, 1, 4, 5, 128, 16384, 777)),
        # many samples of one document, and a prefix that outweighs everything
        ("prefix_many", _prefix(256, 1, 8, 4, 128, 32768, 512)),
        # decoding with tallies, ragged contexts
        ("tally_decode", _tally(32, 1, 4, 5, 128, 4096)),
        # the tallies of whole prompts
        ("tally_prompts", _tally(4, 1000, 2, 6, 64, 1500)),
        # one conversation's cache is halved
        ("evict_one", _evict(1, 4, 128, 2048, 1024, 4, 128)),
        # a batch of long contexts down to an eighth, one that is not a power of two
        ("evict_batch", _evict(32, 4, 128, 16384, 2000, 4, 256)),
        # small heads, odd sizes
        ("evict_odd", _evict(7, 2, 64, 5001, 3333, 1, 77)),
    ]
    return [{"name": name, **case} for name, case in named]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """More cases of the same ranges: from one token to thousands, contexts from a few keys to tens of thousands, odd sizes among them."""
    op = rng.choice(["window", "window", "prefix", "tally", "evict"])
    n_head, group, d_head = rng.choice([(4, 5, 128), (4, 6, 96), (2, 6, 64), (8, 4, 128), (1, 16, 128), (4, 1, 64), (2, 7, 128)])
    least = rng.choice([0.1, 0.5, 0.9])
    if op == "evict":
        L = _log_int(rng, 200, 20000)
        n_seq = _log_int(rng, 1, max(1, min(64, 400000 // L)))
        keep = rng.randint(max(8, L // 8), max(9, L - 1))
        sinks, recent = rng.randint(0, min(8, keep // 4)), rng.randint(0, keep // 2)
        return _evict(n_seq, n_head, d_head, L, keep, sinks, recent, least=least)
    if op == "prefix":
        P, L = _log_int(rng, 100, 20000), _log_int(rng, 16, 800)
        n = rng.choice([1, 1, 1, rng.randint(2, min(12, L))])
        return _prefix(_log_int(rng, 1, 128 // n), n, n_head, group, d_head, P, L, least=least)
    prompt = rng.random() < 0.5
    if op == "tally":
        L = _log_int(rng, 50, 2000 if prompt else 8000)
        n = _log_int(rng, 2, L) if prompt else 1
        n_seq = _log_int(rng, 1, max(1, min(48, 4000 // n if prompt else 200000 // L)))
        return _tally(n_seq, n, n_head, group, d_head, L, least=least)
    L = _log_int(rng, 50, 4000 if prompt else 20000)
    n = _log_int(rng, 2, L) if prompt else 1
    n_seq = _log_int(rng, 1, max(1, min(64, 4000 // n if prompt else 400000 // L)))
    window, sinks = _log_int(rng, 8, L), rng.choice([0, 1, 4, 16])
    rolling = rng.random() < 0.4
    if rolling:                                    # room for the sinks, the window and the tokens of the call
        L = window + sinks + n
    return _window(n_seq, n, n_head, group, d_head, L, window, sinks, rolling=rolling, by_token=rng.random() < 0.3,
                   idle=0 if n_seq < 4 else rng.choice([0, 1]), least=least)


# ---------------------------------------------------------------- what the cases hold

def _lengths(c):
    """Keys that each sequence has (0: a padded entry); with rolling caches, positions that it has seen."""
    room = 6 * c["L"] if c.get("rolling") else c["L"]
    low = max(c["n"], 1, int(c["least"] * room))
    got = [low + int((room - low) * ((i + 1) * 0.6180339887498949 % 1.0)) for i in range(c["n_seq"])]
    if c["least"] == 1.0:
        got = [room] * c["n_seq"]
    idle = c.get("idle", 0)
    return got[:c["n_seq"] - idle] + [0] * idle


def _sight(c, last):
    """(first key behind the sinks, number of visible sinks) of a token at position `last`."""
    if c["op"] != "window":
        return 0, 0
    first = max(0, last - c["window"] + 1)
    return first, min(c["sinks"], first, last + 1)


def work(c):
    n_head, group, d_head = c["n_head"], c["group"], c["d_head"]
    if c["op"] == "evict":
        have = _lengths(c)
        kept = [min(n, c["keep"]) for n in have]
        return {"bytes": n_head * (sum(have) * 4 + sum(kept) * (8 * d_head + 4 + 4)), "flops": 0}
    pairs = keys = 0
    for n in _lengths(c):
        if n == 0:
            continue
        seen = 0
        for last in range(n - c["n"], n):
            first, sinks = _sight(c, last)
            pairs += last + 1 - first + sinks
            seen = max(seen, sinks)
        first = _sight(c, n - c["n"])[0]
        keys += n - first + min(seen, first)
    rows = c["n_seq"] * c["n"] * n_head * group
    pairs += c["n_seq"] * c["n"] * c.get("P", 0)
    size = n_head * (keys + c.get("P", 0)) * d_head * 4 + rows * (d_head * 4 + 4)
    if c["op"] == "tally":
        size += c["n_seq"] * n_head * c["L"] * 8
    return {"bytes": size, "flops": 4 * d_head * pairs * n_head * group}


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, gain=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * gain).to(dtype)

    n_seq, n, n_head, group, d_head, L = (c[k] for k in ("n_seq", "n", "n_head", "group", "d_head", "L"))
    s = {"case": c, "scale": 1.0 / math.sqrt(d_head)}
    s["have"] = torch.tensor(_lengths(c), dtype=torch.int32).cuda()
    if c.get("by_token"):
        s["K"], s["V"] = (normal(n_seq, L, n_head, d_head).transpose(1, 2) for _ in range(2))
    else:
        s["K"], s["V"] = (normal(n_seq, n_head, L, d_head) for _ in range(2))
    if c["op"] in ("tally", "evict"):
        # accumulated weights: a few heavy keys, a third that never got any
        t = torch.exp(2.0 * torch.randn((n_seq, n_head, L), generator=gen, device="cuda")) * 0.05
        s["tally"] = torch.where(torch.rand((n_seq, n_head, L), generator=gen, device="cuda") < 1 / 3, torch.zeros_like(t), t)
        s["tally_out"] = torch.zeros_like(s["tally"])
    if c["op"] == "evict":
        keep = c["keep"]
        s["K_out"], s["V_out"] = (torch.zeros((n_seq, n_head, keep, d_head), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["tally_out"] = torch.zeros((n_seq, n_head, keep), device="cuda")
        s["kept"] = torch.full((n_seq, n_head, keep), -1, dtype=torch.int32, device="cuda")
        s["have_out"] = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
    else:
        T = n_seq * n
        s["q"] = normal(T, n_head, group, d_head, gain=2.0)
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros((T, n_head, group), device="cuda")
        s["tok_seq"] = torch.arange(n_seq, dtype=torch.int32, device="cuda").repeat_interleave(n)
        ago = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
        s["pos"] = torch.where(s["have"][:, None] > 0, s["have"][:, None] - 1 - ago, -1).reshape(T).contiguous()
        if c["op"] == "prefix":
            s["Kp"], s["Vp"] = (normal(n_head, c["P"], d_head) for _ in range(2))
    if own:
        import paper_2404_05567_b200 as dm
        if c["op"] == "evict":
            s["desc"] = dm.make_attention_desc(None, s["K"])
            size = dm.dsmoe_evict_workspace_size(s["desc"])
        else:
            s["desc"] = dm.make_attention_desc(s["q"], s["K"], s["scale"])
            kind = {"window": dm.ATTENTION_WINDOW, "prefix": dm.ATTENTION_PREFIX, "tally": dm.ATTENTION_TALLY}[c["op"]]
            size = dm.dsmoe_attention_workspace_size(s["desc"], kind, c.get("P", 0))
        s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2404_05567_b200 as dm
    c = s["case"]
    if c["op"] == "evict":
        dm.dsmoe_cache_evict(s["desc"], c["keep"], c["sinks"], c["recent"], s["have"], s["tally"], s["K"], s["V"], s["kept"], s["have_out"],
                             s["tally_out"], s["K_out"], s["V_out"], s["ws"])
        return {k: s[k] for k in ("kept", "have_out", "tally_out", "K_out", "V_out")}
    common = s["q"], s["K"], s["V"], s["tok_seq"], s["pos"], s["out"], s["lse"]
    if c["op"] == "window":
        dm.dsmoe_window_attention(s["desc"], c["window"], c["sinks"], c["rolling"], *common, s["ws"])
    elif c["op"] == "prefix":
        dm.dsmoe_prefix_attention(s["desc"], s["Kp"], s["Vp"], *common, s["ws"])
    else:
        dm.dsmoe_tally_attention(s["desc"], *common, s["tally"], s["tally_out"], s["ws"])
        return {"out": s["out"], "lse": s["lse"], "tally": s["tally_out"]}
    return {"out": s["out"], "lse": s["lse"]}


# ---------------------------------------------------------------- the plain form

def _soft(logits, seen):
    """Unnormalised weights, their sum and the logarithm of the sum of the exponentials, in a row's place zeros where it sees nothing."""
    if seen is not None:
        logits = logits.masked_fill(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    w = torch.exp(logits - top)
    total = w.sum(-1, keepdim=True)
    return w, total, top + torch.log(total)


def _plain_attention(s):
    c = s["case"]
    n_seq, n, n_head, group, d_head, L = (c[k] for k in ("n_seq", "n", "n_head", "group", "d_head", "L"))
    q = (s["q"].float() * s["scale"]).view(n_seq, n, n_head, group, d_head).permute(0, 2, 1, 3, 4).reshape(n_seq, n_head, n * group, d_head)
    pos = s["pos"].view(n_seq, n, 1)
    slot = torch.arange(L, device="cuda", dtype=torch.int32)
    if c.get("rolling"):
        # the position that a slot holds: the latest one up to the sequence's last that lies there
        last = pos.amax(1, keepdim=True)
        key = torch.where(slot < c["sinks"], slot.expand(n_seq, 1, L), last - torch.remainder(last - slot, L - c["sinks"]))
        key = torch.where((slot >= c["sinks"]) & (key < c["sinks"]), -1, key)
    else:
        key = slot.expand(n_seq, 1, L)
    seen = (key >= 0) & (key <= pos)
    if c["op"] == "window":
        seen = seen & ((pos - key < c["window"]) | (key < c["sinks"]))
    seen = seen[:, None, :, None, :].expand(n_seq, 1, n, group, L).reshape(n_seq, 1, n * group, L)
    logits = torch.matmul(q, s["K"].float().transpose(-1, -2))
    if c["op"] == "prefix":
        P = c["P"]
        shared = torch.matmul(q.transpose(0, 1).reshape(n_head, n_seq * n * group, d_head), s["Kp"].float().transpose(-1, -2))
        shared = shared.view(n_head, n_seq, n * group, P).transpose(0, 1)
        logits, seen = torch.cat((shared, logits), -1), torch.cat((torch.ones_like(shared, dtype=torch.bool), seen.expand(logits.shape)), -1)
        w, total, lse = _soft(logits, seen)
        out = torch.matmul(w[..., P:], s["V"].float())
        shared = w[..., :P].transpose(0, 1).reshape(n_head, n_seq * n * group, P)
        out = out + torch.matmul(shared, s["Vp"].float()).view(n_head, n_seq, n * group, d_head).transpose(0, 1)
    else:
        w, total, lse = _soft(logits, seen)
        out = torch.matmul(w, s["V"].float())
    out = torch.where(total > 0, out / total, torch.zeros_like(out))

    def by_token(x):
        return x.view(n_seq, n_head, n, group, -1).transpose(1, 2).reshape(n_seq * n, n_head, group, -1)

    got = {"out": by_token(out).to(torch.bfloat16), "lse": by_token(lse)[..., 0]}
    if c["op"] == "tally":
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
        got["tally"] = s["tally"] + w.sum(2)
    return got


def _plain_evict(s):
    c = s["case"]
    n_seq, n_head, L, keep = (c[k] for k in ("n_seq", "n_head", "L", "keep"))
    slot, have = torch.arange(L, device="cuda", dtype=torch.int32), s["have"][:, None, None]
    # in the order of being kept: the sinks and the recent ones, then by tally, ties to the lower index, then what is no key
    rank = torch.where((slot < c["sinks"]) | (slot >= have - c["recent"]) | (have <= keep), math.inf, s["tally"])
    rank = torch.where(slot < have, rank, -math.inf)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    kept = torch.where(torch.gather(slot.expand(n_seq, n_head, L), 2, order) < have, order, L)
    kept = torch.sort(kept, dim=-1).values
    real = kept < L
    at = torch.where(real, kept, 0)
    row = at[..., None].expand(*at.shape, c["d_head"])
    return {"kept": torch.where(real, kept, -1).to(torch.int32),
            "have_out": torch.clamp(s["have"], max=keep),
            "tally_out": torch.where(real, torch.gather(s["tally"], 2, at), s["tally_out"]),
            "K_out": torch.where(real[..., None], torch.gather(s["K"], 2, row), s["K_out"]),
            "V_out": torch.where(real[..., None], torch.gather(s["V"], 2, row), s["V_out"])}


def run(state):
    if own:
        return _own(state)
    return _plain_evict(state) if state["case"]["op"] == "evict" else _plain_attention(state)


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "evict":
        return _exact_evict(s)
    n, n_head, group, d_head = (c[k] for k in ("n", "n_head", "group", "d_head"))
    T = c["n_seq"] * n
    out = torch.zeros((T, n_head, group, d_head), dtype=torch.float64, device="cuda")
    lse = torch.full((T, n_head, group), -math.inf, dtype=torch.float64, device="cuda")
    tally = s["tally"].double() if c["op"] == "tally" else None
    for i, have in enumerate(_lengths(c)):
        lo = max(0, have - n - c.get("window", have) + 1)        # no token of this sequence sees a key before that, sinks apart
        at = torch.cat((torch.arange(min(c.get("sinks", 0), lo)), torch.arange(lo, have))).cuda()
        slot = at
        if c.get("rolling"):
            ring = c["L"] - c["sinks"]
            slot = torch.where(at < c["sinks"], at, c["sinks"] + (at - c["sinks"]) % ring)
        for j in range(n_head):
            keys, values = s["K"][i, j, slot].double(), s["V"][i, j, slot].double()
            if c["op"] == "prefix":
                keys, values = torch.cat((s["Kp"][j].double(), keys)), torch.cat((s["Vp"][j].double(), values))
            step = max(1, (1 << 27) // max(1, group * len(keys)))
            for a in range(0, n, step):
                b = min(n, a + step)
                t = slice(i * n + a, i * n + b)
                x = torch.einsum("tgd,kd->tgk", s["q"][t, j].double(), keys) * s["scale"]
                p = torch.arange(have - n + a, have - n + b, device="cuda") if have else torch.full((b - a,), -1, device="cuda")
                hidden = at[None, :] > p[:, None]
                if c["op"] == "window":
                    hidden |= (at[None, :] <= p[:, None] - c["window"]) & (at[None, :] >= c["sinks"])
                if c["op"] == "prefix":
                    hidden = torch.cat((torch.zeros((b - a, c["P"]), dtype=torch.bool, device="cuda"), hidden), 1)
                x[hidden[:, None, :].expand(x.shape)] = -math.inf
                if x.shape[-1] == 0 or not bool((~hidden).any()):
                    continue
                lse[t, j] = torch.logsumexp(x, -1)
                x = torch.exp(x - lse[t, j][..., None])
                out[t, j] = torch.einsum("tgk,kd->tgd", x, values)
                if tally is not None:
                    tally[i, j, at] += x.sum((0, 1))
    got = {"out": out, "lse": lse}
    if tally is not None:
        got["tally"] = tally
    return got


def _exact_evict(s):
    """The rows that stay, found one cache at a time."""
    c = s["case"]
    got = {k: s[k].double() for k in ("tally_out", "K_out", "V_out")}
    for i, have in enumerate(_lengths(c)):
        for j in range(c["n_head"]):
            stay = list(range(have))
            if have > c["keep"]:
                a, b = c["sinks"], have - c["recent"]
                tally = s["tally"][i, j, a:b].cpu().tolist()
                heavy = sorted(range(a, b), key=lambda k: (-tally[k - a], k))[: c["keep"] - a - c["recent"]]
                stay = sorted(heavy + stay[:a] + stay[b:])
            at = torch.tensor(stay, device="cuda")
            for k in ("tally", "K", "V"):
                got[k + "_out"][i, j, : len(stay)] = s[k][i, j, at].double()
    return {"kept": None, "have_out": None, **got}
