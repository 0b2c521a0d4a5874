"""The operators on a key/value cache that is held in 4 bits, as cases that can be timed and compared.

  write    dsmoe_quant_cache_write: tokens' keys and values are quantised into their slots of the cache, and come back as the values that it holds
  read     dsmoe_quant_cache_read: keys and values of whole sequences are read back
  attend   dsmoe_quant_attention: attention of decoding tokens and prompts over the cache, with windows, sinks and rolling caches

A row (sequence, head, position) of the cache has d_head values in groups of 32 neighbours.  A group's scale s is its largest magnitude / 7, rounded up
to four significant bits; its values are s * c with c = x / s rounded to an integer (halves to the even one).  c + 8 is stored in 4 bits: with G =
d_head / 32 groups, 32-bit word t * G + g of a row (t < 4) holds the values 32 g + 8 t and the next seven, the first in the lowest bits.  Scales are bf16, with room for
2, 4 or 8 a row.

Head shapes are those of the attention layer (4 heads of 128 with 5 experts a token, 4 of 96 and 2 of 64 with 6) and generic ones.  A case has
n_seq sequences with n neighbouring tokens each; `least` to 1 is the range, relative to the room there is, over which the sequences' lengths
are spread.
"""
import math

import torch

own = False

GROUP = 32


def _case(op, n_seq, n, n_head, group, d_head, L, *, window=0, sinks=0, rolling=False, by_token=False, idle=0, least=0.5):
    """window 0: none; rolling: the cache keeps its first `sinks` positions and the latest others; by_token: it is stored [n_seq][L][n_head][..];
    idle: that many sequences of the batch are padding."""
    return {"op": op, "n_seq": n_seq, "n": n, "n_head": n_head, "group": group, "d_head": d_head, "L": L, "window": window, "sinks": sinks,
            "rolling": rolling, "by_token": by_token, "idle": idle, "least": least}


def listed():
    named = [
        # a decoding batch's new keys go into rolling caches: what counts is latency
        ("write_tokens", _case("write", 64, 1, 4, 5, 128, 2052, sinks=4, rolling=True, by_token=True, idle=2)),
        # prompts of ragged contexts, the odd head width
        ("write_prompts", _case("write", 3, 1111, 4, 6, 96, 2500)),
        # long prompts
        ("write_long_prompts", _case("write", 4, 8192, 4, 5, 128, 8192, least=1.0)),
        # one conversation's cache is read back
        ("read_one", _case("read", 1, 0, 4, 5, 128, 2048)),
        # a batch of long contexts
        ("read_batch", _case("read", 32, 0, 4, 5, 128, 8192, by_token=True)),
        # one conversation, one token, a rolling cache: latency again
        ("attend_one_token", _case("attend", 1, 1, 4, 5, 128, 516, window=512, sinks=4, rolling=True)),
        # a decoding batch with two padded entries, long contexts of ragged lengths
        ("attend_decode", _case("attend", 64, 1, 4, 5, 128, 8192, by_token=True, idle=2)),
        # many short conversations with small heads
        ("attend_short", _case("attend", 256, 1, 2, 6, 64, 500, least=0.1)),
        # two documents of their own each: few rows, very many keys
        ("attend_long", _case("attend", 2, 1, 8, 4, 128, 131072, least=0.9)),
        # sixteen heads that share their keys, the odd head width, a window over a rolling cache
        ("attend_window", _case("attend", 48, 1, 4, 16, 96, 4100, window=4090, sinks=4, rolling=True)),
        # prompts of ragged contexts, a window that ends inside tiles
        ("attend_prompts", _case("attend", 3, 1111, 4, 6, 96, 2500, window=700, sinks=3)),
        # one long prompt
        ("attend_long_prompt", _case("attend", 1, 8192, 4, 5, 128, 8192, least=1.0)),
    ]
    return [{"name": name, **case} for name, case in named]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """More cases of the same ranges: from one token to thousands, contexts from a few keys to tens of thousands, odd sizes among them."""
    op = rng.choice(["write", "read", "attend", "attend", "attend"])
    n_head, group, d_head = rng.choice([(4, 5, 128), (4, 6, 96), (2, 6, 64), (8, 4, 128), (1, 16, 128), (4, 1, 64), (2, 7, 128), (3, 8, 256)])
    more = {"least": rng.choice([0.1, 0.5, 0.9]), "by_token": rng.random() < 0.4}
    if op == "read":
        L = _log_int(rng, 50, 16000)
        return _case(op, _log_int(rng, 1, max(1, min(64, 200000 // L))), 0, n_head, group, d_head, L, **more)
    prompt = rng.random() < 0.4
    L = _log_int(rng, 50, 4000 if prompt else 20000)
    n = _log_int(rng, 2, L) if prompt else 1
    n_seq = _log_int(rng, 1, max(1, min(256, 4000 // n if prompt else 300000 // L)))
    sinks, rolling = rng.choice([0, 1, 4, 16]), rng.random() < 0.4
    window = _log_int(rng, 8, L) if rolling or rng.random() < 0.4 else 0
    if rolling:                                    # room for the sinks, the window and the tokens of the call
        L = window + sinks + n
    return _case(op, n_seq, n, n_head, group, d_head, L, window=window, sinks=sinks, rolling=rolling, idle=0 if n_seq < 4 else rng.choice([0, 1]), **more)


# ---------------------------------------------------------------- what the cases hold

def _lengths(c):
    """Keys that each sequence has, the call's tokens among them (0: a padded entry); with rolling caches, positions that it has seen."""
    room = 6 * c["L"] if c["rolling"] else c["L"]
    low = max(c["n"], 1, int(c["least"] * room))
    got = [low + int((room - low) * ((i + 1) * 0.6180339887498949 % 1.0)) for i in range(c["n_seq"])]
    if c["least"] == 1.0:
        got = [room] * c["n_seq"]
    return got[:c["n_seq"] - c["idle"]] + [0] * c["idle"]


def _sight(c, last):
    """(first key behind the sinks, number of visible sinks) of a token at position `last`."""
    first = max(0, last - c["window"] + 1) if c["window"] else 0
    return first, min(c["sinks"], first, last + 1)


def _scales(d_head):
    """Places for scales in a row."""
    return 2 if d_head <= 64 else 4 if d_head <= 128 else 8


def work(c):
    n_head, group, d_head = c["n_head"], c["group"], c["d_head"]
    held = d_head // 2 + d_head // GROUP * 2       # bytes of a row of the cache
    if c["op"] == "read":
        return {"bytes": 2 * n_head * sum(_lengths(c)) * (held + 2 * d_head), "flops": 0}
    if c["op"] == "write":
        return {"bytes": 2 * n_head * (c["n_seq"] - c["idle"]) * c["n"] * (held + 4 * d_head), "flops": 0}
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
    return {"bytes": 2 * n_head * keys * held + rows * (d_head * 4 + 4), "flops": 4 * d_head * pairs * n_head * group}


# ---- the format, in elementary operations (what a cache holds is also made with them)

def _quantise(x):
    """x [.., d_head] -> integers c and scales [.., d_head / 32], both fp32.  (A quotient that is a border has to come out as that border: no product with
    a reciprocal, which is what a division by a plain number may be.)"""
    x = x.float().unflatten(-1, (-1, GROUP))
    largest = x.abs().amax(-1)
    raw = (largest / torch.full_like(largest, 7.0)).view(torch.int32)
    scale = ((raw + 0xFFFFF) & ~0xFFFFF).view(torch.float32)          # up to four significant bits
    code = torch.where(scale[..., None] > 0, torch.round(x / scale[..., None]), 0.0)
    return code.flatten(-2), scale


def _pack(code):
    """Integers [.., d_head] -> the bytes of the rows [.., d_head / 2]."""
    u = (code + 8).to(torch.uint8).unflatten(-1, (-1, 4, 4, 2)).transpose(-4, -3)      # [.., t, g, byte, half]
    return (u[..., 0] | (u[..., 1] << 4)).flatten(-3)


def _unpack(held):
    """Bytes of rows [.., d_head / 2] -> integers [.., d_head]."""
    b = held.unflatten(-1, (4, -1, 4))
    return torch.stack((b & 15, b >> 4), -1).transpose(-4, -3).flatten(-4).float() - 8


def _values(code, scale):
    return (code.unflatten(-1, (-1, GROUP)) * scale.float()[..., None]).flatten(-2)


def _held(s, name, of=slice(None)):
    """The values of (sequences of) a cache, fp32."""
    return _values(_unpack(s[name][of]), s[name + "_scale"][of][..., :s["case"]["d_head"] // GROUP])


def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n_seq, n, n_head, group, d_head, L = (c[k] for k in ("n_seq", "n", "n_head", "group", "d_head", "L"))
    # keys have wide channels, the same ones throughout
    gain = torch.exp(0.5 * torch.randn((n_head, d_head), generator=gen, device="cuda"))
    gain = gain / gain.square().mean(-1, keepdim=True).sqrt()

    def rows(*shape, wide):
        x = torch.randn((*shape, n_head, d_head), generator=gen, device="cuda")
        return (x * gain if wide else x).to(torch.bfloat16)

    s = {"case": c, "scale": 1.0 / math.sqrt(d_head)}
    have = _lengths(c)
    s["have"] = torch.tensor(have, dtype=torch.int32).cuda()
    for name in ("K", "V"):
        # (zeros are codes like others; a cache that is written anew need not hold more)
        codes = torch.full((n_seq, L, n_head, d_head // 2), 0x88, dtype=torch.uint8, device="cuda")
        scales = torch.zeros((n_seq, L, n_head, _scales(d_head)), dtype=torch.bfloat16, device="cuda")
        for i in range(n_seq) if c["op"] != "write" else ():
            m = min(have[i], L)
            code, scale = _quantise(rows(m, wide=name == "K"))
            codes[i, :m], scales[i, :m, :, :d_head // GROUP] = _pack(code), scale.to(torch.bfloat16)
        codes, scales = codes.transpose(1, 2), scales.transpose(1, 2)
        s[name], s[name + "_scale"] = (codes, scales) if c["by_token"] else (codes.contiguous(), scales.contiguous())
    if c["op"] == "read":
        s["K_out"], s["V_out"] = (torch.zeros((n_seq, n_head, L, d_head), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    else:
        T = n_seq * n
        s["tok_seq"] = torch.arange(n_seq, dtype=torch.int32, device="cuda").repeat_interleave(n)
        ago = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
        s["pos"] = torch.where(s["have"][:, None] > 0, s["have"][:, None] - 1 - ago, -1).reshape(T).contiguous()
        s["live"] = torch.arange((n_seq - c["idle"]) * n, device="cuda")
    if c["op"] == "write":
        s["k"], s["v"] = rows(T, wide=True), rows(T, wide=False)
        s["k_back"], s["v_back"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    if c["op"] == "attend":
        s["q"] = (2.0 * torch.randn((T, n_head, group, d_head), generator=gen, device="cuda")).to(torch.bfloat16)
        s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros((T, n_head, group), device="cuda")
    if own:
        import paper_2404_05567_b200 as dm
        s["cache"] = dm.make_quant_cache(s["K"], s["V"], s["K_scale"], s["V_scale"])
        if c["op"] == "attend":
            s["desc"] = dm.make_quant_attention_desc(s["q"], s["cache"], s["scale"])
            s["ws"] = torch.empty(dm.dsmoe_quant_attention_workspace_size(s["desc"]), dtype=torch.uint8, device="cuda")
    return s


def _outputs(s):
    names = {"write": ("k_back", "v_back", "K_scale", "V_scale"), "read": ("K_out", "V_out"), "attend": ("out", "lse")}
    return {k: s[k] for k in names[s["case"]["op"]]}


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2404_05567_b200 as dm
    c = s["case"]
    if c["op"] == "write":
        dm.dsmoe_quant_cache_write(s["cache"], s["k"], s["v"], s["tok_seq"], s["pos"], c["sinks"], c["rolling"], s["k_back"], s["v_back"])
    elif c["op"] == "read":
        dm.dsmoe_quant_cache_read(s["cache"], s["have"], s["K_out"], s["V_out"])
    else:
        dm.dsmoe_quant_attention(s["desc"], s["cache"], c["window"] or 2 ** 31 - 1, c["sinks"], c["rolling"], s["q"], s["tok_seq"], s["pos"], s["out"],
                                 s["lse"], s["ws"])
    return _outputs(s)


# ---------------------------------------------------------------- the plain form

def _slot(c, pos):
    ring = c["L"] - c["sinks"]
    return torch.where(pos < c["sinks"], pos, c["sinks"] + (pos - c["sinks"]) % ring) if c["rolling"] else pos


def _plain_write(s):
    c, live = s["case"], s["live"]
    seq, slot = s["tok_seq"][live].long(), _slot(c, s["pos"][live]).long()
    for x, name, back in (("k", "K", "k_back"), ("v", "V", "v_back")):
        code, scale = _quantise(s[x][live])
        s[name][seq, :, slot] = _pack(code)
        s[name + "_scale"][seq, :, slot, :c["d_head"] // GROUP] = scale.to(torch.bfloat16)
        s[back][live] = _values(code, scale).to(torch.bfloat16)
    return _outputs(s)


def _plain_read(s):
    slot = torch.arange(s["case"]["L"], device="cuda")
    real = (slot < s["have"][:, None])[:, None, :, None]
    return {name + "_out": torch.where(real, _held(s, name).to(torch.bfloat16), s[name + "_out"]) for name in ("K", "V")}


def _plain_attend(s):
    c = s["case"]
    n_seq, n, n_head, group, d_head, L = (c[k] for k in ("n_seq", "n", "n_head", "group", "d_head", "L"))
    q = (s["q"].float() * s["scale"]).view(n_seq, n, n_head, group, d_head).permute(0, 2, 1, 3, 4).reshape(n_seq, n_head, n * group, d_head)
    pos = s["pos"].view(n_seq, n, 1)
    slot = torch.arange(L, device="cuda", dtype=torch.int32)
    if c["rolling"]:
        # the position that a slot holds: the latest one up to the sequence's last that lies there
        last = pos.amax(1, keepdim=True)
        key = torch.where(slot < c["sinks"], slot.expand(n_seq, 1, L), last - torch.remainder(last - slot, L - c["sinks"]))
        key = torch.where((slot >= c["sinks"]) & (key < c["sinks"]), -1, key)
    else:
        key = slot.expand(n_seq, 1, L)
    seen = (key >= 0) & (key <= pos)
    if c["window"]:
        seen = seen & ((pos - key < c["window"]) | (key < c["sinks"]))
    seen = seen[:, None, :, None, :].expand(n_seq, 1, n, group, L).reshape(n_seq, 1, n * group, L)
    logits = torch.matmul(q, _held(s, "K").transpose(-1, -2)).masked_fill(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    w = torch.exp(logits - top)
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, _held(s, "V"))
    out = torch.where(total > 0, out / total, torch.zeros_like(out))

    def by_token(x):
        return x.view(n_seq, n_head, n, group, -1).transpose(1, 2).reshape(n_seq * n, n_head, group, -1)

    return {"out": by_token(out).to(torch.bfloat16), "lse": by_token(top + torch.log(total))[..., 0].contiguous()}


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[state["case"]["op"]](state)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_scale(x):
    """Largest magnitude / 7, up to four significant bits."""
    mantissa, exponent = torch.frexp(x.double().unflatten(-1, (-1, GROUP)).abs().amax(-1) / 7)
    return torch.ldexp(torch.ceil(mantissa * 16) / 16, exponent)


def _exact_rows(s, name, i, j, at):
    """Values of one sequence's and head's slots, their nibbles taken one by one."""
    d_head = s["case"]["d_head"]
    G = d_head // GROUP
    held = s[name][i, j, at].long()
    scale = s[name + "_scale"][i, j, at].double()
    got = torch.empty((held.shape[0], d_head), dtype=torch.float64, device="cuda")
    for x in range(d_head):
        g, t, k = x // GROUP, x % GROUP // 8, x % 8
        got[:, x] = ((held[:, 4 * (t * G + g) + k // 2] >> 4 * (k % 2) & 15) - 8) * scale[:, g]
    return got


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "write":
        got = {}
        for x, name in (("k", "K"), ("v", "V")):
            live = s["live"]
            scale = _exact_scale(s[x][live])
            value = s[x][live].double().unflatten(-1, (-1, GROUP))
            back, held = s[x + "_back"].double(), s[name + "_scale"].double()
            back[live] = (torch.round(value / scale[..., None]) * scale[..., None]).flatten(-2)
            held[s["tok_seq"][live].long(), :, _slot(c, s["pos"][live]).long(), :c["d_head"] // GROUP] = scale
            got[x + "_back"], got[name + "_scale"] = back, held
        return got
    if c["op"] == "read":
        got = {name + "_out": torch.zeros(s[name + "_out"].shape, dtype=torch.float64, device="cuda") for name in ("K", "V")}
        for i, have in enumerate(_lengths(c)):
            for j in range(c["n_head"]):
                for name in ("K", "V"):
                    got[name + "_out"][i, j, :have] = _exact_rows(s, name, i, j, slice(0, have))
        return got
    n, n_head, group, d_head = (c[k] for k in ("n", "n_head", "group", "d_head"))
    T = c["n_seq"] * n
    out = torch.zeros((T, n_head, group, d_head), dtype=torch.float64, device="cuda")
    lse = torch.full((T, n_head, group), -math.inf, dtype=torch.float64, device="cuda")
    for i, have in enumerate(_lengths(c)):
        lo = max(0, have - n - c["window"] + 1) if c["window"] else 0        # no token of this sequence sees a key before that, sinks apart
        at = torch.cat((torch.arange(min(c["sinks"], lo)), torch.arange(lo, have))).cuda()
        if len(at) == 0:
            continue
        slot = at
        if c["rolling"]:
            ring = c["L"] - c["sinks"]
            slot = torch.where(at < c["sinks"], at, c["sinks"] + (at - c["sinks"]) % ring)
        for j in range(n_head):
            keys, values = _exact_rows(s, "K", i, j, slot), _exact_rows(s, "V", i, j, slot)
            step = max(1, (1 << 27) // (group * len(keys)))
            for a in range(0, n, step):
                b = min(n, a + step)
                t = slice(i * n + a, i * n + b)
                x = torch.einsum("tgd,kd->tgk", s["q"][t, j].double(), keys) * s["scale"]
                p = torch.arange(have - n + a, have - n + b, device="cuda")
                hidden = at[None, :] > p[:, None]
                if c["window"]:
                    hidden |= (at[None, :] <= p[:, None] - c["window"]) & (at[None, :] >= c["sinks"])
                x[hidden[:, None, :].expand(x.shape)] = -math.inf
                lse[t, j] = torch.logsumexp(x, -1)
                out[t, j] = torch.einsum("tgk,kd->tgd", torch.exp(x - lse[t, j][..., None]), values)
    return {"out": out, "lse": lse}
