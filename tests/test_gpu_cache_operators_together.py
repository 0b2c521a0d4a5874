"""The operators on a key/value cache as a server uses them together (GPU required): a prompt whose keys are tallied, its cache thinned out in place, then
tokens one by one, each of which is stored, attends and tallies, with evictions whenever a cache is full; and the same caches under a window and behind
a shared prefix, all calls with one workspace."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import attention, evict, logit_error, lse_tolerance, out_tolerance, tally_tolerance, visible

pytestmark = pytest.mark.gpu

SINKS, RECENT, WINDOW = 2, 10, 21


def bf16(rng, *shape, by=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * by).astype(np.float32)).to(torch.bfloat16).cuda()


def plain(x):
    return x.float().cpu().numpy().astype(np.float64)


class Server:
    """Sequences with a cache of L slots each, a tally of its keys, their lengths on the device, and P keys that they all share."""

    def __init__(self, n_seq, n_head, group, d, L, prompt, P, seed):
        rng = np.random.default_rng(seed)
        self.n_seq, self.n_head, self.group, self.d, self.L, self.P, self.scale = n_seq, n_head, group, d, L, P, d ** -0.5
        self.K, self.V = bf16(rng, n_seq, n_head, L, d), bf16(rng, n_seq, n_head, L, d)
        self.Kp, self.Vp = bf16(rng, n_head, P, d), bf16(rng, n_head, P, d)
        self.tally = torch.zeros((n_seq, n_head, L), device="cuda")
        self.length = torch.full((n_seq,), prompt, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.seqs = torch.arange(n_seq, dtype=torch.int32, device="cuda")
        # a prompt's tokens and the next ones' inputs
        self.prompt_q = bf16(rng, n_seq * prompt, n_head, group, d, by=2.0)
        self.prompt_seq = self.seqs.repeat_interleave(prompt)
        self.prompt_pos = torch.arange(prompt, dtype=torch.int32, device="cuda").repeat(n_seq)
        self.q, self.k, self.v = bf16(rng, n_seq, n_head, group, d, by=2.0), bf16(rng, n_seq, n_head, 1, d), bf16(rng, n_seq, n_head, 1, d)
        self.outs = [torch.zeros_like(self.q) for _ in range(3)]
        self.lses = [torch.zeros((n_seq, n_head, group), device="cuda") for _ in range(3)]
        self.prompt_out = torch.zeros_like(self.prompt_q)
        self.prompt_lse = torch.zeros((n_seq * prompt, n_head, group), device="cuda")
        self.kept = torch.zeros((n_seq, n_head, 2 * L // 3), dtype=torch.int32, device="cuda")
        many, one = (dm.make_attention_desc(q, self.K, self.scale, out) for q, out in ((self.prompt_q, self.prompt_out), (self.q, self.outs[0])))
        cache = dm.make_attention_desc(None, self.K)
        self.many, self.one, self.cache = many, one, cache
        size = max(dm.dsmoe_attention_workspace_size(many, dm.ATTENTION_TALLY), dm.dsmoe_attention_workspace_size(one, dm.ATTENTION_TALLY),
                   dm.dsmoe_attention_workspace_size(one, dm.ATTENTION_WINDOW), dm.dsmoe_attention_workspace_size(one, dm.ATTENTION_PREFIX, P),
                   dm.dsmoe_evict_workspace_size(cache))
        self.ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def take_prompt(self):
        dm.dsmoe_tally_attention(self.many, self.prompt_q, self.K, self.V, self.prompt_seq, self.prompt_pos, self.prompt_out, self.prompt_lse, None,
                                 self.tally, self.ws, self.status)

    def thin_out(self):
        keep = self.kept.shape[2]
        dm.dsmoe_cache_evict(self.cache, keep, SINKS, RECENT, self.length, self.tally, self.K, self.V, self.kept, self.length, self.tally, self.K, self.V,
                             self.ws, self.status)

    def step(self):
        """A token each: it is stored, attends to all, tallies; to its window; to the shared keys and all of its own."""
        at = self.length.long()[:, None, None]
        place = at[..., None].expand(self.n_seq, self.n_head, 1, self.d)
        self.K.scatter_(2, place, self.k)
        self.V.scatter_(2, place, self.v)
        self.tally.scatter_(2, at.expand(self.n_seq, self.n_head, 1), 0.0)
        dm.dsmoe_tally_attention(self.one, self.q, self.K, self.V, self.seqs, self.length, self.outs[0], self.lses[0], self.tally, self.tally, self.ws,
                                 self.status)
        dm.dsmoe_window_attention(self.one, WINDOW, SINKS, False, self.q, self.K, self.V, self.seqs, self.length, self.outs[1], self.lses[1], self.ws,
                                  self.status)
        dm.dsmoe_prefix_attention(self.one, self.Kp, self.Vp, self.q, self.K, self.V, self.seqs, self.length, self.outs[2], self.lses[2], self.ws,
                                  self.status)
        self.length += 1

    def state(self):
        return [x.clone() for x in (self.K, self.V, self.tally, self.length, self.kept, *self.outs, *self.lses)]

    def restore(self, state):
        for x, y in zip((self.K, self.V, self.tally, self.length, self.kept, *self.outs, *self.lses), state):
            x.copy_(y)


def check(s, q, out, lse, tokens, tally=None, tally_in=None, window=None, prefix=False):
    """Against the plain form, on the cache as it is."""
    K, V, q_np, got, got_lse = plain(s.K), plain(s.V), plain(q), plain(out), plain(lse)
    Kp, Vp = plain(s.Kp), plain(s.Vp)
    added, error, rows = np.zeros((s.n_seq, s.n_head, s.L)), np.zeros((s.n_seq, s.n_head, s.L)), np.zeros((s.n_seq, 1, 1))
    for t, (seq, pos) in enumerate(tokens):
        seen = np.array(visible(pos, window, SINKS if window else 0), dtype=int)
        rows[seq] += s.group
        for j in range(s.n_head):
            k, v, at = K[seq, j], V[seq, j], seen
            if prefix:
                k, v, at = np.concatenate((Kp[j], k)), np.concatenate((Vp[j], v)), np.concatenate((np.arange(s.P), s.P + seen))
            o, x, w, absolute, spread = attention(q_np[t, j], k, v, s.scale, at)
            assert (np.abs(got[t, j] - o) <= out_tolerance(o, absolute, spread, s.d)).all()
            assert (np.abs(got_lse[t, j] - x) <= lse_tolerance(x, spread, s.d)).all()
            if tally is not None:
                np.add.at(added[seq, j], at, w.sum(0))
                np.add.at(error[seq, j], at, (w * (np.expm1(2 * logit_error(spread, s.d)) + 2.0 ** -20)[:, None]).sum(0))
    if tally is not None:
        before = plain(tally_in)
        assert (np.abs(plain(tally) - before - added) <= tally_tolerance(before, added, error, rows)).all()


def check_eviction(s, before):
    """before: K, V, tally, length as they were.  What stays is exact, given the tallies."""
    K, V, tally, length = before[:4]
    keep = s.kept.shape[2]
    for q in range(s.n_seq):
        n = length[q].item()
        assert s.length[q].item() == min(n, keep)
        for j in range(s.n_head):
            stay = evict(tally[q, j].cpu().numpy(), n, keep, SINKS, RECENT)
            assert s.kept[q, j].tolist() == stay + [-1] * (keep - len(stay))
            at = torch.tensor(stay, device="cuda")
            for now, was in ((s.K, K), (s.V, V), (s.tally, tally)):
                assert torch.equal(now[q, j, :len(stay)], was[q, j][at])


# (group and prompt: prompts on the streaming kernel, and on the 128-row one; heads that share keys and ones that do not)
@pytest.mark.parametrize("n_seq,n_head,group,d,L,prompt,P", [(2, 2, 3, 64, 96, 90, 150), (3, 1, 8, 128, 150, 140, 300), (2, 3, 1, 32, 60, 60, 40),
                                                              (12, 1, 5, 96, 75, 74, 130)])
def test_a_prompt_and_the_tokens_after_it(n_seq, n_head, group, d, L, prompt, P):
    s = Server(n_seq, n_head, group, d, L, prompt, P, seed=L)
    s.take_prompt()
    tokens = list(zip(s.prompt_seq.tolist(), s.prompt_pos.tolist()))
    check(s, s.prompt_q, s.prompt_out, s.prompt_lse, tokens, s.tally, torch.zeros_like(s.tally))
    before = s.state()
    s.thin_out()
    check_eviction(s, before)
    begin = s.state()
    steps = 2 * (L - s.kept.shape[2]) + 3                # the caches fill up twice
    for i in range(steps):
        rng = np.random.default_rng(1000 + i)
        for x, by in ((s.q, 2.0), (s.k, 1.0), (s.v, 1.0)):
            x.copy_(bf16(rng, *x.shape, by=by))
        before = s.state()
        s.step()
        tally_in = before[2].scatter(2, before[3].long()[:, None, None].expand(n_seq, n_head, 1), 0.0)
        now = list(enumerate(before[3].tolist()))
        check(s, s.q, s.outs[0], s.lses[0], now, s.tally, tally_in)
        check(s, s.q, s.outs[1], s.lses[1], now, window=WINDOW)
        check(s, s.q, s.outs[2], s.lses[2], now, prefix=True)
        if s.length.max().item() == L:
            before = s.state()
            s.thin_out()
            check_eviction(s, before)
    assert s.status.item() == 0
    # the same steps as two graphs, one of them with the eviction
    want = s.state()
    s.restore(begin)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        s.step()
    with torch.cuda.graph(graphs[1]):
        s.step()
        s.thin_out()
    s.restore(begin)
    n = begin[3].max().item()
    for i in range(steps):
        rng = np.random.default_rng(1000 + i)
        for x, by in ((s.q, 2.0), (s.k, 1.0), (s.v, 1.0)):
            x.copy_(bf16(rng, *x.shape, by=by))
        n += 1
        graphs[n == L].replay()
        if n == L:
            n = s.kept.shape[2]
    torch.cuda.synchronize()
    for x, y in zip(s.state(), want):
        assert torch.equal(x, y)


def test_two_servers_at_once():
    """Two streams, each with its own caches and workspace and no wait between them, do what they do one after the other."""
    sizes = ((2, 2, 3, 64, 300, 280, 500), (5, 2, 8, 128, 420, 401, 900))
    states = []
    for at_once in (False, True):
        servers = [Server(*x, seed=i) for i, x in enumerate(sizes)]
        streams = [torch.cuda.Stream() if at_once else torch.cuda.current_stream() for _ in servers]
        torch.cuda.synchronize()
        for turn in range(12):
            for s, stream in zip(servers, streams):
                with torch.cuda.stream(stream):
                    if turn == 0:
                        s.take_prompt()
                        s.thin_out()
                    s.step()
                    if turn % 5 == 4:
                        s.thin_out()
        torch.cuda.synchronize()
        assert all(s.status.item() == 0 for s in servers)
        states.append([x for s in servers for x in s.state() + [s.prompt_out, s.prompt_lse]])
    for x, y in zip(*states):
        assert torch.equal(x, y)
