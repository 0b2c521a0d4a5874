"""The operators on a cache in 4 bits as a server uses them together (GPU required): a prompt is written and attended to, then tokens one by one, which are written
and attend; with a cache of all positions and a rolling one, eagerly and as a captured graph, all calls with one workspace; and two servers on two
streams at once."""
import numpy as np
import pytest
import torch

import paper_2404_05567_b200 as dm
from cache_attention_reference import attention, lse_tolerance, visible
from quant_cache_reference import GROUP, quant_logit_error, quant_out_tolerance, quantise, scales_of, slot_of, taken_as_prompts, unpack, values

pytestmark = pytest.mark.gpu

WINDOW, SINKS = 33, 2


def bf16(rng, *shape, by=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * by).astype(np.float32)).to(torch.bfloat16).cuda()


def plain(x):
    return x.double().cpu().numpy()


class Server:
    """n_seq sequences, whose prompts have `prompt` tokens each; caches of L slots, with a window and rolling if `rolling`."""

    def __init__(self, n_seq, n_head, group, d, L, prompt, steps, rolling, seed):
        rng = np.random.default_rng(seed)
        self.n_seq, self.n_head, self.group, self.d, self.L, self.prompt, self.scale = n_seq, n_head, group, d, L, prompt, d ** -0.5
        self.window, self.sinks, self.rolling = (WINDOW, SINKS, True) if rolling else (2 ** 31 - 1, 0, False)
        held = [torch.zeros((n_seq, L, n_head, w), dtype=t, device="cuda").transpose(1, 2)
                for w, t in ((d // 2, torch.uint8), (d // 2, torch.uint8), (scales_of(d), torch.bfloat16), (scales_of(d), torch.bfloat16))]
        self.cache = dm.make_quant_cache(*held)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.seqs = torch.arange(n_seq, dtype=torch.int32, device="cuda")
        self.prompt_seq, self.prompt_pos = self.seqs.repeat_interleave(prompt), torch.arange(prompt, dtype=torch.int32, device="cuda").repeat(n_seq)
        T = n_seq * prompt
        self.prompt_q, self.prompt_k, self.prompt_v = bf16(rng, T, n_head, group, d, by=2.0), bf16(rng, T, n_head, d), bf16(rng, T, n_head, d)
        self.steps_q = bf16(rng, steps, n_seq, n_head, group, d, by=2.0)
        self.steps_kv = bf16(rng, steps, n_seq, 2, n_head, d)
        self.q, self.kv = torch.empty_like(self.steps_q[0]), torch.empty_like(self.steps_kv[0])
        self.pos = torch.full((n_seq,), prompt, dtype=torch.int32, device="cuda")
        self.prompt_out, self.out = torch.zeros_like(self.prompt_q), torch.zeros_like(self.q)
        self.prompt_lse, self.lse = (torch.zeros((n, n_head, group), device="cuda") for n in (T, n_seq))
        self.many = dm.make_quant_attention_desc(self.prompt_q, self.cache, self.scale)
        self.one = dm.make_quant_attention_desc(self.q, self.cache, self.scale)
        self.ws = torch.empty(max(dm.dsmoe_quant_attention_workspace_size(d) for d in (self.many, self.one)), dtype=torch.uint8, device="cuda")

    def take_prompt(self):
        dm.dsmoe_quant_cache_write(self.cache, self.prompt_k, self.prompt_v, self.prompt_seq, self.prompt_pos, self.sinks, self.rolling, dev_status=self.status)
        dm.dsmoe_quant_attention(self.many, self.cache, self.window, self.sinks, self.rolling, self.prompt_q, self.prompt_seq, self.prompt_pos, self.prompt_out,
                                 self.prompt_lse, self.ws, self.status)

    def step(self):
        """A token each: its key and value, slices of one tensor, are written, then it attends."""
        dm.dsmoe_quant_cache_write(self.cache, self.kv[:, 0], self.kv[:, 1], self.seqs, self.pos, self.sinks, self.rolling, dev_status=self.status)
        dm.dsmoe_quant_attention(self.one, self.cache, self.window, self.sinks, self.rolling, self.q, self.seqs, self.pos, self.out, self.lse, self.ws, self.status)
        self.pos += 1

    def feed(self, i):
        self.q.copy_(self.steps_q[i])
        self.kv.copy_(self.steps_kv[i])

    # ---- what it should be
    def rows(self, steps):
        """Keys' and values' rows by position as they are held, [n_seq, positions, n_head, d], and the scales."""
        got = []
        for i, x in enumerate((self.prompt_k, self.prompt_v)):
            x = np.concatenate((plain(x).reshape(self.n_seq, self.prompt, self.n_head, self.d), plain(self.steps_kv[:steps, :, i]).transpose(1, 0, 2, 3)), 1)
            code, scale = quantise(x)
            got += [values(code, scale), scale]
        return got

    def check(self, rows, q, out, lse, tokens, prompt):
        K, Ks, V, Vs = rows
        q, got, got_lse = plain(q), plain(out), plain(lse)
        for t, (s, p) in enumerate(tokens):
            at = np.array(visible(p, None if self.window > self.L else self.window, self.sinks), dtype=int)
            for j in range(self.n_head):
                o, x, _, absolute, spread = attention(q[t, j], K[s, :, j], V[s, :, j], self.scale, at)
                error = quant_logit_error(q[t, j], self.scale, Ks[s, :, j][at], spread, self.d)
                assert (np.abs(got[t, j] - o) <= quant_out_tolerance(o, absolute, error, prompt, len(at), Vs[s, :, j][at].max())).all()
                assert (np.abs(got_lse[t, j] - x) <= error + lse_tolerance(x, spread, self.d)).all()

    def check_cache(self, rows, last):
        """Slots hold the latest positions that go there."""
        for codes, scales, v, sc in ((self.cache.tensors[0], self.cache.tensors[2], rows[0], rows[1]), (self.cache.tensors[1], self.cache.tensors[3], rows[2], rows[3])):
            held = values(unpack(codes.cpu().numpy()), plain(scales)[..., : self.d // GROUP])
            for p in range(last + 1):
                slot = slot_of(p, self.L, self.sinks, self.rolling)
                if not any(slot_of(x, self.L, self.sinks, self.rolling) == slot for x in range(p + 1, last + 1)):
                    assert np.array_equal(held[:, :, slot], v[:, p])


@pytest.mark.parametrize("rolling", [False, True])
@pytest.mark.parametrize("n_head,group,d", [(4, 5, 128), (2, 6, 64), (3, 12, 96), (2, 3, 160)])
def test_prompt_then_tokens(n_head, group, d, rolling):
    n_seq, prompt, steps = 3, 150, 40
    s = Server(n_seq, n_head, group, d, WINDOW + SINKS + prompt if rolling else 256, prompt, steps, rolling, seed=d + group)
    as_prompts = taken_as_prompts(n_seq * prompt, n_seq, n_head, group, s.L, d, s.scale)
    assert as_prompts == (n_head > 2)
    rows = s.rows(steps)
    s.take_prompt()
    s.check(rows, s.prompt_q, s.prompt_out, s.prompt_lse, [(i, p) for i in range(n_seq) for p in range(prompt)], as_prompts)
    s.check_cache(rows, prompt - 1)
    s.feed(0)
    s.step()
    s.check(rows, s.q, s.out, s.lse, [(i, prompt) for i in range(n_seq)], False)
    # the rest as a graph
    s.feed(1)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.step()
    for i in range(1, steps):
        s.feed(i)
        graph.replay()
        if i in (1, steps // 2, steps - 1):
            s.check(rows, s.q, s.out, s.lse, [(k, prompt + i) for k in range(n_seq)], False)
    s.check_cache(rows, prompt + steps - 1)
    assert s.status.item() == 0


def test_two_servers_on_two_streams():
    """... each of which gets what it gets alone."""
    def make():
        return [Server(3, 4, 5, 128, 1300, 1200, 6, False, seed=1), Server(40, 2, 9, 64, 105, 70, 6, True, seed=2)]

    def run(servers, streams):
        outs = [[], []]
        for s, x in zip(servers, streams):
            with torch.cuda.stream(x):
                s.take_prompt()
        for i in range(6):
            for s, x, o in zip(servers, streams, outs):
                with torch.cuda.stream(x):
                    s.feed(i)
                    s.step()
                    o += [s.out.clone(), s.lse.clone()]
        torch.cuda.synchronize()
        return outs + [[s.prompt_out for s in servers]]
    one = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = run(make(), (one, one))
    torch.cuda.synchronize()
    servers = make()
    torch.cuda.synchronize()
    got = run(servers, (torch.cuda.Stream(), torch.cuda.Stream()))
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
