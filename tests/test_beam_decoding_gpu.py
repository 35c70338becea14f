"""Beam search over a layer with adapters, as it is served: a prompt a request through packed products with the adapter that the request asks for, linear attention
with its states in a cache, and then token after token: products and adapters, attention, head, the selection of the beams, and the states that follow them.  Each stage
against the definition in 64 bits on what the stage before it left."""
import math

import numpy as np
import pytest
import torch

from oracle import rwkvq_oracle as orc
from paper_2505_03803_b200 import binding as B
from tests import helpers as H
from tests import test_beam_gpu as S
from tests import test_block_gpu as T
from tests import test_linattn_gpu as L
from tests import test_lowrank_gpu as A

pytestmark = pytest.mark.gpu

HEADS, N, VOCAB, RANK, ADAPTERS = 4, 64, 1024, 24, 3
D = HEADS * N


def f64(t):
    return t.double().cpu().numpy()


class Decoder:
    """R, K, V with the token shift, O and the head packed; adapters on R, V and O; a slot of the cache for each beam."""

    def __init__(self, requests, beams, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.requests, self.beams, self.rows = requests, beams, requests * beams
        self.w = [H.pack_sq(H.random_sq_codes(seed, D, D)), H.pack_vq(H.random_vq_codes(seed + 1, D, D, 6), 6), H.pack_sq(H.random_sq_codes(seed + 2, D, D)),
                  H.pack_vq(H.random_vq_codes(seed + 3, D, D, 8), 8)]
        self.head = H.pack_sq(H.random_sq_codes(seed + 4, VOCAB, D))
        self.mu = [H.pack_mu(H.random_mu_codes(seed + 5 + i, D)) for i in range(3)]
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.embedding = (0.3 * r(VOCAB, D)).half()
        self.adapters = {i: (r(ADAPTERS, RANK, D).div(D ** 0.5).half(), (r(ADAPTERS, D, RANK) * 0.1).half()) for i in (0, 2, 3)}
        self.ranks = torch.tensor([24, 8, 17], dtype=torch.int32, device="cuda")
        self.scale = torch.rand(ADAPTERS, generator=g, device="cuda") + 0.5
        self.request_adapter = [i % (ADAPTERS + 1) - 1 for i in range(requests)]
        self.adapter = torch.tensor(self.request_adapter, dtype=torch.int32, device="cuda").repeat_interleave(beams)
        self.logw, self.u = -torch.exp(r(1, HEADS, N) - 2.0), r(HEADS, N)
        slots = self.rows
        self.state = torch.zeros((slots, HEADS, N, N), device="cuda")
        self.xprev = torch.zeros((slots, D), dtype=torch.float16, device="cuda")
        self.parts = B.make_state_parts([self.state, self.xprev])
        self.slots = torch.arange(self.rows, dtype=torch.int32, device="cuda").flip(0).view(requests, beams).contiguous()          # any order
        self.scores = torch.zeros((requests, beams), device="cuda")
        self.next_scores = torch.zeros_like(self.scores)
        self.tokens, self.parents = (torch.zeros((requests, beams), dtype=torch.int32, device="cuda") for _ in range(2))
        self.finished, self.next_finished = (torch.zeros((requests, beams), dtype=torch.uint8, device="cuda") for _ in range(2))
        most = self.rows
        self.x, self.xp = (torch.zeros((most, D), dtype=torch.float16, device="cuda") for _ in range(2))
        self.r, self.k, self.v, self.att = (torch.zeros((most, D), dtype=torch.float16, device="cuda") for _ in range(4))
        self.y, self.y16, self.logits = torch.zeros((most, D), device="cuda"), torch.zeros((most, D), dtype=torch.float16, device="cuda"), torch.zeros((most, VOCAB), device="cuda")
        self.gemv_ws = torch.zeros(max([256] + [B.rwkvq_gemv_workspace_bytes(w.desc, most) for w in self.w + [self.head]]), dtype=torch.uint8, device="cuda")
        self.linattn_ws = torch.full((max(16, B.rwkvq_linattn_workspace_bytes(most, most, HEADS, N)),), 0xFF, dtype=torch.uint8, device="cuda")
        self.select_ws = torch.full((B.rwkvq_beam_select_workspace_bytes(requests, beams, VOCAB, beams),), 0xFF, dtype=torch.uint8, device="cuda")
        self.seq_start = torch.arange(self.rows + 1, dtype=torch.int32, device="cuda")
        self.eos = 7

    def adapt(self, i, x, y, adapter, seq_start=None, x_prev=None, xprev0=None):
        a, b = self.adapters[i]
        mixed = i < 3
        B.rwkvq_lowrank(x, a, b, y, adapter, seq_start=seq_start, ranks=self.ranks, scale=self.scale, x_prev=x_prev, xprev0=xprev0,
                        mu_desc=self.mu[i].desc if mixed else None, mu_image=self.mu[i].dev if mixed else None)

    def prompts(self, prompts):
        """The requests' prompts, one after another in one list of rows; what they leave goes to the first beam's slot of each, and from there to the others'."""
        T, heads = sum(len(p) for p in prompts), lambda t: t.view(-1, HEADS, N)
        starts = torch.tensor(np.concatenate([[0], np.cumsum([len(p) for p in prompts])]), dtype=torch.int32, device="cuda")
        x = self.embedding[torch.cat(prompts)].bfloat16()
        r, k, v, att = (torch.empty((T, D), dtype=torch.bfloat16, device="cuda") for _ in range(4))
        adapter = torch.tensor(self.request_adapter, dtype=torch.int32, device="cuda")
        x_prev = torch.cat([torch.zeros_like(x[:1]), x[:-1]])
        x_prev[starts[:-1].long()] = 0
        ones = []
        for i, y in enumerate((r, k, v)):
            for a, b in zip(starts.tolist(), starts.tolist()[1:]):
                ws = torch.empty(max(16, B.rwkvq_prefill_workspace_bytes(self.w[i].desc, b - a, True)), dtype=torch.uint8, device="cuda")
                B.rwkvq_gemm_prefill(self.w[i].desc, self.w[i].dev, self.mu[i].desc, self.mu[i].dev, x[a:b], None, b - a, y[a:b], ws)
            ones.append(y.clone())
            if i in self.adapters:
                self.adapt(i, x, y, adapter, seq_start=starts)
        first = self.slots[:, 0].contiguous()
        ws = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(T, len(prompts), HEADS, N)), dtype=torch.uint8, device="cuda")
        B.rwkvq_linattn(heads(r), heads(k), heads(v), self.logw.expand(T, HEADS, N), self.u, heads(att), self.state, seq_start=starts, slots=first, workspace=ws)
        self.xprev[first.long()] = x[starts[1:].long() - 1].half()
        B.rwkvq_state_reorder(self.parts, torch.zeros_like(self.parents), slots=self.slots)
        self.scores.fill_(-math.inf)
        self.scores[:, 0] = 0.0
        self.tokens.copy_(torch.tensor([[int(p[-1])] * self.beams for p in prompts], dtype=torch.int32))
        self.finished.zero_()
        return x, x_prev, ones, (r, k, v), att, starts

    def step(self, keep=None):
        """A token of every beam.  keep: a list for what the products leave before the adapters add to it."""
        at = self.slots.view(-1).long()
        self.x.copy_(self.embedding[self.tokens.view(-1).long()])
        self.xp.copy_(self.xprev[at])
        for i, y in enumerate((self.r, self.k, self.v)):
            B.rwkvq_gemv(self.w[i].desc, self.w[i].dev, self.mu[i].desc, self.mu[i].dev, self.x, self.xp, self.rows, y, self.gemv_ws)
            if keep is not None:
                keep.append(y.clone())
            if i in self.adapters:
                self.adapt(i, self.x, y, self.adapter, x_prev=self.xp)
        self.xprev[at] = self.x
        heads = lambda t: t.view(-1, HEADS, N)
        B.rwkvq_linattn(heads(self.r), heads(self.k), heads(self.v), self.logw.expand(self.rows, HEADS, N), self.u, heads(self.att), self.state, seq_start=self.seq_start,
                        slots=self.slots.view(-1), workspace=self.linattn_ws)
        B.rwkvq_gemv(self.w[3].desc, self.w[3].dev, None, None, self.att, None, self.rows, self.y, self.gemv_ws)
        if keep is not None:
            keep += [self.y.clone(), self.state.clone(), self.xprev.clone()]
        self.adapt(3, self.att, self.y, self.adapter)
        self.y16.copy_(self.y)
        B.rwkvq_gemv(self.head.desc, self.head.dev, None, None, self.y16, None, self.rows, self.logits, self.gemv_ws)
        B.rwkvq_beam_select(self.logits, self.scores, self.next_scores, self.parents, self.tokens, finished=self.finished, eos=self.eos, finished_out=self.next_finished,
                            workspace=self.select_ws)
        B.rwkvq_state_reorder(self.parts, self.parents, slots=self.slots)
        self.scores.copy_(self.next_scores)
        self.finished.copy_(self.next_finished)

    def check_product(self, w, x64, out, rounding):
        ref, tol = orc.gemv(w.w_hat, x64), orc.tolerance(w.w_hat, x64)
        assert (np.abs(f64(out) - ref) <= tol + rounding * np.abs(ref) + 2.0 ** -25).all()        # fp16 has subnormals half a step of which is 2^-25

    def check_adapter(self, i, lens, adapter, x, x_prev, before, after, x_type, y_type):
        c = object.__new__(A.Case)
        c.lens, c.ic, c.oc, c.rank, c.xt, c.wt, c.yt, c.front, c.adapter = lens, D, D, RANK, x_type, "f16", y_type, 0, adapter
        c.x, c.x_prev, c.xprev0, c.y, c.ranks, c.scale = x.cpu(), None if x_prev is None else x_prev.cpu(), None, before.cpu(), self.ranks.cpu(), self.scale.cpu()
        c.A, c.B, c.mu = self.adapters[i][0].cpu(), self.adapters[i][1].cpu(), None if x_prev is None else self.mu[i]
        ref, tol = c.expected()
        assert ((after.double().cpu() - ref).abs() <= tol).all()

    def check_attention(self, rkv, before, after, out, lens, slots, dtype):
        T = rkv[0].shape[0]
        c = dict(rkv=torch.stack(rkv, 1).view(T, 3, HEADS, N).cpu(), lw=self.logw.cpu(), u=self.u.cpu(), slots=slots.cpu(), state=before.cpu(), dtype=dtype, lens=lens,
                 starts=np.concatenate([[0], np.cumsum(lens)]).tolist())
        ref, tol, state, state_tol = L.expected(c)
        L.near(out.view(T, HEADS, N), ref, tol, "attention")
        L.near(after, state, state_tol, "states")


def prompts_of(requests, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(0, VOCAB, (n,), generator=g, device="cuda") for n in [1, 40, 75, 3, 17, 2][:requests]]


@pytest.mark.parametrize("requests,beams", [(1, 4), (4, 2), (3, 5), (5, 1)])
def test_prompts_then_beams(requests, beams):
    m = Decoder(requests, beams, 60 + requests)
    prompts = prompts_of(requests, 1)
    x, x_prev, ones, rkv, att, starts = m.prompts(prompts)
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    lens, prev = [len(p) for p in prompts], f64(x_prev)
    for i in range(3):
        m.check_product(m.w[i], orc.token_shift(f64(x), prev, m.mu[i].w_hat), ones[i], A.HALF_ULP["bf16"])
        if i in m.adapters:
            m.check_adapter(i, lens, m.request_adapter, x, x_prev, ones[i], rkv[i], "bf16", "bf16")
        else:
            assert torch.equal(ones[i], rkv[i])
    where = m.slots.long()
    for b in range(beams):          # every beam of a request begins with what its prompt left
        assert torch.equal(m.state[where[:, b]], m.state[where[:, 0]]) and torch.equal(m.xprev[where[:, b]], x[starts[1:].long() - 1].half())
    after = torch.zeros_like(m.state)
    after[where[:, 0]] = m.state[where[:, 0]]
    m.check_attention(rkv, torch.zeros_like(m.state), after, att, lens, m.slots[:, 0], "bf16")
    row_adapter = m.adapter.tolist()
    for step in range(4):
        before, scores, tokens, finished, xp, keep = m.state.clone(), m.scores.clone(), m.tokens.clone(), m.finished.clone(), m.xprev[m.slots.view(-1).long()], []
        if step == 2:
            finished[:, 0] = 1          # a beam that has ended keeps its place by its score alone
            m.finished.copy_(finished)
        m.step(keep)
        torch.cuda.synchronize()
        assert B.rwkvq_device_status() == 0
        x64 = f64(m.embedding[tokens.view(-1).long()])
        assert np.array_equal(f64(m.x), x64) and torch.equal(m.xp, xp)
        for i, y in enumerate((m.r, m.k, m.v)):
            m.check_product(m.w[i], orc.token_shift(x64, f64(xp), m.mu[i].w_hat), keep[i], A.HALF_ULP["f16"])
            if i in m.adapters:
                m.check_adapter(i, [1] * m.rows, row_adapter, m.x, xp, keep[i], y, "f16", "f16")
        m.check_attention((m.r, m.k, m.v), before, keep[4], m.att, [1] * m.rows, m.slots.view(-1), "f16")
        m.check_product(m.w[3], f64(m.att), keep[3], A.HALF_ULP["f32"])
        m.check_adapter(3, [1] * m.rows, row_adapter, m.att, None, keep[3], m.y, "f16", "f32")
        m.check_product(m.head, f64(m.y16), m.logits, A.HALF_ULP["f32"])
        ref = S.totals(m.logits.cpu(), scores.cpu(), finished.cpu(), m.eos)
        best, _ = S.order(ref, m.logits.cpu(), VOCAB)
        got = torch.gather(ref, 1, (m.parents.long() * VOCAB + m.tokens.long()).cpu())
        fin = torch.isfinite(got)
        assert torch.equal(fin, torch.isfinite(best[:, :beams])) and ((got - best[:, :beams]).abs()[fin] <= 2 * S.LSE).all()
        assert ((m.scores.double().cpu() - got).abs()[fin] <= S.LSE + 2.0 ** -23 * got[fin].abs()).all()
        assert torch.equal(m.finished != 0, (torch.gather(finished, 1, m.parents.long()) != 0) | (m.tokens == m.eos))
        follow = torch.gather(m.slots, 1, m.parents.long()).view(-1).long()
        assert torch.equal(m.state[m.slots.view(-1).long()], keep[4][follow]) and torch.equal(m.xprev[m.slots.view(-1).long()], keep[5][follow])


def outcome(m):
    return [t.clone() for t in (m.state, m.xprev, m.scores, m.tokens, m.parents, m.finished, m.logits)]


def test_a_captured_step_replayed():
    m = Decoder(3, 4, 80)
    m.prompts(prompts_of(3, 2))
    m.step()
    start = outcome(m)
    eager = []
    for _ in range(3):
        m.step()
        eager.append(outcome(m))
    back = lambda: [t.copy_(s) for t, s in zip((m.state, m.xprev, m.scores, m.tokens, m.parents, m.finished, m.logits), start)]
    back()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step()
    back()
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outcome(m), want))
    assert B.rwkvq_device_status() == 0


def test_two_searches_on_two_streams():
    searches = [Decoder(2, 4, 90), Decoder(4, 3, 91)]
    alone = []
    for m in searches:
        m.prompts(prompts_of(m.requests, 3))
        start = outcome(m)
        for _ in range(5):
            m.step()
        torch.cuda.synchronize()
        alone.append(outcome(m))
        for t, s in zip((m.state, m.xprev, m.scores, m.tokens, m.parents, m.finished, m.logits), start):
            t.copy_(s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in searches]
    for _ in range(5):
        for m, s in zip(searches, streams):
            with torch.cuda.stream(s):
                m.step()
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    for m, want in zip(searches, alone):
        assert all(torch.equal(a, b) for a, b in zip(outcome(m), want))


def test_blocks_follow_their_beams():
    """A chain of whole blocks: a batch whose sequences took over others' states goes on as these do."""
    from paper_2505_03803_b200 import stack as stack_mod
    m = stack_mod.BlockStack(512, 1792, 2, 64, 6, tag="beams", kmeans_iters=2)
    m.set_token(1)
    m.run_step_host()
    m.set_token(2)
    m.run_step_host()
    torch.cuda.synchronize()
    parents = torch.tensor([[2, 0, 0], [0, 2, 1]], dtype=torch.int32, device="cuda")
    rows = torch.tensor([2, 0, 0, 3, 5, 4], device="cuda")
    kept = [(st[k], st[k].clone()) for st in m.states for k in "abp"] + [(o.xprev, o.xprev.clone()) for o in m.ops if o.xprev is not None]
    assert any(not torch.equal(was[0], was[2]) for _, was in kept)
    m.follow(parents)
    torch.cuda.synchronize()
    assert all(torch.equal(now, was[rows]) for now, was in kept)
    by = {(o.layer, o.name): o for o in m.ops}
    token, prev, (a0, b0, p0) = m.x0_host.clone().numpy().astype(np.float64), f64(by[(0, "R")].xprev), (f64(m.states[0][k]) for k in "abp")
    m.run_step_host()
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    # the next token's products read what the parents left: the token shift, and the WKV history in front of O
    w_hat, mu_hat = T._decode(m, by[(0, "R")])
    T._check_product("R", type("M", (), {"w_hat": w_hat}), orc.token_shift(token, prev, mu_hat), by[(0, "R")].y)
    w_hat, _ = T._decode(m, by[(0, "O")])
    wkv, _, _ = orc.wkv_step(a0 * np.exp(p0), b0 * np.exp(p0), f64(by[(0, "K")].y), f64(by[(0, "V")].y), f64(m.states[0]["u"]), f64(m.states[0]["w"]))
    T._check_product("O", type("M", (), {"w_hat": w_hat}), T._f16(orc.time_mix_gate(f64(by[(0, "R")].y), wkv)), by[(0, "O")].y)
    with pytest.raises(ValueError):
        m.follow(parents[:1])
