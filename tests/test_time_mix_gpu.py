"""The operators around the recurrence as a time-mix layer runs them: activations to 8 bits, R, K and V products side by side into one buffer, linear
attention with its state in a cache, its outputs to 8 bits, O product.  Each stage against the definition in 64 bits on what the stage before it left."""
import numpy as np
import pytest
import torch

from paper_2505_03803_b200 import binding as B
from tests import test_fp8_gpu as F
from tests import test_linattn_gpu as L

pytestmark = pytest.mark.gpu


class TimeMix:
    """Weights in 8 bits, decays, a cache of states; buffers for up to `most` rows."""

    def __init__(self, heads, slots, most, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.n, self.d, self.most = heads, 64, heads * 64, most
        d, pitch = self.d, B.rwkvq_fp8_scale_pitch(heads * 64)
        self.codes, self.scales = [], []
        for _ in range(4):
            w = (torch.randn((d, d), generator=g, device="cuda") / d ** 0.5).half()
            self.codes.append(torch.empty((d, d), dtype=torch.float8_e4m3fn, device="cuda"))
            self.scales.append(torch.empty(((d + 127) // 128, pitch), dtype=torch.uint8, device="cuda"))
            B.rwkvq_fp8_quantize(w, self.codes[-1], self.scales[-1], 128)
        self.logw = -torch.exp(torch.randn((heads, 64), generator=g, device="cuda") - 2.0)
        self.u = torch.randn((heads, 64), generator=g, device="cuda")
        self.state = torch.zeros((slots, heads, 64, 64), device="cuda")
        self.x_codes, self.x_scale = torch.empty((most, d), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((most, pitch), dtype=torch.uint8, device="cuda")
        self.a_codes, self.a_scale = torch.empty_like(self.x_codes), torch.empty_like(self.x_scale)
        self.rkv = torch.empty((most, 3, heads, 64), dtype=torch.bfloat16, device="cuda")
        self.att = torch.empty((most, heads, 64), dtype=torch.bfloat16, device="cuda")
        self.y = torch.empty((most, d), device="cuda")
        self.workspace = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(most, slots, heads, 64)), dtype=torch.uint8, device="cuda")

    def run(self, x, seq_start=None, slots=None):
        T, H, n = x.shape[0], self.heads, self.n
        xc, xs, ac, as_, rkv, att, y = (t[:T] for t in (self.x_codes, self.x_scale, self.a_codes, self.a_scale, self.rkv, self.att, self.y))
        B.rwkvq_fp8_quantize(x, xc, xs, 1)
        for i in range(3):
            B.rwkvq_gemm_fp8(self.codes[i], self.scales[i], xc, xs, rkv[:, i].reshape(T, self.d) if T == 1 else rkv.view(T, 3 * self.d)[:, i * self.d:(i + 1) * self.d])
        B.rwkvq_linattn(rkv[:, 0], rkv[:, 1], rkv[:, 2], self.logw.unsqueeze(0).expand(T, H, n), self.u, att, self.state, seq_start=seq_start, slots=slots,
                        workspace=self.workspace)
        B.rwkvq_fp8_quantize(att.view(T, self.d), ac, as_, 1)
        B.rwkvq_gemm_fp8(self.codes[3], self.scales[3], ac, as_, y)
        return y

    def check(self, x, lens, slots, before):
        """The stages of the run just made, whose states were `before`."""
        T = x.shape[0]
        host = lambda t: t.view(torch.uint8).cpu().numpy() if t.element_size() == 1 else t.double().cpu()
        codes, scale = F.quantize_exact(host(x).numpy(), 1)
        assert np.array_equal(host(self.x_codes[:T]), codes) and np.array_equal(host(self.x_scale[:T])[:, :scale.shape[1]], scale)
        for i in range(3):
            F.check_product(self.rkv[:T, i].reshape(T, self.d), "bf16", host(self.codes[i]), host(self.scales[i]), host(self.x_codes[:T]), host(self.x_scale[:T]))
        c = dict(rkv=self.rkv[:T].cpu(), lw=self.logw.cpu().unsqueeze(0), u=self.u.cpu(), slots=slots, state=before.cpu(), dtype="bf16", lens=lens,
                 starts=np.concatenate([[0], np.cumsum(lens)]).tolist())
        ref, tol, S, tolS = L.expected(c)
        L.near(self.att[:T], ref, tol, "attention")
        L.near(self.state, S, tolS, "states")
        codes, scale = F.quantize_exact(host(self.att[:T].view(T, self.d)).numpy(), 1)
        assert np.array_equal(host(self.a_codes[:T]) & 127, codes & 127)
        F.check_product(self.y[:T], "f32", host(self.codes[3]), host(self.scales[3]), host(self.a_codes[:T]), host(self.a_scale[:T]))


def activations(T, d, seed):
    return torch.randn((T, d), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def test_a_prompt_then_its_tokens():
    m = TimeMix(heads=3, slots=1, most=90, seed=1)
    for step, T in enumerate([90, 1, 1, 1]):
        before = m.state.clone()
        x = activations(T, m.d, 10 + step)
        m.run(x)
        torch.cuda.synchronize()
        assert B.rwkvq_device_status() == 0
        m.check(x, [T], None, before)


def test_a_serving_batch_of_prompts_and_tokens():
    m = TimeMix(heads=2, slots=9, most=200, seed=2)
    for step, (lens, slots) in enumerate([([100, 1, 0, 33, 1], [3, 0, 8, 5, 1]), ([1, 1, 1, 1, 1], [5, 3, 8, 1, 0]), ([17, 1, 150], [2, 3, 4])]):
        before, T = m.state.clone(), sum(lens)
        x = activations(T, m.d, 20 + step)
        seq_start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
        slots = torch.tensor(slots, dtype=torch.int32)
        m.run(x, seq_start, slots.cuda())
        torch.cuda.synchronize()
        assert B.rwkvq_device_status() == 0
        m.check(x, lens, slots, before)


@pytest.mark.parametrize("T", [1, 100])
def test_captured_and_replayed(T):
    m = TimeMix(heads=3, slots=1, most=T, seed=3)
    x = activations(T, m.d, 30)
    m.run(x)
    first, state = m.y[:T].clone(), m.state.clone()
    graph = torch.cuda.CUDAGraph()
    m.state.zero_()
    with torch.cuda.graph(graph):
        m.run(x)
    m.state.zero_()
    m.y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(m.y[:T], first) and torch.equal(m.state, state)
    graph.replay()                        # goes on from the state that it left
    torch.cuda.synchronize()
    assert not torch.equal(m.state, state) and torch.isfinite(m.y).all()


def test_two_layers_on_two_streams():
    # each with its own buffers: nothing of a call is kept in the library for another to meet
    layers = [TimeMix(heads=2, slots=1, most=120, seed=s) for s in (4, 5)]
    xs = [activations(120, m.d, 40 + i) for i, m in enumerate(layers)]
    alone = []
    for m, x in zip(layers, xs):
        m.run(x)
        torch.cuda.synchronize()
        alone.append((m.y.clone(), m.state.clone()))
        m.state.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for m, x, s in zip(layers, xs, streams):
            with torch.cuda.stream(s):
                m.state.zero_()
                m.run(x)
    torch.cuda.synchronize()
    for m, (y, state) in zip(layers, alone):
        assert torch.equal(m.y, y) and torch.equal(m.state, state)
