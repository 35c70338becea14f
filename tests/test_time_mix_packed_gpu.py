"""Linear attention between packed products: R, K, V of a prompt or of a batch of tokens from 3-bit codes and codebooks (with the token shift), the recurrence with its states in a
cache, O from a packed matrix or, its input quantized, from one of 8 bits.  Each stage against the definition in 64 bits on what the stage before it left."""
import numpy as np
import pytest
import torch

from oracle import rwkvq_oracle as orc
from paper_2505_03803_b200 import binding as B
from tests import helpers as H
from tests import test_fp8_gpu as F
from tests import test_linattn_gpu as L

pytestmark = pytest.mark.gpu

HEADS, N = 8, 64
D = HEADS * N


def f64(t):
    return t.double().cpu().numpy()


class Layer:
    def __init__(self, slots, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.w = [H.pack_sq(H.random_sq_codes(seed, D, D)), H.pack_vq(H.random_vq_codes(seed + 1, D, D, 6), 6), H.pack_sq(H.random_sq_codes(seed + 2, D, D)),
                  H.pack_vq(H.random_vq_codes(seed + 3, D, D, 8), 8)]
        self.mu = [H.pack_mu(H.random_mu_codes(seed + 4 + i, D)) for i in range(3)]
        w8 = (torch.randn((D, D), generator=g, device="cuda") / D ** 0.5).half()
        self.o8 = torch.empty((D, D), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((D // 128, B.rwkvq_fp8_scale_pitch(D)), dtype=torch.uint8, device="cuda")
        B.rwkvq_fp8_quantize(w8, *self.o8, 128)
        self.logw = -torch.exp(torch.randn((1, HEADS, N), generator=g, device="cuda") - 2.0)
        self.u = torch.randn((HEADS, N), generator=g, device="cuda")
        self.state = torch.zeros((slots, HEADS, N, N), device="cuda")

    def prompt(self, x, xprev0, shift, seq_start=None, slots=None):
        """x [T, D] bf16: (r, k, v, attention, O packed, codes and scales of the attention, O in 8 bits)."""
        T = x.shape[0]
        r, k, v, att = (torch.empty((T, D), dtype=torch.bfloat16, device="cuda") for _ in range(4))
        ws = [torch.empty(max(16, B.rwkvq_prefill_workspace_bytes(w.desc, T, shift)), dtype=torch.uint8, device="cuda") for w in self.w]
        B.rwkvq_gemm_prefill_grouped([dict(desc=w.desc, W=w.dev, mu_desc=m.desc if shift else None, mu=m.dev if shift else None, X=x, xprev0=xprev0, Y=y, workspace=b)
                                      for w, m, y, b in zip(self.w, self.mu, (r, k, v), ws)], T, B.RWKVQ_BF16)
        self.recurrence(r, k, v, att, seq_start, slots)
        y, y8 = torch.empty((T, D), device="cuda"), torch.empty((T, D), device="cuda")
        w = self.w[3]
        B.rwkvq_gemm_prefill(w.desc, w.dev, None, None, att, None, T, y, ws[3])
        return (r, k, v, att, y) + self.eight_bits(att, y8)

    def tokens(self, x, xprev, shift, slots=None):
        """One token of each of x's sequences, x [T, D] fp16."""
        T = x.shape[0]
        r, k, v, att = (torch.empty((T, D), dtype=torch.float16, device="cuda") for _ in range(4))
        y, y8 = torch.empty((T, D), device="cuda"), torch.empty((T, D), device="cuda")
        ws = [torch.zeros(max(256, B.rwkvq_gemv_workspace_bytes(w.desc, T)), dtype=torch.uint8, device="cuda") for w in self.w]
        for w, m, to, b in zip(self.w, self.mu, (r, k, v), ws):
            B.rwkvq_gemv(w.desc, w.dev, m.desc if shift else None, m.dev if shift else None, x, xprev if shift else None, T, to, b)
        self.recurrence(r, k, v, att, torch.arange(T + 1, dtype=torch.int32, device="cuda") if T > 1 else None, slots)
        B.rwkvq_gemv(self.w[3].desc, self.w[3].dev, None, None, att, None, T, y, ws[3])
        return (r, k, v, att, y) + self.eight_bits(att, y8)

    def recurrence(self, r, k, v, att, seq_start, slots):
        T, n_seq = r.shape[0], 1 if seq_start is None else seq_start.numel() - 1
        ws = torch.full((max(16, B.rwkvq_linattn_workspace_bytes(T, n_seq, HEADS, N)),), 0xFF, dtype=torch.uint8, device="cuda")
        heads = lambda t: t.view(T, HEADS, N)
        B.rwkvq_linattn(heads(r), heads(k), heads(v), self.logw.expand(T, HEADS, N), self.u, heads(att), self.state, seq_start=seq_start, slots=slots, workspace=ws)

    def eight_bits(self, att, y8):
        codes, scale = torch.empty(att.shape, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros((att.shape[0], B.rwkvq_fp8_scale_pitch(D)), dtype=torch.uint8, device="cuda")
        B.rwkvq_fp8_quantize(att, codes, scale, 1)
        B.rwkvq_gemm_fp8(*self.o8, codes, scale, y8)
        torch.cuda.synchronize()
        assert B.rwkvq_device_status() == 0
        return codes, scale, y8

    def check(self, got, x, prev, shift, dtype, lens, slots, before):
        r, k, v, att, y, codes, scale, y8 = got
        half = L.HALF_ULP[dtype]

        def product(w, x64, out, rounding):
            ref, tol = orc.gemv(w.w_hat, x64), orc.tolerance(w.w_hat, x64)
            err = np.abs(f64(out) - ref)
            # fp16 has subnormals half a step of which is 2^-25
            assert (err <= tol + rounding * np.abs(ref) + 2.0 ** -25).all(), np.max(err / tol)

        x64 = f64(x)
        for w, m, out in zip(self.w, self.mu, (r, k, v)):
            product(w, orc.token_shift(x64, prev, m.w_hat) if shift else x64, out, half)
        T = x.shape[0]
        c = dict(rkv=torch.stack([r, k, v], 1).view(T, 3, HEADS, N).cpu(), lw=self.logw.cpu(), u=self.u.cpu(), slots=slots, state=before.cpu(), dtype=dtype, lens=lens,
                 starts=np.concatenate([[0], np.cumsum(lens)]).tolist())
        ref, tol, S, tolS = L.expected(c)
        L.near(att.view(T, HEADS, N), ref, tol, "attention")
        L.near(self.state, S, tolS, "states")
        product(self.w[3], f64(att), y, L.HALF_ULP["f32"])
        ref_codes, ref_scale = F.quantize_exact(f64(att), 1)
        codes, scale = codes.view(torch.uint8).cpu().numpy(), scale.cpu().numpy()
        assert np.array_equal(codes, ref_codes) and np.array_equal(scale[:, :ref_scale.shape[1]], ref_scale)       # all eight bits, the signs too
        w8, s8 = (t.view(torch.uint8).cpu().numpy() for t in self.o8)
        F.check_product(y8, "f32", w8, s8, codes, scale)


def activations(T, seed, dtype=torch.bfloat16):
    return (0.3 * torch.randn((T, D), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")).to(dtype)


def test_a_prompt_with_the_token_shift_then_its_tokens():
    m = Layer(slots=1, seed=1)
    x, first = activations(75, 2), activations(1, 3)
    before = m.state.clone()
    got = m.prompt(x, first.view(-1), True)
    m.check(got, x, np.concatenate([f64(first), f64(x)[:-1]]), True, "bf16", [75], None, before)
    last = x[-1:].half()
    for step in range(3):
        before, x = m.state.clone(), activations(1, 10 + step, torch.float16)
        m.check(m.tokens(x, last, True), x, f64(last), True, "f16", [1], None, before)
        last = x


def test_a_batch_of_prompts_then_their_tokens():
    m = Layer(slots=6, seed=20)
    lens, slots = [40, 1, 0, 67, 3], torch.tensor([5, 0, 3, 1, 4], dtype=torch.int32)
    x, before = activations(sum(lens), 21), m.state.clone()
    starts = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    m.check(m.prompt(x, None, False, starts, slots.cuda()), x, None, False, "bf16", lens, slots, before)
    for step, order in enumerate(([5, 0, 3, 1, 4], [4, 1, 5])):
        slots, before, x = torch.tensor(order, dtype=torch.int32), m.state.clone(), activations(len(order), 30 + step, torch.float16)
        m.check(m.tokens(x, None, False, slots.cuda()), x, None, False, "f16", [1] * len(order), slots, before)


@pytest.mark.parametrize("T", [1, 130])
def test_captured_and_replayed(T):
    m = Layer(slots=1, seed=40)
    x = activations(T, 41)
    want = [t.clone() for t in m.prompt(x, None, False)]
    state = m.state.clone()
    r, k, v, att = (torch.empty((T, D), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    ws = [torch.empty(max(16, B.rwkvq_prefill_workspace_bytes(w.desc, T, False)), dtype=torch.uint8, device="cuda") for w in m.w[:3]]
    lw = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(T, 1, HEADS, N)), dtype=torch.uint8, device="cuda")
    codes, scale, y8 = (torch.zeros_like(t) for t in want[5:])
    heads = lambda t: t.view(T, HEADS, N)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for w, y, b in zip(m.w, (r, k, v), ws):
            B.rwkvq_gemm_prefill(w.desc, w.dev, None, None, x, None, T, y, b)
        B.rwkvq_linattn(heads(r), heads(k), heads(v), m.logw.expand(T, HEADS, N), m.u, heads(att), m.state, workspace=lw)
        B.rwkvq_fp8_quantize(att, codes, scale, 1)
        B.rwkvq_gemm_fp8(*m.o8, codes, scale, y8)
    for _ in range(3):
        m.state.zero_()
        for t in (r, k, v, att, y8):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((r, k, v, att, y8), (*want[:4], want[7])):
            assert torch.equal(a, b)
        assert torch.equal(m.state, state)
    assert B.rwkvq_device_status() == 0
