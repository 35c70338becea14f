"""The operators around the packed projections as cases that can be timed and compared: linear attention with
decaying state (prompts, ragged batches, single tokens), the 8-bit floating-point quantizer and the product of
its codes.

A case is a dict of plain values; `op` names the operator.  `listed()` holds the named cases, `draw(rng)` makes one
more of the same ranges, `prepare(case, seed)` builds what a program has in hand before the call, `run(state)` is
one pass: the framework's entry points where `own` is true, their plain form in elementary torch operations where
it is not.  `exact(case, seed)` gives the definition in 64 bits, `work(case)` what a pass cannot do without.

  linattn       out_t = r_t (S + (u k_t) v_t^T), S <- diag(exp(lw_t)) S + k_t v_t^T, per sequence and head
  fp8_quantize  codes of 8 bits with one power-of-two scale per group of 128 columns of one row, or of 128 rows
  fp8_product   Y = X W^T of such codes
"""
from __future__ import annotations

import math
import random

import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def listed():
    return [
        # Decoding one sequence, the 1.6B-class width: one token, 32 heads of 64.  All latency.
        dict(name="linattn_token_b1", op="linattn", seqs=1, tokens=1, heads=32, n=64, dtype="f16", decay="channel", decay_f32=True, static=False,
             bonus=True, slots=0),
        # A serving batch of 96 sequences, one token each, their states scattered over a cache of 128 slots; 7B-class width.
        dict(name="linattn_token_b96", op="linattn", seqs=96, tokens=96, heads=64, n=64, dtype="bf16", decay="channel", decay_f32=True, static=False,
             bonus=True, slots=128),
        # A short prompt of odd length, 1.6B-class width, decays in the activations' type.
        dict(name="linattn_prompt_203", op="linattn", seqs=1, tokens=203, heads=32, n=64, dtype="bf16", decay="channel", decay_f32=False, static=False,
             bonus=True, slots=0),
        # A long prompt, 7B-class width.
        dict(name="linattn_prompt_2048", op="linattn", seqs=1, tokens=2048, heads=64, n=64, dtype="bf16", decay="channel", decay_f32=True, static=False,
             bonus=True, slots=0),
        # A ragged batch: prompts of very different lengths, single tokens and empty sequences among them, one decay per head.
        dict(name="linattn_ragged", op="linattn", seqs=11, tokens=5000, heads=64, n=64, dtype="f16", decay="head", decay_f32=True, static=False,
             bonus=True, slots=16),
        # 32-bit activations, heads of 128, the same decays for all tokens, no bonus.
        dict(name="linattn_prompt_f32", op="linattn", seqs=1, tokens=1111, heads=16, n=128, dtype="f32", decay="channel", decay_f32=True, static=True,
             bonus=False, slots=0),
        # The activations of a prompt in front of an 8-bit product.
        dict(name="fp8_rows_2048", op="fp8_quantize", rows=2048, cols=4096, block=1, dtype="bf16"),
        # The largest matrix of a 7B-class layer converted to 8 bits.
        dict(name="fp8_blocks_14336", op="fp8_quantize", rows=14336, cols=4096, block=128, dtype="f16"),
        # One token through a d x d projection: all latency and weight bytes.
        dict(name="fp8_product_m1", op="fp8_product", tokens=1, oc=4096, ic=4096, out="f32"),
        # A small decode batch through the channel-mix value projection.
        dict(name="fp8_product_m13", op="fp8_product", tokens=13, oc=4096, ic=14336, out="f16"),
        # A short prompt of odd length, 1.6B-class channel-mix key.
        dict(name="fp8_product_m203", op="fp8_product", tokens=203, oc=7168, ic=2048, out="bf16"),
        # A long prompt, 7B-class channel-mix key.
        dict(name="fp8_product_m2048", op="fp8_product", tokens=2048, oc=14336, ic=4096, out="bf16"),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    op = rng.choice(["linattn", "linattn", "linattn", "fp8_quantize", "fp8_product", "fp8_product"])
    if op == "linattn":
        n = rng.choice([64, 64, 64, 128])
        heads = _log(rng, 1, 64) if n == 64 else _log(rng, 1, 32)
        seqs = rng.choice([1, 1, _log(rng, 1, 128)])
        tokens = rng.choice([seqs, _log(rng, 1, 5000)])
        return dict(op=op, seqs=seqs, tokens=tokens, heads=heads, n=n, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    decay=rng.choice(["channel", "channel", "head"]), decay_f32=rng.random() < 0.6, static=rng.random() < 0.2,
                    bonus=rng.random() < 0.8, slots=rng.choice([0, seqs + rng.randint(0, 20)]))
    if op == "fp8_quantize":
        return dict(op=op, rows=_log(rng, 1, 8192), cols=_log(rng, 128, 7168, 16), block=rng.choice([1, 128]), dtype=rng.choice(["bf16", "f16", "f32"]))
    return dict(op=op, tokens=rng.choice([_log(rng, 1, 32), _log(rng, 1, 2048)]), oc=_log(rng, 64, 14336, rng.choice([1, 64])),
                ic=_log(rng, 128, 4096, 16), out=rng.choice(["f32", "bf16", "f16"]))


# ---- inputs -------------------------------------------------------------------------------------------------
def lengths(case):
    """Sequence lengths of a case (a property of the case, not of the seed): all one where tokens == seqs, otherwise very uneven, some zero."""
    seqs, tokens = case["seqs"], case["tokens"]
    if seqs == 1:
        return [tokens]
    if tokens == seqs:
        return [1] * seqs
    rng = random.Random(f"{seqs} {tokens}")
    share = [0.0 if rng.random() < 0.1 else math.exp(rng.uniform(0.0, 4.0)) for _ in range(seqs)]
    share[0] = max(share[0], 1.0)
    out = [int(tokens * s / sum(share)) for s in share]
    out[0] += tokens - sum(out)
    return out


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _groups(cols):
    return (cols + 127) // 128


def _pitch(cols):
    """Bytes of a row of scales: one byte per group of 128 columns, a multiple of 16."""
    return (_groups(cols) + 15) // 16 * 16


def _activations(g, rows, cols, dtype):
    """N(0, 1) with eight outlier channels twenty times as large."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    at = torch.randperm(cols, generator=g, device="cuda")[:8]
    x[:, at] *= 20.0
    return x.to(TORCH[dtype])


def _weights(g, rows, cols, dtype):
    """N(0, 0.02), some rows heavier."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    x *= 0.02 * torch.exp(0.5 * torch.randn((rows, 1), generator=g, device="cuda"))
    return x.to(TORCH[dtype])


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=case)
    if case["op"] == "linattn":
        T, H, n, dt = case["tokens"], case["heads"], case["n"], TORCH[case["dtype"]]
        # r, k, v as the products leave them: side by side in one buffer
        rkv = torch.randn((T, 3, H, n), generator=g, device="cuda").to(dt)
        st["r"], st["k"], st["v"] = rkv[:, 0], rkv[:, 1], rkv[:, 2]
        rows = 1 if case["static"] else T
        shape = (rows, H, n) if case["decay"] == "channel" else (rows, H)
        # decays exp(-exp(z)): from channels that remember thousands of tokens to some that forget at once
        lw = -torch.exp(torch.randn(shape, generator=g, device="cuda") * 1.5 - 2.5)
        lw = torch.where(torch.rand(shape, generator=g, device="cuda") < 0.002, torch.full_like(lw, -math.inf), lw)
        st["logw"] = (lw if case["decay_f32"] else lw.to(dt)).expand(T, *shape[1:])
        st["u"] = torch.randn((H, n), generator=g, device="cuda") * 0.5 if case["bonus"] else None
        lens = lengths(case)
        starts = [0]
        for l in lens:
            starts.append(starts[-1] + l)
        st["starts"] = starts
        st["seq_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        n_slots = case["slots"] or case["seqs"]
        st["slots"] = torch.randperm(n_slots, generator=g, device="cuda")[:case["seqs"]].to(torch.int32) if case["slots"] else None
        st["state"] = torch.randn((n_slots, H, n, n), generator=g, device="cuda")
        st["state_out"] = st["state"].clone()
        if own:
            from paper_2505_03803_b200 import binding as B
            st["out"] = torch.empty((T, H, n), dtype=dt, device="cuda")
            st["workspace"] = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(T, case["seqs"], H, n)), dtype=torch.uint8, device="cuda")
        return st
    if case["op"] == "fp8_quantize":
        make = _activations if case["block"] == 1 else _weights
        st["x"] = make(g, case["rows"], case["cols"], case["dtype"])
        if own:
            st["codes"] = torch.empty((case["rows"], case["cols"]), dtype=torch.float8_e4m3fn, device="cuda")
            rows = case["rows"] if case["block"] == 1 else (case["rows"] + 127) // 128
            st["scale"] = torch.empty((rows, _pitch(case["cols"])), dtype=torch.uint8, device="cuda")
        return st
    st["w_codes"], st["w_scale"] = _quantize_plain(_weights(g, case["oc"], case["ic"], "f16"), 128)
    st["x_codes"], st["x_scale"] = _quantize_plain(_activations(g, case["tokens"], case["ic"], "bf16"), 1)
    if own:
        st["y"] = torch.empty((case["tokens"], case["oc"]), dtype=TORCH[case["out"]], device="cuda")
    return st


# ---- one pass -----------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    if case["op"] == "linattn":
        return _linattn_plain(case, st)
    if case["op"] == "fp8_quantize":
        codes, scale = _quantize_plain(st["x"], case["block"])
        return {"codes": codes, "scale": scale[:, :_groups(case["cols"])]}
    y = _values(st["x_codes"], st["x_scale"], 1) @ _values(st["w_codes"], st["w_scale"], 128).T
    return {"y": y.to(TORCH[case["out"]])}


def _run_own(case, st):
    from paper_2505_03803_b200 import binding as B
    if case["op"] == "linattn":
        one = case["seqs"] == 1
        B.rwkvq_linattn(st["r"], st["k"], st["v"], st["logw"], st["u"], st["out"], st["state"], state_out=st["state_out"],
                        seq_start=None if one else st["seq_start"], slots=st["slots"], workspace=st["workspace"])
        return {"out": st["out"], "state": st["state_out"]}
    if case["op"] == "fp8_quantize":
        B.rwkvq_fp8_quantize(st["x"], st["codes"], st["scale"], case["block"])
        return {"codes": st["codes"], "scale": st["scale"][:, :_groups(case["cols"])]}
    B.rwkvq_gemm_fp8(st["w_codes"], st["w_scale"], st["x_codes"], st["x_scale"], st["y"])
    return {"y": st["y"]}


def _linattn_plain(case, st):
    """The recurrence, one token of every sequence after the other, in 32 bits."""
    lens = [b - a for a, b in zip(st["starts"], st["starts"][1:])]
    T, H, n, dt = case["tokens"], case["heads"], case["n"], TORCH[case["dtype"]]
    slot = st["slots"].long() if st["slots"] is not None else torch.arange(case["seqs"], device="cuda")
    u = st["u"] if st["u"] is not None else torch.ones((H, n), device="cuda")
    r, k, v = st["r"].float(), st["k"].float(), st["v"].float()
    w = torch.exp(st["logw"].float())
    if case["decay"] == "head":
        w = w.unsqueeze(-1).expand(T, H, n)
    out = torch.empty((T, H, n), device="cuda")
    S = st["state"][slot]
    # longest first, so that the sequences still running are the first ones
    order = sorted(range(case["seqs"]), key=lambda i: -lens[i])
    S = S[torch.tensor(order, device="cuda")]
    first = torch.tensor([st["starts"][i] for i in order], device="cuda")
    for t in range(max(lens)):
        m = sum(1 for i in order if lens[i] > t) if len(order) > 1 else 1
        at = first[:m] + t if m > 1 else slice(st["starts"][order[0]] + t, st["starts"][order[0]] + t + 1)
        rt, kt, vt, wt = r[at], k[at], v[at], w[at]
        Sm = S[:m]
        out[at] = torch.einsum("mhi,mhij->mhj", rt, Sm) + (rt * u * kt).sum(-1, keepdim=True) * vt
        S[:m] = wt.unsqueeze(-1) * Sm + kt.unsqueeze(-1) * vt.unsqueeze(-2)
    st["state_out"][slot[torch.tensor(order, device="cuda")]] = S
    return {"out": out.to(dt), "state": st["state_out"]}


def _quantize_plain(x, block):
    """(codes, scales): per group the smallest power of two by which the largest magnitude comes to at most 448 = 1.75 * 2^8."""
    rows, cols = x.shape
    G = _groups(cols)
    f = torch.zeros(((rows + block - 1) // block * block, G * 128), device="cuda")
    f[:rows, :cols] = x.float()
    f = f.view(-1, block, G, 128)
    a = f.abs().amax(dim=(1, 3))
    m, e = torch.frexp(a)                     # a = m * 2^e, 0.5 <= m < 1
    e = torch.where(m > 0.875, e - 8, e - 9)
    e = torch.where(a > 0, e, torch.zeros_like(e)).clamp(-126, 127)
    codes = torch.ldexp(f, -e.view(-1, 1, G, 1)).view(-1, G * 128)[:rows, :cols].to(torch.float8_e4m3fn).contiguous()
    scale = torch.full((f.shape[0], _pitch(cols)), 127, dtype=torch.uint8, device="cuda")
    scale[:, :G] = (e + 127).to(torch.uint8)
    return codes, scale


def _values(codes, scale, block):
    """What codes and scales stand for, in 32 bits (exact)."""
    rows, cols = codes.shape
    s = torch.exp2(scale[:, :_groups(cols)].float() - 127.0)
    s = s.repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return codes.float() * s


# ---- the definition in 64 bits ------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "linattn":
        return _linattn_exact(case, st)
    if case["op"] == "fp8_quantize":
        # the numbers that the codes round; the scales are whole numbers
        x = st["x"].double()
        rows, cols = x.shape
        v = torch.empty_like(x)
        b = case["block"]
        for r0 in range(0, rows, max(b, 1024 // b * b)):
            r1 = min(rows, r0 + max(b, 1024 // b * b))
            for c0 in range(0, cols, 128):
                part = x[r0:r1, c0:c0 + 128]
                top = part.abs().amax(1) if b == 1 else torch.stack([p.abs().max() for p in part.split(b)]).repeat_interleave(b)[:r1 - r0]
                e = torch.ceil(torch.log2(top / 448.0)).nan_to_num(neginf=0.0).clamp(-126, 127)
                e = e + (top > 448.0 * 2.0 ** e).double() - ((e > -126) & (top > 0) & (top <= 448.0 * 2.0 ** (e - 1))).double()
                v[r0:r1, c0:c0 + 128] = part / (2.0 ** e).unsqueeze(1)
        return {"codes": v, "scale": None}
    x = st["x_codes"].double()
    w = st["w_codes"].double()
    y = torch.zeros((case["tokens"], case["oc"]), dtype=torch.float64, device="cuda")
    for g in range(_groups(case["ic"])):
        c = slice(128 * g, 128 * g + 128)
        sx = 2.0 ** (st["x_scale"][:, g].double() - 127.0)
        sw = (2.0 ** (st["w_scale"][:, g].double() - 127.0)).repeat_interleave(128)[:case["oc"]]
        y += (x[:, c] @ w[:, c].T) * sx.unsqueeze(1) * sw.unsqueeze(0)
    return {"y": y}


def _linattn_exact(case, st):
    """Pieces of 32 tokens: what each token sees of the state in front of the piece and of the tokens before it in the piece, by the sums of the logarithms."""
    T, H, n = case["tokens"], case["heads"], case["n"]
    state = st["state_out"].double()
    u = st["u"].double() if st["u"] is not None else torch.ones((H, n), dtype=torch.float64, device="cuda")
    out = torch.empty((T, H, n), dtype=torch.float64, device="cuda")
    slot = st["slots"].tolist() if st["slots"] is not None else list(range(case["seqs"]))
    for q, (a, b) in enumerate(zip(st["starts"], st["starts"][1:])):
        S = st["state"][slot[q]].double()
        for t0 in range(a, b, 32):
            t1 = min(b, t0 + 32)
            C = t1 - t0
            r, k, v = (st[x][t0:t1].double() for x in "rkv")
            lw = st["logw"][t0:t1].double().clamp(min=-1e5)
            lw = lw.unsqueeze(-1).expand(C, H, n) if case["decay"] == "head" else lw
            L = torch.zeros((C + 1, H, n), dtype=torch.float64, device="cuda")
            L[1:] = torch.cumsum(lw, 0)                                        # L[t]: all decays before token t
            seen = torch.exp((L[:C].unsqueeze(1) - L[1:].unsqueeze(0)).clamp(max=0.0))      # [t][s]: decays between s and t
            A = torch.einsum("thi,tshi,shi->tsh", r, seen, k) * torch.ones((C, C), device="cuda").tril(-1).unsqueeze(-1)
            A[range(C), range(C)] = (r * u * k).sum(-1)
            out[t0:t1] = torch.einsum("thi,hij->thj", r * torch.exp(L[:C]), S) + torch.einsum("tsh,shj->thj", A, v)
            S = torch.exp(L[C]).unsqueeze(-1) * S + torch.einsum("shi,shj->hij", k * torch.exp(L[C] - L[1:]), v)
        state[slot[q]] = S
    return {"out": out, "state": state}


# ---- what a pass cannot do without --------------------------------------------------------------------------
def work(case):
    if case["op"] == "linattn":
        T, H, n, es = case["tokens"], case["heads"], case["n"], SIZE[case["dtype"]]
        ws = 4 if case["decay_f32"] else es
        decays = (1 if case["static"] else T) * H * (n if case["decay"] == "channel" else 1)
        live = sum(1 for l in lengths(case) if l)
        return {"bytes": 4 * T * H * n * es + decays * ws + 8 * live * H * n * n + (4 * H * n if case["bonus"] else 0),
                "flops": T * H * (4 * n * n + 6 * n)}
    if case["op"] == "fp8_quantize":
        rows, cols = case["rows"], case["cols"]
        groups = ((rows + case["block"] - 1) // case["block"]) * _groups(cols)
        return {"bytes": rows * cols * (SIZE[case["dtype"]] + 1) + groups, "flops": 2 * rows * cols}
    M, oc, ic = case["tokens"], case["oc"], case["ic"]
    return {"bytes": oc * ic + M * ic + M * oc * SIZE[case["out"]] + (M + (oc + 127) // 128) * _groups(ic), "flops": 2 * M * oc * ic}
