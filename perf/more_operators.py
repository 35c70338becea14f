"""What a decode step of many requests needs beside the packed products, as cases that can be timed and compared: low-rank adapters, beam search's
selection, and the states that follow their beams.

A case is a dict of plain values; `op` names the operator.  `listed()` holds the named cases, `draw(rng)` makes one more of the same ranges,
`prepare(case, seed)` builds what a program has in hand before the call, `run(state)` is one pass: the framework's entry points where `own` is true,
their plain form in elementary torch operations where it is not.  `exact(case, seed)` gives the definition in 64 bits, `work(case)` what a pass cannot
do without.

  lowrank   y_t += s_a B_a (A_a x_t), a the adapter of t's sequence; x_t mixed with the token before it where the projection's input is
  select    the largest of score_k + log softmax(logits_k)_v over beams k and tokens v of a request; ties go to the lowest (k, v)
  reorder   state[slot of beam b] = state[slot of b's parent], all layers, in place
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
        # Decoding one sequence, 1.6B-class width, one small adapter, token shift in front.  All latency.
        dict(name="lowrank_token_b1", op="lowrank", seqs=1, tokens=1, ic=2048, oc=2048, rank=16, ragged_ranks=False, adapters=4, free=0.0, x="f16", w="f16", y="f32", mix=True),
        # A serving batch of 96 sequences, one token each, 7B-class width, 64 adapters of very different ranks in memory, some sequences without one.
        dict(name="lowrank_token_b96", op="lowrank", seqs=96, tokens=96, ic=4096, oc=4096, rank=64, ragged_ranks=True, adapters=64, free=0.1, x="f16", w="bf16", y="f32", mix=True),
        # A serving batch that shares three adapters, channel-mix key.
        dict(name="lowrank_token_shared", op="lowrank", seqs=48, tokens=48, ic=4096, oc=14336, rank=32, ragged_ranks=False, adapters=3, free=0.0, x="bf16", w="bf16", y="bf16", mix=False),
        # A short prompt of odd length, 1.6B-class channel-mix key.
        dict(name="lowrank_prompt_203", op="lowrank", seqs=1, tokens=203, ic=2048, oc=7168, rank=32, ragged_ranks=False, adapters=2, free=0.0, x="bf16", w="bf16", y="f32", mix=True),
        # A long prompt, 7B-class d x d projection.
        dict(name="lowrank_prompt_2048", op="lowrank", seqs=1, tokens=2048, ic=4096, oc=4096, rank=64, ragged_ranks=False, adapters=2, free=0.0, x="bf16", w="bf16", y="bf16", mix=False),
        # Prompts of very different lengths, single tokens and empty sequences among them, odd ranks up to 128.
        dict(name="lowrank_ragged", op="lowrank", seqs=11, tokens=3001, ic=4096, oc=4096, rank=128, ragged_ranks=True, adapters=8, free=0.1, x="f16", w="f16", y="f32", mix=True),
        # One request of four beams, its first step (all beams the same, one alive), logits as the head's product leaves them.
        dict(name="select_b1", op="select", requests=1, beams=4, vocab=65536, picks=4, dtype="f32", first=True, done=0.0, kept=1.0, pad=0),
        # A serving batch, twice as many candidates as beams, some beams finished.
        dict(name="select_b32", op="select", requests=32, beams=8, vocab=65536, picks=16, dtype="bf16", first=False, done=0.1, kept=1.0, pad=0),
        # An odd vocabulary in rows of another length, a grammar that leaves few tokens.
        dict(name="select_odd", op="select", requests=7, beams=5, vocab=50277, picks=5, dtype="f16", first=False, done=0.0, kept=0.001, pad=3),
        # Four beams of one request, 1.6B-class: matrix states and two token-shift rows in each of 24 layers.
        dict(name="reorder_b1", op="reorder", requests=1, beams=4, slots=4, layers=24, heads=32, n=64, d=2048),
        # Four requests of eight beams, their states scattered over a cache, 7B-class.
        dict(name="reorder_b4", op="reorder", requests=4, beams=8, slots=40, layers=32, heads=64, n=64, d=4096),
        # The per-channel sums of a chain of four blocks at its widest batch: no matrix states, small rows.
        dict(name="reorder_rows", op="reorder", requests=2, beams=8, slots=16, layers=4, heads=0, n=0, d=2048),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    op = rng.choice(["lowrank", "lowrank", "lowrank", "select", "select", "reorder"])
    if op == "lowrank":
        seqs = rng.choice([1, _log(rng, 2, 128)])
        tokens = rng.choice([seqs, _log(rng, 1, 2500)])
        return dict(op=op, seqs=seqs, tokens=tokens, ic=_log(rng, 64, 7168, 8), oc=_log(rng, 64, 7168, 8), rank=_log(rng, 8, 128, 8), ragged_ranks=rng.random() < 0.5,
                    adapters=_log(rng, 1, 32), free=rng.choice([0.0, 0.2]), x=rng.choice(["bf16", "bf16", "f16", "f32"]), w=rng.choice(["bf16", "f16"]),
                    y=rng.choice(["f32", "bf16", "f16"]), mix=rng.random() < 0.5)
    if op == "select":
        beams = rng.choice([1, 2, 3, 4, 5, 8, 12, 16])
        return dict(op=op, requests=_log(rng, 1, max(1, 256 // beams)), beams=beams, vocab=_log(rng, 256, 65536), picks=rng.choice([beams, 2 * beams]),
                    dtype=rng.choice(["f32", "bf16", "f16"]), first=rng.random() < 0.2, done=rng.choice([0.0, 0.3]), kept=rng.choice([1.0, 1.0, 0.01]), pad=rng.choice([0, 0, 5, 8]))
    beams, requests = rng.choice([2, 3, 4, 5, 8, 16]), _log(rng, 1, 4)
    return dict(op=op, requests=requests, beams=beams, slots=beams * requests + rng.choice([0, 7]), layers=_log(rng, 1, 24), heads=rng.choice([0, _log(rng, 1, 32)]), n=64,
                d=_log(rng, 64, 4096, 8))


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


def adapters_of(case):
    """(adapter of each sequence, -1: none; rank of each adapter): properties of the case."""
    rng = random.Random(f"{case['seqs']} {case['adapters']} {case['rank']}")
    ranks = [rng.randint(max(1, case["rank"] // 8), case["rank"]) if case["ragged_ranks"] else case["rank"] for _ in range(case["adapters"])]
    if case["ragged_ranks"]:
        ranks[-1] = case["rank"]
    return [-1 if rng.random() < case["free"] else rng.randrange(case["adapters"]) for _ in range(case["seqs"])], ranks


def parents_of(case):
    """The parents of each request's beams, a property of the case: the better a beam, the more of them go on from it; the first request's stay where they are but one."""
    rng = random.Random(f"{case['requests']} {case['beams']}")
    K = case["beams"]
    out = [sorted(min(int(rng.expovariate(3.0 / K)), K - 1) for _ in range(K)) for _ in range(case["requests"])]
    for p in out:
        rng.shuffle(p)
    out[0] = list(range(K - 1)) + [0]
    return out


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=case)
    if case["op"] == "lowrank":
        T, S, ic, oc, r, n = (case[c] for c in ("tokens", "seqs", "ic", "oc", "rank", "adapters"))
        # N(0, 1) with eight outlier channels twenty times as large; one row more in front, so that the rows before are a view
        x = torch.randn((T + 1, ic), generator=g, device="cuda")
        x[:, torch.randperm(ic, generator=g, device="cuda")[:8]] *= 20.0
        st["x_all"] = x.to(TORCH[case["x"]])
        st["x"] = st["x_all"][1:]
        st["A"] = (torch.randn((n, r, ic), generator=g, device="cuda") / ic ** 0.5).to(TORCH[case["w"]])
        st["B"] = (torch.randn((n, oc, r), generator=g, device="cuda") * 0.2).to(TORCH[case["w"]])
        st["scale"] = torch.rand((n,), generator=g, device="cuda") + 0.5
        st["y"] = torch.randn((T, oc), generator=g, device="cuda").to(TORCH[case["y"]])
        adapter, ranks = adapters_of(case)
        st["lens"] = lengths(case)
        starts = [0]
        for l in st["lens"]:
            starts.append(starts[-1] + l)
        st["starts"] = starts
        st["seq_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        st["adapter"] = torch.tensor(adapter, dtype=torch.int32, device="cuda")
        st["ranks"] = torch.tensor(ranks, dtype=torch.int32, device="cuda")
        st["mu"] = None
        if case["mix"]:
            # a token-shift vector as the framework stores it: 64 pairs and an index of six bits for every two columns
            st["table"] = torch.rand((64, 2), generator=g, device="cuda").half()
            st["index"] = torch.randint(0, 64, (ic // 2,), generator=g, device="cuda")
            st["mu"] = st["table"][st["index"]].view(ic)
            st["x_prev"] = st["x_all"][:T]
            if own:
                from paper_2505_03803_b200 import binding as B
                blob = B.rwkvq_pack(None, 1, ic, B.RWKVQ_VQ, 6, codes=dict(q=st["index"].to(torch.uint8).cpu().numpy(), codebook=st["table"].cpu().numpy()))
                st["mu_desc"], st["mu_image"] = blob.desc, blob.to_device()
        return st
    if case["op"] == "select":
        R, K, V = case["requests"], case["beams"], case["vocab"]
        logits = torch.randn((R * K, V + case["pad"]), generator=g, device="cuda") * 2.5
        if case["first"]:
            logits = logits[::K].repeat_interleave(K, 0)
        if case["kept"] < 1.0:
            logits = torch.where(torch.rand(logits.shape, generator=g, device="cuda") < case["kept"], logits, torch.full_like(logits, -math.inf))
        st["logits"] = logits.to(TORCH[case["dtype"]])[:, :V]
        st["scores"] = -torch.rand((R, K), generator=g, device="cuda") * 4.0 - 10.0
        if case["first"]:
            st["scores"] = torch.where(torch.arange(K, device="cuda") == 0, 0.0, -math.inf).expand(R, K).contiguous()
        st["finished"] = (torch.rand((R, K), generator=g, device="cuda") < case["done"]).to(torch.uint8) if case["done"] else None
        st["eos"] = V // 2
        if own:
            from paper_2505_03803_b200 import binding as B
            P = case["picks"]
            st["next"] = torch.empty((R, P), device="cuda")
            st["parents"], st["tokens"] = (torch.empty((R, P), dtype=torch.int32, device="cuda") for _ in range(2))
            st["workspace"] = torch.empty(max(16, B.rwkvq_beam_select_workspace_bytes(R, K, V, P)), dtype=torch.uint8, device="cuda")
        return st
    R, K, L, S = case["requests"], case["beams"], case["layers"], case["slots"]
    st["parents"] = torch.tensor(parents_of(case), dtype=torch.int32, device="cuda")
    st["slots"] = torch.randperm(S, generator=g, device="cuda")[:R * K].to(torch.int32).view(R, K)
    # token-shift rows of both halves of a layer, and its matrix state, or the sums of the per-channel recurrence
    st["rows"] = torch.randn((2, L, S, case["d"]), generator=g, device="cuda").half()
    st["sums"] = torch.randn((L, S, case["heads"], case["n"], case["n"]) if case["heads"] else (3 * L, S, case["d"]), generator=g, device="cuda")
    if own:
        from paper_2505_03803_b200 import binding as B
        st["parts"] = B.make_state_parts([*st["sums"].unbind(0), *st["rows"].flatten(0, 1).unbind(0)])
    return st


# ---- one pass -----------------------------------------------------------------------------------------------
def run(st):
    case = st["case"]
    if own:
        return _run_own(case, st)
    if case["op"] == "lowrank":
        return _lowrank_plain(case, st)
    if case["op"] == "select":
        return _select_plain(case, st)
    to = st["slots"].long()
    at = torch.gather(to, 1, st["parents"].long()).flatten()
    for x in (st["sums"], st["rows"].flatten(0, 1)):
        x[:, to.flatten()] = x[:, at]
    return {"sums": st["sums"], "rows": st["rows"]}


def _run_own(case, st):
    from paper_2505_03803_b200 import binding as B
    if case["op"] == "lowrank":
        single = case["seqs"] in (1, case["tokens"])
        B.rwkvq_lowrank(st["x"], st["A"], st["B"], st["y"], st["adapter"], seq_start=None if single else st["seq_start"], ranks=st["ranks"] if case["ragged_ranks"] else None,
                        scale=st["scale"], x_prev=st["x_prev"] if case["mix"] else None, mu_desc=st["mu_desc"] if case["mix"] else None,
                        mu_image=st["mu_image"] if case["mix"] else None)
        return {"y": st["y"]}          # the projection's output, to which the adapters are added in place
    if case["op"] == "select":
        B.rwkvq_beam_select(st["logits"], st["scores"], st["next"], st["parents"], st["tokens"], finished=st["finished"], eos=st["eos"], workspace=st["workspace"])
        return {"scores": st["next"], "parents": st["parents"], "tokens": st["tokens"]}
    B.rwkvq_state_reorder(st["parts"], st["parents"], slots=st["slots"])
    return {"sums": st["sums"], "rows": st["rows"]}


def _lowrank_plain(case, st):
    """Every adapter's rows of A in one product, what is not a row's own adapter's is masked, and one product with all of B."""
    T, ic, oc, r, n = (case[c] for c in ("tokens", "ic", "oc", "rank", "adapters"))
    x = st["x"].float()
    if case["mix"]:
        x = (x + (st["x_prev"].float() - x) * st["mu"].float()).to(TORCH[case["x"]]).float()
    lens = st["seq_start"][1:] - st["seq_start"][:-1]
    mine = torch.repeat_interleave(st["adapter"], lens, output_size=T)
    h = (x @ st["A"].float().view(n * r, ic).T).view(T, n, r)
    live = (mine.view(T, 1) == torch.arange(n, device="cuda")).unsqueeze(-1) & (torch.arange(r, device="cuda") < st["ranks"].view(n, 1))
    h = torch.where(live, h * st["scale"].view(n, 1), torch.zeros_like(h))
    d = h.view(T, n * r) @ st["B"].float().permute(0, 2, 1).reshape(n * r, oc)
    st["y"].copy_(st["y"].float() + d)
    return {"y": st["y"]}


def _select_plain(case, st):
    """All totals of a request side by side, in 64 bits (candidates of different beams come near one another), sorted."""
    R, K, V, P = (case[c] for c in ("requests", "beams", "vocab", "picks"))
    l = st["logits"].double()
    m = l.amax(1, keepdim=True).clamp(min=-1e300)
    score = st["scores"].double().view(R * K, 1)
    total = score + (l - m - torch.log(torch.exp(l - m).sum(1, keepdim=True)))
    total = torch.where((l == -math.inf) | (score == -math.inf), -math.inf, total)
    if st["finished"] is not None:
        end = torch.where(torch.arange(V, device="cuda") == st["eos"], score, -math.inf)
        total = torch.where(st["finished"].view(R * K, 1) != 0, end, total)
    best, at = torch.sort(total.view(R, K * V), dim=1, descending=True, stable=True)
    best, at = best[:, :P], at[:, :P]
    return {"scores": best.float(), "parents": (at // V).int(), "tokens": (at % V).int()}


# ---- the definition in 64 bits ------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "lowrank":
        adapter, ranks = adapters_of(case)
        y = st["y"].double()
        for a, t0, t1 in zip(adapter, st["starts"], st["starts"][1:]):
            if a < 0 or t0 == t1:
                continue
            x = st["x"][t0:t1].double()
            if case["mix"]:
                mu = st["table"].double()[st["index"]].flatten()
                x = ((1.0 - mu) * x + mu * st["x_all"][t0:t1].double()).to(TORCH[case["x"]]).double()
            r = ranks[a]
            y[t0:t1] += torch.einsum("tr,or->to", torch.einsum("ti,ri->tr", x, st["A"][a, :r].double()), st["B"][a, :, :r].double()) * st["scale"][a].double()
        return {"y": y}
    if case["op"] == "select":
        # the totals of what is chosen, beam by beam, from each beam's own best
        R, K, V, P = (case[c] for c in ("requests", "beams", "vocab", "picks"))
        out = torch.full((R, P), -math.inf, dtype=torch.float64, device="cuda")
        for q in range(R):
            every = []
            for k in range(K):
                s = st["scores"][q, k].double()
                if st["finished"] is not None and st["finished"][q, k]:
                    every.append(s.view(1))
                elif s > -math.inf:
                    best = torch.log_softmax(st["logits"][q * K + k].double(), 0).nan_to_num(nan=-math.inf).sort(descending=True).values[:P]
                    every.append(s + best)
            every = torch.cat(every).sort(descending=True).values[:P]
            out[q, :len(every)] = every
        return {"scores": out, "parents": None, "tokens": None}
    sums, rows = st["sums"].clone(), st["rows"].clone()
    for slots, parents in zip(st["slots"].tolist(), parents_of(case)):
        for b, p in enumerate(parents):
            sums[:, slots[b]] = st["sums"][:, slots[p]]
            rows[:, :, slots[b]] = st["rows"][:, :, slots[p]]
    return {"sums": sums.double(), "rows": rows.double()}


# ---- what a pass cannot do without --------------------------------------------------------------------------
def work(case):
    if case["op"] == "lowrank":
        ic, oc = case["ic"], case["oc"]
        adapter, ranks = adapters_of(case)
        tokens = flops = 0
        for a, l in zip(adapter, lengths(case)):
            if a >= 0:
                tokens += l
                flops += 2 * l * ranks[a] * (ic + oc)
        used = {a for a, l in zip(adapter, lengths(case)) if a >= 0 and l}
        rows = tokens + (1 if case["mix"] and tokens else 0)                          # the rows before are the same rows but one
        # the adapters are added to a product's output: rows that have one are read and written
        return {"bytes": rows * ic * SIZE[case["x"]] + 2 * tokens * oc * SIZE[case["y"]] + 2 * sum(ranks[a] for a in used) * (ic + oc), "flops": max(flops, 1)}
    if case["op"] == "select":
        R, K, V = case["requests"], case["beams"], case["vocab"]
        rows = R if case["first"] else R * K * (1.0 - case["done"])
        return {"bytes": rows * V * SIZE[case["dtype"]] + R * (4 * K + 12 * case["picks"]), "flops": 4 * rows * V}
    moved = sum(len({p for b, p in enumerate(ps) if p != b}) + sum(p != b for b, p in enumerate(ps)) for ps in parents_of(case))
    each = case["layers"] * (4 * (case["heads"] * case["n"] ** 2 if case["heads"] else 3 * case["d"]) + 4 * case["d"])
    return {"bytes": moved * each, "flops": 0}
