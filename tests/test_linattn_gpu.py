"""Linear attention with decaying state (rwkvq_linattn) against the recurrence in 64 bits."""
import math

import pytest
import torch

from paper_2505_03803_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# of a sum's terms, the part that may be lost where an output's operands are split for the tensor cores: two terms of eight bits each (off by 2^-17
# of either operand, the product of the two second ones left out: 2^-16) or three (2^-25 each, three products of 2^-24 left out), and as much again
SPLIT = {"f32": 10 * 2.0 ** -24, "f16": 2.0 ** -14, "bf16": 2.0 ** -14}
E24 = 2.0 ** -24


def reference(r, k, v, lw, u, S, parts):
    """One sequence, double precision: r, k, v [T, H, N], lw [T, H, N], u [H, N], S [H, N, N].  Returns (out, its tolerance, S, its tolerance).

    Tolerances: per token a decay (its exponential and the logarithms' sum) and two roundings, against the magnitudes M that were added up; a sum of x in
    logarithms that is off by 16 * 2^-24 * x makes a term e^-x off by x e^-x <= 0.74 e^(-x/2), so also against H, in which decays are square roots."""
    T, H, N = r.shape
    M, Hm = S.abs().clone(), S.abs().clone()
    E = torch.zeros_like(S)
    out, tol = torch.empty_like(r), torch.empty_like(r)
    for t in range(T):
        kv = k[t].unsqueeze(-1) * v[t].unsqueeze(-2)
        cur = S + u.unsqueeze(-1) * kv
        out[t] = torch.einsum("hi,hij->hj", r[t], cur)
        mag = torch.einsum("hi,hij->hj", r[t].abs(), M + u.abs().unsqueeze(-1) * kv.abs())
        half = torch.einsum("hi,hij->hj", r[t].abs(), Hm)
        tol[t] = torch.einsum("hi,hij->hj", r[t].abs(), E) + ((N + 16) * E24 + parts) * mag + 12 * E24 * half
        w = torch.exp(lw[t]).unsqueeze(-1)
        S = w * S + kv
        M = w * M + kv.abs()
        Hm = w.sqrt() * Hm + kv.abs()
        E = w * E + E24 * (8 * M + 2 * Hm)
    return out, tol, S, E + 12 * E24 * Hm


def make(seed, lens, heads, n, dtype, decay="channel", decay_f32=True, static=False, bonus=True, extra_slots=0, pad=0, strong=True):
    g = torch.Generator().manual_seed(seed)
    T = sum(lens) + pad
    dt = TYPES[dtype]
    c = dict(lens=lens, heads=heads, n=n, dtype=dtype, T=T, pad=pad)
    rkv = torch.randn((T, 3, heads, n), generator=g).to(dt)
    rows = 1 if static else T
    shape = (rows, heads, n) if decay == "channel" else (rows, heads)
    lw = -torch.exp(torch.randn(shape, generator=g) * 2.0 - 2.0)
    if strong:
        lw = torch.where(torch.rand(shape, generator=g) < 0.03, torch.full_like(lw, -math.inf), lw)
        lw = torch.where(torch.rand(shape, generator=g) < 0.03, torch.zeros_like(lw), lw)
    c["rkv"], c["lw"] = rkv, lw if decay_f32 else lw.to(dt)
    c["u"] = torch.randn((heads, n), generator=g) if bonus else None
    n_slots = len(lens) + extra_slots
    c["slots"] = torch.randperm(n_slots, generator=g)[:len(lens)].to(torch.int32) if extra_slots else None
    c["state"] = torch.randn((n_slots, heads, n, n), generator=g)
    starts = [0]
    for l in lens:
        starts.append(starts[-1] + l)
    c["starts"] = starts
    return c


def expected(c, state=True, device="cpu"):
    c = {x: y.to(device) if torch.is_tensor(y) and x != "slots" else y for x, y in c.items()}
    r, k, v = (c["rkv"][:, i].double() for i in range(3))
    T, H, n = r.shape
    lw = c["lw"].double()
    if lw.dim() == 2:
        lw = lw.unsqueeze(-1).expand(lw.shape[0], H, n)
    lw = lw.expand(T, H, n)
    u = c["u"].double() if c["u"] is not None else torch.ones((H, n), dtype=torch.float64, device=device)
    S = c["state"].double().clone() if state else torch.zeros_like(c["state"], dtype=torch.float64)
    tolS = torch.zeros_like(S)
    out, tol = torch.zeros_like(r), torch.zeros_like(r)
    for i, (a, b) in enumerate(zip(c["starts"], c["starts"][1:])):
        s = i if c["slots"] is None else int(c["slots"][i])
        if a == b and state:
            continue
        out[a:b], tol[a:b], S[s], tolS[s] = reference(r[a:b], k[a:b], v[a:b], lw[a:b], u, S[s], SPLIT[c["dtype"]])
    tol = tol + HALF_ULP[c["dtype"]] * out.abs() + 2.0 ** -24 * (c["dtype"] == "f16")
    return out.cpu(), tol.cpu(), S.cpu(), tolS.cpu()


def call(c, in_place=True, state=True, keep=True, stream=None, ragged=None):
    dev = {x: None if c[x] is None else c[x].cuda() for x in ("rkv", "lw", "u", "slots", "state")}
    out = torch.full((c["T"], c["heads"], c["n"]), 7.0, dtype=TYPES[c["dtype"]], device="cuda")
    lw = dev["lw"].expand(c["T"], *dev["lw"].shape[1:])
    ws = torch.full((max(16, B.rwkvq_linattn_workspace_bytes(c["T"], len(c["lens"]), c["heads"], c["n"])),), 0xFF, dtype=torch.uint8, device="cuda")
    seq_start = torch.tensor(c["starts"], dtype=torch.int32, device="cuda") if len(c["lens"]) > 1 or c["pad"] or ragged else None
    st = dev["state"] if state else None
    st_out = dev["state"] if in_place else torch.full_like(dev["state"], 9.0)
    if not keep:
        st_out = None
    r, k, v = dev["rkv"][:, 0], dev["rkv"][:, 1], dev["rkv"][:, 2]
    B.rwkvq_linattn(r, k, v, lw, dev["u"], out, st, state_out=st_out, seq_start=seq_start, slots=dev["slots"], workspace=ws, stream=stream)
    torch.cuda.synchronize()
    return out, st_out, dev["state"]


def near(got, ref, tol, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    err = (got - ref).abs()
    worst = (err / tol.clamp(min=1e-300)).max().item() if err.numel() else 0.0
    assert (err <= tol).all(), f"{what}: max err/tol {worst} at {torch.nonzero(err > tol)[:3].tolist()}"


def check(c, **kw):
    out, st, _ = call(c, **kw)
    ref, tol, S, tolS = expected(c)
    rows = c["starts"][-1]
    near(out[:rows], ref[:rows], tol[:rows], "out")
    assert (out[rows:] == 7).all(), "rows behind the last sequence"
    near(st, S, tolS, "state")


LENGTHS = [[1], [2], [15], [16], [17], [33], [64], [100], [257], [1] * 7, [0, 3, 0, 17, 1, 64, 0], [130, 2, 65, 1], [48, 48, 48], [5] * 20, [700, 1, 1, 1]]


@pytest.mark.parametrize("lens", LENGTHS, ids=lambda l: "-".join(map(str, l[:7])))
@pytest.mark.parametrize("dtype", list(TYPES))
def test_lengths(lens, dtype):
    check(make(len(lens) * 1000 + sum(lens), lens, 3, 64, dtype, extra_slots=2 if len(lens) > 1 else 0))


@pytest.mark.parametrize("lens", [[1], [17], [200], [1] * 5, [0, 40, 1, 129]], ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("dtype", list(TYPES))
def test_heads_of_128(lens, dtype):
    check(make(sum(lens), lens, 2, 128, dtype))


@pytest.mark.parametrize("decay", ["channel", "head"])
@pytest.mark.parametrize("decay_f32", [True, False])
@pytest.mark.parametrize("static", [True, False])
@pytest.mark.parametrize("lens", [[3], [70], [1] * 4, [50, 0, 90]], ids=lambda l: "-".join(map(str, l)))
def test_forms_of_decay(decay, decay_f32, static, lens):
    check(make(sum(lens) + 5, lens, 5, 64, "bf16", decay=decay, decay_f32=decay_f32, static=static))


@pytest.mark.parametrize("lens", [[1], [90], [1, 1, 1], [30, 70]], ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_without_bonus_and_into_another_state(lens, dtype):
    c = make(sum(lens) + 9, lens, 2, 64, dtype, bonus=False)
    out, st, before = call(c, in_place=False)
    ref, tol, S, tolS = expected(c)
    near(out, ref, tol, "out")
    near(st, S, tolS, "state")
    assert torch.equal(before.cpu(), c["state"]), "the states read are left as they were"


@pytest.mark.parametrize("lens", [[1], [90], [0, 1, 1, 0], [30, 0, 70]], ids=lambda l: "-".join(map(str, l)))
def test_from_zeros_and_kept_or_not(lens):
    c = make(sum(lens) + 11, lens, 2, 64, "bf16")
    ref, tol, S, tolS = expected(c, state=False)
    out, st, _ = call(c, in_place=False, state=False)
    near(out, ref, tol, "out")
    near(st, S, tolS, "state")
    out2, st, _ = call(c, state=False, keep=False)
    assert st is None and torch.equal(out, out2)


@pytest.mark.parametrize("lens", [[1, 1], [40, 90]], ids=str)
def test_rows_behind_the_last_sequence_and_states_of_none(lens):
    c = make(sum(lens), lens, 2, 64, "f16", extra_slots=3, pad=21)
    out, st, _ = call(c)
    used = set(c["slots"].tolist())
    for s in range(st.shape[0]):
        if s not in used:
            assert torch.equal(st[s].cpu(), c["state"][s])
    check(c)


def test_everything_forgotten_and_nothing():
    # decays of zero: an output sees its own token and the one before, the state is the last token's; decays of one: plain sums
    for value in (-math.inf, 0.0, -200.0):
        for lens in ([1], [100]):
            c = make(3, lens, 2, 64, "f32", strong=False)
            c["lw"].fill_(value)
            check(c)


def test_slow_decays_over_a_long_sequence():
    # one chunk's decays are 1 - 1e-4 and less: what is lost would be lost over and over
    c = make(4, [1500], 1, 64, "bf16", static=True, strong=False)
    c["lw"] = -torch.logspace(-7, -3, 64).reshape(1, 1, 64)
    check(c)


def test_continued_in_pieces():
    # a prompt in one call, or in pieces that hand the state on (chunked prefill, then single tokens)
    c = make(21, [170], 2, 64, "f32")
    ref, tol, S, tolS = expected(c)
    dev = {x: c[x].cuda() for x in ("rkv", "lw", "u", "state")}
    out = torch.empty((170, 2, 64), device="cuda")
    at = 0
    for piece in (64, 1, 33, 70, 1, 1):
        sl = slice(at, at + piece)
        ws = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(piece, 1, 2, 64)), dtype=torch.uint8, device="cuda")
        B.rwkvq_linattn(dev["rkv"][sl, 0], dev["rkv"][sl, 1], dev["rkv"][sl, 2], dev["lw"][sl], dev["u"], out[sl], dev["state"], workspace=ws)
        at += piece
    near(out, ref, tol, "out")
    near(dev["state"], S, tolS, "state")


def test_nothing_to_do_keeps_states():
    c = make(1, [0, 0], 2, 64, "bf16")
    out, st, _ = call(c, in_place=False)
    assert out.numel() == 0 and torch.equal(st.cpu(), c["state"])


@pytest.mark.parametrize("lens", [[1, 1, 1, 1], [20, 30, 40, 50]], ids=str)
def test_bad_slots_are_reported_and_left_out(lens):
    c = make(31, lens, 2, 64, "bf16", extra_slots=2)
    c["slots"] = torch.tensor([4, 4, 17, 1], dtype=torch.int32)       # the second has the first one's, the third does not exist
    out, st, _ = call(c)
    assert B.rwkvq_device_status() == 1
    assert B.rwkvq_device_status() == 0
    c2 = dict(c, slots=torch.tensor([4, 2, 3, 1], dtype=torch.int32))
    ref, tol, S, tolS = expected(c2)
    a = c["starts"]
    near(out[a[0]:a[1]], ref[a[0]:a[1]], tol[a[0]:a[1]], "first")
    near(out[a[3]:a[4]], ref[a[3]:a[4]], tol[a[3]:a[4]], "last")
    assert (out[a[1]:a[3]] == 7).all()
    for s in (0, 2, 3, 5):
        assert torch.equal(st[s].cpu(), c["state"][s])
    near(st[[4, 1]], S[[4, 1]], tolS[[4, 1]], "states")


def test_slot_of_none_begins_with_zeros():
    lens = [40, 1, 25]
    c = make(32, lens, 2, 64, "f32")
    c["slots"] = torch.tensor([-1, 2, -1], dtype=torch.int32)
    out, st, _ = call(c)
    assert B.rwkvq_device_status() == 0
    z = dict(c, state=c["state"].clone(), slots=None)
    z["state"][0], z["state"][1], z["state"][2] = 0, c["state"][2], 0
    ref, tol, S, tolS = expected(z)
    near(out, ref, tol, "out")
    near(st[2], S[1], tolS[1], "state")
    assert torch.equal(st[:2].cpu(), c["state"][:2])


def test_rows_out_of_order_are_reported():
    c = make(33, [20, 30, 10], 2, 64, "bf16")
    c["starts"] = [0, 20, 70, 60]                  # the second ends behind the rows, the third before it begins
    out, st, _ = call(c)
    assert B.rwkvq_device_status() == 1
    assert torch.equal(st[1:].cpu(), c["state"][1:]) and (out[20:] == 7).all()
    c["starts"] = [0, 20, 20, 20]
    ref, tol, S, tolS = expected(c)
    near(out[:20], ref[:20], tol[:20], "first")


@pytest.mark.parametrize("lens", [[1, 1, 1], [80, 5, 200]], ids=str)
def test_repeated_captured_and_on_another_stream(lens):
    c = make(41, lens, 3, 64, "bf16", extra_slots=1)
    first, st, _ = call(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other, st2, _ = call(c, stream=s)
    assert torch.equal(first, other) and torch.equal(st, st2)
    dev = {x: c[x].cuda() for x in ("rkv", "lw", "u", "slots", "state")}
    out, st_out = torch.zeros_like(first), torch.zeros_like(dev["state"])
    ws = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(c["T"], len(lens), 3, 64)), dtype=torch.uint8, device="cuda")
    seq_start = torch.tensor(c["starts"], dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rwkvq_linattn(dev["rkv"][:, 0], dev["rkv"][:, 1], dev["rkv"][:, 2], dev["lw"], dev["u"], out, dev["state"], state_out=st_out, seq_start=seq_start,
                        slots=dev["slots"], workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(st_out[c["slots"].long()], st[c["slots"].long()])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("n", [64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_token_does_not_see_what_comes_after_it(dtype, n, value):
    # infinities and NaN in one token's r, k or v: the outputs before it are what they are without it, and other heads' and value columns' are all
    T, at = 75, 37
    c = make(51, [T], 2, n, dtype, strong=False)
    ref, tol, S, tolS = expected(c)
    for which in range(3):
        bad = dict(c, rkv=c["rkv"].clone())
        bad["rkv"][at, which, 1, 5] = value
        out, st, _ = call(bad)
        near(out[:at], ref[:at], tol[:at], f"before {'rkv'[which]}")
        near(out[:, 0], ref[:, 0], tol[:, 0], "the other head")
        near(st[:, 0], S[:, 0], tolS[:, 0], "the other head's state")
        if which == 0:
            near(out[at + 1:], ref[at + 1:], tol[at + 1:], "r is its own token's alone")
            near(st, S, tolS, "r is not in the state")
        if which == 2:
            columns = [j for j in range(n) if j != 5]
            near(out[:, 1][:, columns], ref[:, 1][:, columns], tol[:, 1][:, columns], "other values")
            near(st[:, 1][:, :, columns], S[:, 1][:, :, columns], tolS[:, 1][:, :, columns], "other values' state")
            assert not torch.isfinite(out[at:, 1, 5].float()).any()


# sizes at which blocks of rows are dealt out evenly and some have rows of two heads, at which a head is one block, and at which it is several
@pytest.mark.parametrize("lens,heads,n,dtype", [([2000], 64, 64, "bf16"), ([700, 1100, 1, 0, 300, 20], 64, 64, "f16"), ([1000], 80, 128, "bf16"), ([40], 200, 64, "f32"),
                                                ([500], 150, 64, "bf16"), ([9] * 60, 40, 64, "bf16"), ([1500], 64, 64, "f32")], ids=str)
def test_many_heads(lens, heads, n, dtype):
    c = make(61, lens, heads, n, dtype)
    out, st, _ = call(c)
    assert B.rwkvq_device_status() == 0
    ref, tol, S, tolS = expected(c, device="cuda")
    near(out, ref, tol, "out")
    near(st, S, tolS, "state")


@pytest.mark.parametrize("lens", [[1, 1], [30, 100]], ids=str)
def test_rows_in_front_of_the_first_sequence(lens):
    c = make(62, lens, 2, 64, "bf16", pad=23)
    c["starts"] = [x + 19 for x in c["starts"]]
    out, st, _ = call(c, ragged=True)
    ref, tol, S, tolS = expected(c)
    a, b = c["starts"][0], c["starts"][-1]
    near(out[a:b], ref[a:b], tol[a:b], "out")
    near(st, S, tolS, "state")
    assert (out[:a] == 7).all() and (out[b:] == 7).all()


def test_one_sequence_with_a_slot():
    for T in (1, 60):
        c = make(63, [T], 2, 64, "f16", extra_slots=4)
        check(c)


def test_a_cache_of_more_than_32_bits():
    # 8200 slots of 64 heads: the last state begins behind 2^31 numbers
    slots, heads = 8200, 64
    state = torch.empty((slots, heads, 64, 64), device="cuda")
    assert state.numel() > 2 ** 31
    for lens in ([1, 1], [40, 3]):
        c = make(64, lens, heads, 64, "bf16")
        ids = torch.tensor([slots - 1, 3], dtype=torch.int32)
        state[ids.long()] = c["state"].cuda()
        T = sum(lens)
        rkv, out = c["rkv"].cuda(), torch.empty((T, heads, 64), dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(T, 2, heads, 64)), dtype=torch.uint8, device="cuda")
        B.rwkvq_linattn(rkv[:, 0], rkv[:, 1], rkv[:, 2], c["lw"].cuda(), c["u"].cuda(), out, state, slots=ids.cuda(), workspace=ws,
                        seq_start=torch.tensor(c["starts"], dtype=torch.int32, device="cuda"))
        ref, tol, S, tolS = expected(c, device="cuda")
        near(out, ref, tol, "out")
        near(state[ids.long()], S, tolS, "state")


@pytest.mark.parametrize("what", ["heads apart", "values apart", "another type", "short logw", "decays of a third type", "u in half", "states in half", "states strided",
                                  "states of another count", "slots short", "slots of 64 bits", "rows on the host", "workspace short", "workspace strided"])
def test_binding_refuses(what):
    T, H, N, n_seq = 64, 2, 64, 2
    z = lambda *s, dtype=torch.float16: torch.zeros(s, dtype=dtype, device="cuda")
    size = B.rwkvq_linattn_workspace_bytes(T, n_seq, H, N)
    a = dict(r=z(T, H, N), k=z(T, H, N), v=z(T, H, N), logw=z(T, H, N), u=z(H, N, dtype=torch.float32), out=z(T, H, N), state=z(3, H, N, N, dtype=torch.float32),
             seq_start=torch.tensor([0, 30, 64], dtype=torch.int32, device="cuda"), slots=torch.tensor([2, 0], dtype=torch.int32, device="cuda"),
             workspace=z(size, dtype=torch.uint8))
    bad = {"heads apart": dict(r=z(T, 2 * H, N)[:, ::2]), "values apart": dict(v=z(T, H, 2 * N)[..., ::2]), "another type": dict(k=z(T, H, N, dtype=torch.bfloat16)),
           "short logw": dict(logw=z(T - 1, H, N)), "decays of a third type": dict(logw=z(T, H, N, dtype=torch.bfloat16)), "u in half": dict(u=z(H, N)),
           "states in half": dict(state=z(3, H, N, N)), "states strided": dict(state=z(3, H, N, 2 * N, dtype=torch.float32)[..., ::2]),
           "states of another count": dict(state_out=z(4, H, N, N, dtype=torch.float32)), "slots short": dict(slots=a["slots"][:1]),
           "slots of 64 bits": dict(slots=a["slots"].long()), "rows on the host": dict(seq_start=a["seq_start"].cpu()),
           "workspace short": dict(workspace=z(size - 16, dtype=torch.uint8)), "workspace strided": dict(workspace=z(2 * size, dtype=torch.uint8)[::2])}
    B.rwkvq_linattn(**a)
    with pytest.raises(B.RwkvqError):
        B.rwkvq_linattn(**dict(a, **bad[what]))
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0


# lists that fall back: a sequence that begins in front of an entry before its own may share rows with one that is computed
@pytest.mark.parametrize("starts,good,heads", [([0, 100, 50, 150], [0], 2), ([0, 2000, 1000, 2500], [0], 64), ([0, 30, 20, 64, 90], [0, 3], 3), ([40, 10, 50, 90], [2], 2),
                                               ([0, 3, 1, 5], [0], 2), ([0, 700, 600, 1300, 1300, 1290, 1400], [0, 3], 40)], ids=str)
@pytest.mark.parametrize("slots", [False, True])
def test_a_sequence_that_begins_in_front_of_an_earlier_one_is_left_out(starts, good, heads, slots):
    n_seq = len(starts) - 1
    c = make(71, [max(starts)], heads, 64, "bf16", extra_slots=n_seq + 1)
    c["lens"], c["starts"] = [0] * n_seq, starts
    c["slots"] = torch.randperm(n_seq + 2, generator=torch.Generator().manual_seed(5))[:n_seq].to(torch.int32) if slots else None
    out, st, _ = call(c, ragged=True)
    assert B.rwkvq_device_status() == 1 and B.rwkvq_device_status() == 0
    rest, kept = torch.ones(c["T"], dtype=torch.bool), torch.ones(n_seq + 2, dtype=torch.bool)
    for i in good:
        a, b, s = starts[i], starts[i + 1], int(c["slots"][i]) if slots else i
        one = dict(c, starts=[a, b], slots=torch.tensor([s], dtype=torch.int32))
        ref, tol, S, tolS = expected(one, device="cuda")
        near(out[a:b], ref[a:b], tol[a:b], f"sequence {i}")
        near(st[s], S[s], tolS[s], f"state of sequence {i}")
        rest[a:b], kept[s] = False, False
    assert (out[rest.cuda()] == 7).all() and torch.equal(st.cpu()[kept], c["state"][kept])


def apart(x, gap, fill=float("nan")):
    """x on the device, its rows `gap` elements further apart than they are long (NaN between them)."""
    T, row = x.shape[0], x[0].numel()
    wide = torch.full((T, row + gap), fill, dtype=x.dtype, device="cuda")
    view = wide[:, :row].view(x.shape)
    view.copy_(x)
    return view, wide[:, row:]


@pytest.mark.parametrize("lens", [[1], [7], [16], [90], [1] * 6, [40, 0, 1, 70, 5]], ids=lambda l: "-".join(map(str, l)))
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("decay", ["channel", "head"])
@pytest.mark.parametrize("n", [64, 128])
def test_every_row_stride_is_its_own(lens, dtype, decay, n):
    # r, k, v, logw and out each with another distance from row to row: none can be taken for another's
    heads = 4
    c = make(sum(lens) + 81, lens, heads, n, dtype, decay=decay, decay_f32=len(lens) % 2 == 1)
    r, k, v = (apart(c["rkv"][:, i], gap)[0] for i, gap in enumerate((8, 24, 40)))
    lw = apart(c["lw"], 56)[0]
    out, between = apart(torch.full((c["T"], heads, n), 7.0, dtype=TYPES[dtype]), 72, 5.0)
    state = c["state"].cuda()
    ws = torch.empty(max(16, B.rwkvq_linattn_workspace_bytes(c["T"], len(lens), heads, n)), dtype=torch.uint8, device="cuda")
    starts = torch.tensor(c["starts"], dtype=torch.int32, device="cuda") if len(lens) > 1 else None
    B.rwkvq_linattn(r, k, v, lw, c["u"].cuda(), out, state, seq_start=starts, workspace=ws)
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    ref, tol, S, tolS = expected(c)
    near(out, ref, tol, "out")
    near(state, S, tolS, "state")
    assert (between == 5).all()


def test_every_row_stride_is_its_own_where_rows_are_cut():
    c = make(82, [1300], 64, 64, "bf16")
    r, k, v = (apart(c["rkv"][:, i], gap)[0] for i, gap in enumerate((8, 24, 40)))
    lw, (out, between), state = apart(c["lw"], 56)[0], apart(torch.full((1300, 64, 64), 7.0, dtype=torch.bfloat16), 72, 5.0), c["state"].cuda()
    ws = torch.empty(B.rwkvq_linattn_workspace_bytes(1300, 1, 64, 64), dtype=torch.uint8, device="cuda")
    B.rwkvq_linattn(r, k, v, lw, c["u"].cuda(), out, state, workspace=ws)
    ref, tol, S, tolS = expected(c, device="cuda")
    near(out, ref, tol, "out")
    near(state, S, tolS, "state")
    assert (between == 5).all()


@pytest.mark.parametrize("lens", [[1] * 40 + [30], [200] + [1] * 199, [1] * 150 + [0] * 60 + [170, 1, 0], [2] * 30, [0] * 100 + [90] + [1] * 5, [3, 1, 9, 1, 1, 1, 25] + [1] * 45], ids=lambda l: f"{len(l)}-{max(l)}")
@pytest.mark.parametrize("dtype", list(TYPES))
def test_a_long_sequence_among_short_ones(lens, dtype):
    check(make(91 + len(lens), lens, 2, 64, dtype, extra_slots=3))


def test_a_long_sequence_among_short_ones_where_rows_are_cut():
    c = make(92, [1] * 700 + [800] + [1] * 150, 24, 64, "bf16")
    out, st, _ = call(c)
    assert B.rwkvq_device_status() == 0
    ref, tol, S, tolS = expected(c, device="cuda")
    near(out, ref, tol, "out")
    near(st, S, tolS, "state")
