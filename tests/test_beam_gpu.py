"""Beam search's selection (rwkvq_beam_select) against the definition in 64 bits, and the states that follow (rwkvq_state_reorder), bit for bit."""
import math

import pytest
import torch

from paper_2505_03803_b200 import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# The logarithm of a row's sum.  A term e^-d is taken at -d log2 e, rounded (d < 128: off by less than 2^-17, relative to the term, which for large d is small beside the sum:
# d e^-d < 1) twice, 2^-22 for the exponential, and a thread adds up to 2^11 terms in fp32, four at a time.
LSE = 2.0 ** -15


def totals(logits, scores, finished, eos):
    R, K = scores.shape
    l = logits.double().clone()
    l[torch.isnan(l)] = -math.inf
    m = l.amax(1, keepdim=True)
    e = torch.where(l == m, torch.ones_like(l), torch.exp(l - m.clamp(min=-1e300)))
    e[l == -math.inf] = 0.0
    out = torch.where(m == math.inf, torch.where(l == math.inf, 0.0, -math.inf), l - m) - torch.log(e.sum(1, keepdim=True))
    s = scores.double().reshape(R * K, 1)
    out = torch.where((l == -math.inf) | (out == -math.inf) | ~torch.isfinite(s), -math.inf, out + s)
    if finished is not None:
        done = finished.reshape(-1) != 0
        out[done] = -math.inf
        out[done, eos] = torch.where(torch.isfinite(s), s, -math.inf)[done, 0]
    return out.view(R, -1)


def select(logits, scores, picks, finished=None, eos=0, stream=None, row_pad=0, row_at=0):
    R, K = scores.shape
    V = logits.shape[1]
    buf = torch.full((R * K, V + row_pad + row_at), 100.0, dtype=logits.dtype, device="cuda")        # what lies beside the rows would be chosen
    view = buf[:, row_at:row_at + V]
    view.copy_(logits)
    ns = torch.empty((R, picks), device="cuda")
    pa, to = (torch.full((R, picks), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    done = torch.full((R, picks), 9, dtype=torch.uint8, device="cuda")
    ws = torch.full((B.rwkvq_beam_select_workspace_bytes(R, K, V, picks),), 0xFF, dtype=torch.uint8, device="cuda")
    B.rwkvq_beam_select(view, scores.cuda(), ns, pa, to, finished=None if finished is None else finished.cuda(), eos=eos, finished_out=done, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    return ns.cpu(), pa.cpu(), to.cpu(), done.cpu()


def order(ref, logits, V):
    """Totals falling; where they are equal the lower beam, and within a beam the larger logit (that of two totals of 64 bits may be lost: 1e-30 beside 8), then the lower token."""
    R = ref.shape[0]
    l = torch.where(ref == -math.inf, 0.0, logits.double().view(R, -1)).nan_to_num(nan=0.0)
    first = torch.sort(l.view(R, -1, V), dim=2, descending=True, stable=True).indices
    first = (first + V * torch.arange(first.shape[1]).view(1, -1, 1)).view(R, -1)
    best, at = torch.sort(torch.gather(ref, 1, first), dim=1, descending=True, stable=True)
    at = torch.gather(first, 1, at)
    # those of probability zero by their places
    zero = best == -math.inf
    at[zero] = (torch.where(zero, at, -1).sort(dim=1).values)[zero] if zero.any() else at[zero]
    return best, at


def check(logits, scores, picks, finished=None, eos=0, **kw):
    R, K = scores.shape
    V = logits.shape[1]
    ns, pa, to, done = select(logits, scores, picks, finished, eos, **kw)
    ref = totals(logits, scores, finished, eos)
    best, at = order(ref, logits, V)
    flat = pa.long() * V + to.long()
    tol = LSE + 2.0 ** -23 * best[:, :picks].abs().nan_to_num(posinf=0.0)
    same = flat == at[:, :picks]
    got = torch.gather(ref, 1, flat)
    # a place may go to another candidate only where the two are as near one another as the sums are exact
    assert (same | ((got - best[:, :picks]).abs() <= 2 * LSE)).all(), (torch.nonzero(~same)[:4].tolist(), flat[~same][:4], at[:, :picks][~same][:4])
    assert same.float().mean() > 0.98
    fin = torch.isfinite(best[:, :picks])
    assert ((ns.double() - got).abs()[fin] <= tol[fin]).all() and (ns[~fin] == -math.inf).all()
    for r in range(R):
        assert len(set(flat[r].tolist())) == picks
    was = torch.zeros((R, picks), dtype=torch.bool) if finished is None else torch.gather(finished != 0, 1, pa.long())
    assert torch.equal(done != 0, was | (to == eos))


def make(seed, R, K, V, dtype="f32", spread=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((R * K, V), generator=g) * spread).to(TYPES[dtype]), -torch.rand((R, K), generator=g) * 5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("R,K,V,picks", [(1, 1, 1, 1), (1, 1, 7, 7), (2, 3, 5, 15), (1, 4, 65536, 4), (3, 5, 50277, 10), (2, 8, 8191, 16), (1, 64, 1000, 64), (1, 1, 300, 64), (40, 2, 2049, 3),
                                         (5, 16, 33000, 32), (200, 4, 513, 8), (1, 2, 100003, 64), (700, 1, 4097, 2)])
def test_sizes(dtype, R, K, V, picks):
    check(*make(R + K + V, R, K, V, dtype), picks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("row_at", [1, 2, 3, 5, 8, 13])
def test_rows_that_begin_anywhere(dtype, row_at):
    logits, scores = make(row_at, 3, 2, 3000 + row_at, dtype)
    check(logits, scores, 6, row_at=row_at, row_pad=row_at % 4)


@pytest.mark.parametrize("dtype", TYPES)
def test_ties_go_to_the_lowest(dtype):
    for V in (40, 5000, 40000):
        for value in (0.0, 3.5, -2.0):
            logits = torch.full((4, V), value).to(TYPES[dtype])
            ns, pa, to, _ = select(logits, torch.tensor([[-1.0, -1.0], [-2.0, -1.0]]), 20, row_at=1)
            assert pa.tolist() == [[0] * 20, [1] * 20] and to.tolist() == [list(range(20))] * 2
            assert (ns + 1.0 + math.log(V)).abs().max() < 1e-4
        # a few levels: the first of the highest level, wherever they are
        g = torch.Generator().manual_seed(V)
        logits = torch.randint(0, 3, (6, V), generator=g).to(TYPES[dtype])
        for scores in (torch.zeros((2, 3)), torch.tensor([[0.0, -1.0, -2.0], [-3.0, -9.0, -3.0]])):
            ns, pa, to, _ = select(logits, scores, 12)
            for r in range(2):
                l = logits[3 * r:3 * r + 3].double()
                t = totals(logits[3 * r:3 * r + 3], scores[r:r + 1], None, 0).view(3, V)
                want = sorted(((-float(l[k, v]) if scores[r].unique().numel() < 3 and False else -round(float(t[k, v]), 4), k, v) for k in range(3) for v in range(V)))[:12]
                assert [(k, v) for _, k, v in want] == list(zip(pa[r].tolist(), to[r].tolist()))


@pytest.mark.parametrize("dtype", TYPES)
def test_both_zeros_are_one(dtype):
    logits = torch.zeros((2, 700))
    logits[:, ::2] = -0.0
    ns, pa, to, _ = select(logits.to(TYPES[dtype]), torch.tensor([[-0.0, 0.0]]), 9)
    assert pa.tolist() == [[0] * 9] and to.tolist() == [list(range(9))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("low", ["inf", "least"])
def test_masks(dtype, low):
    low = -math.inf if low == "inf" else torch.finfo(TYPES[dtype]).min
    for kept in (0, 1, 3, 40, 1500):
        logits, scores = make(kept, 2, 3, 20000, dtype)
        g = torch.Generator().manual_seed(kept)
        for row in range(6):
            keep = torch.randperm(20000, generator=g)[:kept]
            vals = logits[row, keep].clone()
            logits[row] = low
            logits[row, keep] = vals
        check(logits, scores, 8)
    logits, scores = make(1, 1, 3, 5000, dtype)
    logits[1] = -math.inf                                  # a beam whose mask leaves nothing
    check(logits, scores, 8)
    logits[:, 10:] = -math.inf                             # less than there are places, the last of the alphabet
    logits[0], logits[2, :9] = -math.inf, -math.inf
    check(logits, scores, 8)


def test_rising_and_falling():
    for dtype in ("f32", "f16"):
        up = torch.arange(30000).float() / 4000
        logits = torch.stack([up, up.flip(0), up.roll(777), up.roll(15000).flip(0)]).to(TYPES[dtype])
        check(logits, torch.tensor([[-1.0, -1.5], [-0.5, -0.25]]), 24)


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinities(dtype):
    logits, scores = make(5, 3, 2, 9000, dtype)
    logits[0, 5], logits[0, 8999], logits[1, 77] = math.nan, math.nan, -math.nan
    logits[2, 100], logits[2, 50] = math.inf, math.inf      # share the probability
    logits[3, 0] = math.inf
    logits[4] = math.nan
    check(logits, scores, 7)
    ns, pa, to, _ = select(logits, torch.zeros((3, 2)), 4)
    assert to[1].tolist()[:3] == [0, 50, 100] and pa[1].tolist()[:3] == [1, 0, 0] and torch.allclose(ns[1, :3], torch.tensor([0.0, -math.log(2), -math.log(2)]))


def test_dead_and_finished_beams():
    logits, scores = make(6, 4, 4, 3001)
    scores[0, 1:] = -math.inf                               # a search's first step
    scores[1, 0], scores[1, 2] = math.nan, math.inf
    scores[2] = -math.inf
    check(logits, scores, 8)
    finished = torch.zeros((4, 4), dtype=torch.uint8)
    finished[0, 0], finished[1, 1], finished[3, 2], finished[2] = 1, 7, 1, 1
    check(logits, scores, 8, finished, eos=17)
    check(logits, scores, 8, finished.bool(), eos=3000)
    finished[:] = 1
    check(logits, scores, 8, finished, eos=0)
    bad = logits.clone()
    bad[:] = math.nan                                       # of finished beams nothing is read
    a, b = select(bad, scores, 4, finished, 5), select(logits, scores, 4, finished, 5)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_beams_that_are_the_same():
    logits, scores = make(7, 1, 1, 20000)
    ns, pa, to, _ = select(logits.repeat(4, 1), torch.full((1, 4), -3.0), 8)
    assert pa.tolist() == [[0, 1, 2, 3, 0, 1, 2, 3]] and to[0, :4].unique().numel() == 1 and ns[0, :4].unique().numel() == 1


def test_large_logits():
    logits, scores = make(8, 2, 2, 4000, spread=1.0)
    check(logits * 1e4, scores, 4)
    check(logits * 1e37, scores, 2)
    check(logits * 1e-30, scores, 4)


def test_selection_captured_and_on_another_stream():
    logits, scores = make(9, 4, 4, 30000, "bf16")
    want = select(logits, scores, 4)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = select(logits, scores, 4)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ld, sd, ns = logits.cuda(), scores.cuda(), torch.empty((4, 4), device="cuda")
    pa, to = (torch.empty((4, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty((B.rwkvq_beam_select_workspace_bytes(4, 4, 30000, 4),), dtype=torch.uint8, device="cuda")
    run = lambda: B.rwkvq_beam_select(ld, sd, ns, pa, to, workspace=ws)
    run()
    graphs = []
    for _ in range(2):               # two graphs, one workspace
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        graphs.append(g)
    for i in range(4):
        pa.zero_(), to.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(pa.cpu(), want[1]) and torch.equal(to.cpu(), want[2]) and torch.equal(ns.cpu(), want[0])


def test_rows_behind_32_bits():
    V, rows = 64, 9
    big = torch.empty(((rows - 1) << 29) + V, dtype=torch.float16, device="cuda").as_strided((rows, V), (1 << 29, 1))
    logits, scores = make(10, 3, 3, V, "f16")
    big.copy_(logits)
    ns, pa, to = torch.empty((3, 5), device="cuda"), *(torch.empty((3, 5), dtype=torch.int32, device="cuda") for _ in range(2))
    ws = torch.empty((B.rwkvq_beam_select_workspace_bytes(3, 3, V, 5),), dtype=torch.uint8, device="cuda")
    B.rwkvq_beam_select(big, scores.cuda(), ns, pa, to, workspace=ws)
    want = select(logits, scores, 5)
    assert torch.equal(pa.cpu(), want[1]) and torch.equal(to.cpu(), want[2]) and torch.equal(ns.cpu(), want[0])


# ---- states -------------------------------------------------------------------------------------------------
def reorder(states, parents, slots=None):
    """What the call leaves, and what it should."""
    want = [s.clone() for s in states]
    R, K = parents.shape
    to = slots if slots is not None else torch.arange(R * K).view(R, K)
    for w, s in zip(want, states):
        for r in range(R):
            for b in range(K):
                w[to[r, b]] = s[to[r, parents[r, b]]]
    B.rwkvq_state_reorder(B.make_state_parts(states), parents.int().cuda(), slots=None if slots is None else slots.int().cuda())
    torch.cuda.synchronize()
    assert all(torch.equal(s, w) for s, w in zip(states, want))
    assert B.rwkvq_device_status() == 0


def states_of(n_slots, shapes, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn((n_slots, *s), generator=g, device="cuda") if t == "f32" else torch.randn((n_slots, *s), generator=g, device="cuda").half() for t, s in shapes]


@pytest.mark.parametrize("R,K", [(1, 1), (1, 2), (3, 4), (2, 5), (1, 8), (5, 16), (1, 33), (2, 64)])
def test_parents(R, K):
    g = torch.Generator().manual_seed(R * K)
    shapes = [("f32", (3, 64, 64)), ("f16", (8,)), ("f16", (2048,)), ("f32", (1000,)), ("f16", (4104,))]
    for kind in range(5):
        parents = {0: torch.arange(K).repeat(R, 1), 1: torch.zeros((R, K), dtype=torch.long), 2: torch.stack([torch.randperm(K, generator=g) for _ in range(R)]),
                   3: torch.randint(0, K, (R, K), generator=g), 4: torch.arange(K).roll(1).repeat(R, 1)}[kind]
        reorder(states_of(R * K, shapes, kind), parents)
        slots = torch.randperm(R * K + 9, generator=g)[:R * K].view(R, K)
        reorder(states_of(R * K + 9, shapes, kind + 10), parents, slots)


def test_many_parts_and_layers_inside_one_buffer():
    parents = torch.tensor([[2, 2, 0, 3], [1, 0, 3, 2]])
    reorder(states_of(8, [("f32", (64,))] * 300), parents)
    whole = torch.randn((8, 5, 3, 64), device="cuda")                  # the layers of a slot side by side
    reorder([whole[:, l] for l in range(5)], parents)
    rows = torch.randn((8, 96), device="cuda").half()
    keep = rows.clone()
    reorder([rows[:, 8:40], rows[:, 48:96]], parents)
    assert torch.equal(rows[:, :8], keep[:, :8]) and torch.equal(rows[:, 40:48], keep[:, 40:48])


def test_bad_entries_leave_a_request_as_it_was():
    base = states_of(12, [("f32", (128,)), ("f16", (24,))])
    parents = torch.tensor([[1, 0, 0], [2, 1, 0], [0, 0, 0]])
    slots = torch.tensor([[0, 1, 2], [3, 4, 5], [9, 7, 8]])

    def run(parents, slots, out):
        states = [s.clone() for s in base]
        want = [s.clone() for s in base]
        for w, s in zip(want, base):
            for r in range(3):
                for b in range(3):
                    if r not in out:
                        w[slots[r, b]] = s[slots[r, parents[r, b]]]
        B.rwkvq_state_reorder(states, parents.int().cuda(), slots=slots.int().cuda())
        torch.cuda.synchronize()
        assert B.rwkvq_device_status() == (1 if out else 0)
        assert all(torch.equal(s, w) for s, w in zip(states, want))

    run(parents, slots, [])
    for value in (-1, 3, 1 << 30, -(1 << 31)):
        p = parents.clone()
        p[1, 2] = value
        run(p, slots, [1])
    for value in (-1, 12, 2 ** 31 - 1):
        s = slots.clone()
        s[2, 1] = value
        run(parents, s, [2])
    for r, b, value, out in ((1, 0, 2, [1]), (2, 2, 0, [2]), (0, 2, 1, [0]), (2, 1, 9, [2])):       # a slot that an earlier entry has
        s = slots.clone()
        s[r, b] = value
        run(parents, s, out)


@pytest.mark.parametrize("R,K,shape", [(2000, 5, (4,)), (700, 64, (8,)), (40, 33, (2000,)), (16384, 64, (4,))])
def test_long_lists(R, K, shape):
    """Slots of an earlier request, far in front, leave a request as it was; all others move."""
    g = torch.Generator().manual_seed(R)
    n = R * K + 100
    slots = torch.randperm(n, generator=g)[:R * K].view(R, K)
    parents = torch.randint(0, K, (R, K), generator=g)
    again = torch.randint(1, R, (5,), generator=g).unique().tolist()
    for r in again:
        slots[r, r % K] = slots[r // 3, (r * 7) % K]
    state = torch.randn((n, *shape), generator=g).cuda()
    if n > 1 << 20:
        state, slots = state[:1 << 20], slots % (1 << 20)          # some are repeated by that, too
    want, flat = state.clone(), slots.view(-1)
    first = torch.full((state.shape[0],), R * K, dtype=torch.int64).scatter_reduce_(0, flat, torch.arange(R * K), "amin")
    good = (first[flat] == torch.arange(R * K)).view(R, K).all(1)
    assert not good[again].any() and good.sum() > R // 2
    want[slots[good].view(-1).cuda()] = state[torch.gather(slots, 1, parents)[good].view(-1).cuda()]
    B.rwkvq_state_reorder([state], parents.int().cuda(), slots=slots.int().cuda())
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 1 and torch.equal(state, want)


def test_reorder_captured_for_other_parents():
    states = states_of(6, [("f32", (2, 64, 64)), ("f16", (512,))])
    parts = B.make_state_parts(states)
    parents = torch.tensor([[0, 1, 2], [0, 1, 2]], dtype=torch.int32, device="cuda")
    B.rwkvq_state_reorder(parts, parents)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rwkvq_state_reorder(parts, parents)
    for p in ([[1, 1, 0], [2, 0, 1]], [[0, 0, 0], [0, 1, 1]]):
        before = [s.clone() for s in states]
        parents.copy_(torch.tensor(p, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        at = torch.tensor([3 * r + v for r, row in enumerate(p) for v in row], device="cuda")
        assert all(torch.equal(s, b[at]) for s, b in zip(states, before))


def test_states_behind_32_bits():
    n = 5
    big = torch.empty((n, 1 << 28), device="cuda")                       # slots a GB apart
    parts = [big[:, :1024], big[:, (1 << 28) - 1024:]]
    for p in parts:
        p.copy_(torch.randn((n, 1024), device="cuda"))
    reorder(parts, torch.tensor([[4, 0, 1, 2, 3]]))
