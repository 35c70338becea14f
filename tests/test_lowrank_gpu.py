"""Low-rank adapters (rwkvq_lowrank) against their definition in 64 bits."""
import math

import pytest
import torch

from paper_2505_03803_b200 import binding as B
from paper_2505_03803_b200 import inputs
from tests import helpers as H

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}           # half the distance of the smallest numbers
E24 = 2.0 ** -24


class Case:
    """Inputs of a call, on the CPU in the types of the call."""

    def __init__(self, seed, lens, ic, oc, rank, adapter, x="f16", w="bf16", y="f32", ranks=None, scale=True, mix=None, pad=0, front=0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.ic, self.oc, self.rank, self.xt, self.wt, self.yt, self.mix = lens, ic, oc, rank, x, w, y, mix
        self.adapter, self.front, self.T = adapter, front, front + sum(lens) + pad
        self.n = max([a for a in adapter] + [0]) + 2
        r = lambda *s: torch.randn(s, generator=g)
        self.x = r(self.T, ic).to(TYPES[x])
        self.x[:, :3] *= 20
        self.A, self.B = (r(self.n, rank, ic) / ic ** 0.5).to(TYPES[w]), r(self.n, oc, rank).to(TYPES[w])
        self.y = r(self.T, oc).to(TYPES[y])
        self.ranks = ranks if ranks is None else torch.tensor((ranks + [0] * self.n)[:self.n], dtype=torch.int32)
        self.scale = torch.rand(self.n, generator=g) + 0.5 if scale else None
        self.x_prev = r(self.T, ic).to(TYPES[x]) if mix == "rows" else None
        self.xprev0 = r(len(lens), ic).to(TYPES[x]) if mix == "first" else None
        self.mu = H.pack_mu(H.random_mu_codes(seed, ic)) if mix else None

    def starts(self):
        s = [self.front]
        for l in self.lens:
            s.append(s[-1] + l)
        return s

    def call(self, listed=True, stream=None, **over):
        up = lambda t: None if t is None else t.cuda()
        k = dict(x=up(self.x), A=up(self.A), B=up(self.B), y=up(self.y), adapter=torch.tensor(self.adapter, dtype=torch.int32, device="cuda"),
                 seq_start=torch.tensor(self.starts(), dtype=torch.int32, device="cuda") if listed else None, ranks=up(self.ranks), scale=up(self.scale),
                 x_prev=up(self.x_prev), xprev0=up(self.xprev0), mu_desc=self.mu.desc if self.mu else None, mu_image=self.mu.dev if self.mu else None)
        k.update(over)
        B.rwkvq_lowrank(**k, stream=stream)
        torch.cuda.synchronize()
        return k["y"]

    def expected(self):
        """(y, tolerance): a product's terms are exact and summed in fp32 by the tensor core, which may cut off what it aligns (2^-23 a term); A x loses 2^-16 where y has 16 bits."""
        y, tol = self.y.double().clone(), torch.zeros_like(self.y, dtype=torch.float64)
        s = self.starts()
        for i, (a, t0, t1) in enumerate(zip(self.adapter, s, s[1:])):
            if a < 0 or t0 == t1:
                continue
            x = self.x[t0:t1].double()
            dx = torch.zeros_like(x)
            if self.mu:
                mu = torch.from_numpy(self.mu.w_hat)
                if self.x_prev is not None:
                    prev = self.x_prev[t0:t1].double()
                else:
                    first = self.xprev0[i:i + 1].double() if self.xprev0 is not None else torch.zeros((1, self.ic), dtype=torch.float64)
                    prev = torch.cat([first, x[:-1]])
                mixed = x + (prev - x) * mu
                dx = HALF_ULP[self.xt] * mixed.abs() + LEAST[self.xt] + 4 * E24 * (x.abs() + prev.abs())
                x = mixed
            r = self.rank if self.ranks is None else int(self.ranks[a])
            A, Bm = self.A[a, :r].double(), self.B[a, :, :r].double()
            h, mag = x @ A.T, x.abs() @ A.abs().T
            dh = dx @ A.abs().T + (self.ic + 8) * 2 * E24 * mag + (2.0 ** -16 if self.yt != "f32" else 0.0) * h.abs()
            k = 1.0 if self.scale is None else float(self.scale[a])
            d = k * (h @ Bm.T)
            dd = abs(k) * ((dh + (self.rank + 8) * 2 * E24 * h.abs()) @ Bm.abs().T)
            y[t0:t1] += d
            tol[t0:t1] = dd + (HALF_ULP[self.yt] + E24) * (y[t0:t1].abs() + dd) + LEAST[self.yt]
        return y, tol


def check(c, **kw):
    got = c.call(**kw).double().cpu()
    ref, tol = c.expected()
    assert torch.isfinite(got).all()
    err = (got - ref).abs()
    assert (err <= tol).all(), f"max err/tol {(err / tol.clamp(min=1e-300)).max().item()} at {torch.nonzero(err > tol)[:3].tolist()}"
    assert B.rwkvq_device_status() == 0


@pytest.mark.parametrize("x,w,y", [(x, w, y) for x in TYPES for w in ("f16", "bf16") for y in TYPES])
def test_types(x, w, y):
    check(Case(1, [5, 1, 40], 200, 136, 24, [1, 0, 2], x, w, y, mix="first"))


@pytest.mark.parametrize("mix", [None, "rows", "first"])
@pytest.mark.parametrize("x,w,y", [(x, w, y) for x in TYPES for w in ("f16", "bf16") for y in TYPES])
def test_types_of_long_sequences(x, w, y, mix):
    """Rows enough for the wide tiles, some of them full, others with a row or with most of them."""
    check(Case(2, [300, 1, 129, 56], 328, 264, 40, [1, 0, 2, -1], x, w, y, mix=mix, pad=3))


@pytest.mark.parametrize("ic,oc", [(8, 8), (16, 24), (32, 16), (40, 1000), (264, 8), (512, 4096), (2048, 2048), (4104, 72), (7168, 264), (9000, 40)])
@pytest.mark.parametrize("rank", [8, 16, 40, 128])
def test_sizes(ic, oc, rank):
    check(Case(ic + oc + rank, [1, 3], ic, oc, rank, [0, 1]))
    check(Case(ic + oc + rank, [19], ic, oc, rank, [1], "bf16", "bf16", "bf16"), listed=False)


@pytest.mark.parametrize("rank", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 100, 127, 128])
def test_ranks_of_their_own(rank):
    c = Case(rank, [1, 2, 33, 1], 328, 200, 128, [0, 1, 2, 2], ranks=[rank, 128, max(1, rank // 2)], w="f16" if rank % 2 else "bf16")
    for a in range(3):          # what lies behind an adapter's rank is not read into anything
        c.A[a, int(c.ranks[a]):] = math.nan
        c.B[a, :, int(c.ranks[a]):] = math.inf
    check(c)


def test_rank_zero_and_no_adapter_leave_the_rows_as_they_were():
    c = Case(3, [1, 4, 20, 1, 30], 64, 48, 16, [0, -1, 1, -1, 2], "bf16", "bf16", "bf16", ranks=[16, 0, 16])
    y = c.call()
    assert torch.equal(y[1:25].cpu(), c.y[1:25]) and torch.equal(y[25:26].cpu(), c.y[25:26])
    check(c)


@pytest.mark.parametrize("lens", [[0], [1], [0, 0, 5, 0], [15, 16, 17, 0, 1], [1] * 40 + [100] + [1] * 7, [129, 64, 63, 65], [300]])
def test_ragged(lens):
    c = Case(sum(lens), lens, 136, 88, 32, [i % 5 - 1 for i in range(len(lens))], mix="first", pad=5, front=3)
    y = c.call()
    n = 3 + sum(lens)
    assert torch.equal(y[:3].cpu(), c.y[:3]) and torch.equal(y[n:].cpu(), c.y[n:]), "rows of no sequence"
    check(c)


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f16", "f16"), ("f16", "bf16"), ("f32", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("lens", [[3, 70, 1, 40, 33] * 6, [1, 2] * 60, [65] * 150])
def test_many_tiles_of_long_rows(x, w, lens):
    """More tiles than the machine has clusters for, so that a block has all columns and its buffers go round, with tiles that are partly filled."""
    c = Case(len(lens), lens, 2056, 392, 40, [i % 4 - 1 for i in range(len(lens))], x, w, "f32", mix="first" if x != "bf16" else None)
    check(c)


@pytest.mark.parametrize("n,adapters", [(1, 1), (2, 1), (16, 1), (17, 1), (33, 2), (50, 7), (96, 96), (300, 3)])
@pytest.mark.parametrize("mix", [None, "rows", "first", "zeros"])
def test_one_row_a_sequence(n, adapters, mix):
    g = torch.Generator().manual_seed(n)
    adapter = [int(v) - (1 if n > 2 else 0) for v in torch.randint(0, adapters + (1 if n > 2 else 0), (n,), generator=g)]
    c = Case(n, [1] * n, 264, 144, 16, adapter, mix=mix)
    a, b = c.call(listed=False), c.call(listed=True)
    assert torch.equal(a, b) or (a - b).abs().max() < 1e-4
    check(c, listed=False)
    check(c, listed=True)


@pytest.mark.parametrize("T", [1, 2, 16, 100, 203])
@pytest.mark.parametrize("mix", ["rows", "first", "zeros"])
def test_token_shift_of_a_prompt(T, mix):
    check(Case(T, [T], 512, 256, 16, [0], "bf16", "bf16", "bf16", mix=mix), listed=False)
    check(Case(T, [T], 512, 256, 16, [0], "f16", "f16", "f32", mix=mix), listed=False)


def test_the_shift_is_that_of_the_products():
    """The rows as rwkvq_gemv mixes them: an adapter that is the identity gives back x_mix, rounded as there."""
    ic = 128
    c = Case(9, [1] * 5, ic, ic, 128, [0] * 5, "f16", "f16", "f32", scale=False, mix="rows")
    c.A[0], c.B[0], c.y = torch.eye(128).half(), torch.eye(128).half(), torch.zeros_like(c.y)
    x, p, mu = c.x.float(), c.x_prev.float(), torch.from_numpy(c.mu.w_hat).float()
    mixed = (x.double() + ((p - x).double() * mu.double())).float().half()         # the difference rounded, product and sum with one rounding: fp32 of an exact double
    assert torch.equal(c.call(listed=False).cpu(), mixed.float())


@pytest.mark.parametrize("n,adapters", [(40, 1100), (257, 1), (700, 700), (1500, 40)])
def test_many_rows_or_many_adapters(n, adapters):
    g = torch.Generator().manual_seed(n)
    adapter = (torch.randint(0, adapters, (n,), generator=g) if adapters < n else torch.randperm(adapters, generator=g)[:n]).tolist()
    adapter[n // 2] = -1
    c = Case(n, [1] * n, 72, 40, 8, adapter, "bf16", "f16" if n % 2 else "bf16", "f32" if n % 2 else "f16")
    check(c, listed=False)


def test_strided_rows():
    c = Case(11, [70], 136, 72, 16, [0], "bf16", "bf16", "f16", mix="rows")
    wide = lambda t, k: torch.full((t.shape[0], t.shape[1] + k), math.nan, dtype=t.dtype).cuda()
    x, p, y = wide(c.x, 8), wide(c.x_prev, 24), wide(c.y, 16)
    x[:, :136], p[:, 24:], y[:, 8:80] = c.x.cuda(), c.x_prev.cuda(), c.y.cuda()
    got = c.call(listed=False, x=x[:, :136], x_prev=p[:, 24:], y=y[:, 8:80])
    assert torch.equal(got.contiguous(), c.call(listed=False)) and torch.isnan(y[:, :8]).all() and torch.isnan(y[:, 80:]).all()


def test_a_row_of_infinities_or_nan_is_its_own():
    for bad in (math.inf, -math.inf, math.nan):
        for x in TYPES:
            c = Case(12, [20, 1, 20], 72, 40, 16, [0, 0, 0], x)
            clean = c.call()
            c.x[7, 5] = bad
            got = c.call()
            keep = [i for i in range(41) if i != 7]
            assert torch.equal(got[keep], clean[keep]) and not torch.isfinite(got[7]).any()


@pytest.mark.parametrize("lens", [[1, 2, 1, 5], [70, 33], [330, 64]])
@pytest.mark.parametrize("x", TYPES)
def test_an_infinity_beside_f16_weights(x, lens):
    """The rows of such inputs are brought to a common size by their largest finite number."""
    for bad in (math.inf, -math.inf, math.nan):
        c = Case(15, lens, 712, 40, 16, [0] * len(lens), x, "f16")
        clean = c.call()
        c.x[7, 300] = bad
        got = c.call()
        keep = [i for i in range(c.T) if i != 7]
        assert torch.equal(got[keep], clean[keep]) and not torch.isfinite(got[7]).any()


@pytest.mark.parametrize("lens", [[1] * 30, [5, 1, 12, 12], [30], [100, 64], [330, 64]])
@pytest.mark.parametrize("x,mix", [("f32", None), ("f32", "rows"), ("bf16", None), ("bf16", "rows"), ("bf16", "first")])
def test_rows_of_all_sizes_beside_f16_weights(x, mix, lens):
    """Rows from 2^-100 to 2^100, some with one number far above the others, some all zero."""
    c = Case(sum(lens), lens, 1032, 72, 40, [i % 2 for i in range(len(lens))], x, "f16", "f32", mix=mix)
    c.y.zero_()
    g = torch.Generator().manual_seed(5)
    size = torch.pow(2.0, torch.randint(-100, 101, (c.T, 1), generator=g).float()) if mix != "first" else torch.full((c.T, 1), 2.0 ** 90)
    c.x = (c.x.float() * size).to(c.x.dtype)
    if c.x_prev is not None:
        c.x_prev = (c.x_prev.float() * size).to(c.x.dtype)
    c.x[::3, 700] *= 2.0 ** 20
    c.x[1::4] = 0
    if c.x_prev is not None:
        c.x_prev[1::4] = 0
    got = c.call().double().cpu()
    ref, tol = c.expected()
    # beside f16 weights a number is off by up to 2^-39 of the largest of its row, A x by up to 2^-38 of its own
    most = c.x.double().abs().amax(1, keepdim=True)
    if c.mu:
        prev = c.x_prev.double() if c.x_prev is not None else torch.cat([c.xprev0[:1].double(), c.x[:-1].double()]).abs()
        most = most + (most + prev.abs().amax(1, keepdim=True)) * float(abs(c.mu.w_hat).max())
    for a, t0, t1 in zip(c.adapter, c.starts(), c.starts()[1:]):
        A, Bm, k = c.A[a].double().abs(), c.B[a].double().abs(), float(c.scale[a])
        h = most[t0:t1] * A.sum(1)
        tol[t0:t1] += k * ((2.0 ** -39 * h + 2.0 ** -38 * h.amax(1, keepdim=True)) @ Bm.T)
    assert torch.isfinite(got).all()
    err = (got - ref).abs()
    assert (err <= tol).all(), f"max err/tol {(err / tol.clamp(min=1e-300)).max().item()}"
    assert B.rwkvq_device_status() == 0


def test_bad_lists_leave_a_sequence_out():
    good = Case(13, [5, 30, 4], 64, 48, 16, [0, 1, 0])
    want, before = good.call().cpu(), good.y
    n = good.n
    for adapter, out in (([0, n, 0], [1]), ([0, -2, 0], [1]), ([n + 5, 1, -3], [0, 2]), ([0, 1 << 30, 0], [1])):
        got = good.call(adapter=torch.tensor(adapter, dtype=torch.int32, device="cuda")).cpu()
        assert B.rwkvq_device_status() == 1
        for i, (a, b) in enumerate(zip(good.starts(), good.starts()[1:])):
            assert torch.equal(got[a:b], (before if i in out else want)[a:b])
    for starts, out in (([0, 5, 35, 40], [2]), ([0, 5, 3, 39], [1, 2]), ([-1, 5, 35, 39], [0]), ([0, 5, 35, 2 ** 31 - 1], [2])):
        got = good.call(seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda")).cpu()
        assert B.rwkvq_device_status() == 1
        for i, (a, b) in enumerate(zip(good.starts(), good.starts()[1:])):
            if i in out:
                assert torch.equal(got[a:b], before[a:b]) or i == 1
            elif i != 2:
                assert torch.equal(got[a:b], want[a:b])
    ranks = torch.full((n,), 16, dtype=torch.int32, device="cuda")
    ranks[1] = 17
    got = good.call(ranks=ranks).cpu()
    assert B.rwkvq_device_status() == 1 and torch.equal(got[5:35], before[5:35]) and torch.equal(got[:5], want[:5])
    # one row a sequence
    c = Case(14, [1] * 20, 64, 48, 16, [0] * 20)
    want = c.call(listed=False).cpu()
    adapter = torch.zeros(20, dtype=torch.int32)
    adapter[3] = 99
    got = c.call(listed=False, adapter=adapter.cuda()).cpu()
    assert B.rwkvq_device_status() == 1 and torch.equal(got[3], c.y[3]) and torch.equal(got[4:], want[4:])


def test_the_same_bits_every_time():
    c = Case(15, [200, 1, 1], 1024, 512, 64, [0, 1, 1], "f16", "bf16", "f32", mix="first")
    y = c.call()
    for _ in range(3):
        assert torch.equal(c.call(), y)


def test_captured_and_replayed_for_other_lists():
    c = Case(16, [3, 60, 1], 256, 128, 32, [0, 1, 2])
    d = Case(16, [3, 60, 1], 256, 128, 32, [2, -1, 0])
    d.lens, d.A, d.B, d.scale, d.n = [40, 0, 24], c.A, c.B, c.scale, c.n
    up = {k: getattr(c, k).cuda() for k in ("x", "A", "B", "y", "scale")}
    adapter, starts = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (c.adapter, c.starts()))
    run = lambda: B.rwkvq_lowrank(up["x"], up["A"], up["B"], up["y"], adapter, seq_start=starts, scale=up["scale"])
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for case in (c, d):
        adapter.copy_(torch.tensor(case.adapter, dtype=torch.int32))
        starts.copy_(torch.tensor(case.starts(), dtype=torch.int32))
        up["y"].copy_(c.y)
        graph.replay()
        torch.cuda.synchronize()
        case.y, case.x = c.y, c.x
        assert torch.equal(up["y"], case.call())


def test_two_streams():
    cs = [Case(s, [200], 512, 512, 32, [0], "bf16", "bf16", "f32") for s in (17, 18)]
    want = [c.call(listed=False) for c in cs]
    ups = [{k: getattr(c, k).cuda() for k in ("x", "A", "B", "y", "scale")} for c in cs]
    adapter = torch.zeros(1, dtype=torch.int32, device="cuda")
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for _ in range(5):
        for u, c, s in zip(ups, cs, streams):
            with torch.cuda.stream(s):
                u["y"].copy_(c.y, non_blocking=False)
                B.rwkvq_lowrank(u["x"], u["A"], u["B"], u["y"], adapter, scale=u["scale"])
    torch.cuda.synchronize()
    assert all(torch.equal(u["y"], w) for u, w in zip(ups, want))


def test_behind_32_bits():
    """An adapter and a row whose elements lie behind 2^31."""
    ic, oc, rank, n = 8192, 64, 128, 2100
    A = torch.empty((n, rank, ic), dtype=torch.bfloat16, device="cuda")
    Bm = torch.zeros((n, oc, rank), dtype=torch.bfloat16, device="cuda")
    c = Case(19, [1, 1], ic, oc, rank, [0, 0], "f16", "bf16", "f32", scale=False)
    want = c.call(listed=False)
    A[n - 1], Bm[n - 1] = c.A[0].cuda(), c.B[0].cuda()
    got = c.call(listed=False, A=A, B=Bm, adapter=torch.full((2,), n - 1, dtype=torch.int32, device="cuda"))
    assert torch.equal(got, want)
    row = 1 << 27
    big = torch.empty((17 * row + ic,), dtype=torch.float16, device="cuda").as_strided((18, ic), (row, 1))
    c = Case(20, [18], ic, oc, rank, [0], "f16", "bf16", "f32", scale=False)
    want = c.call(listed=False)
    big.copy_(c.x)
    assert torch.equal(c.call(listed=False, x=big), want)


def test_tensors_of_other_shapes_are_refused():
    c = Case(16, [4], 64, 48, 16, [0], mix="rows")
    cuda = lambda t: t.cuda()
    for over in (dict(x_prev=cuda(c.x_prev)[:3]), dict(x_prev=cuda(c.x_prev).unsqueeze(0)), dict(x_prev=cuda(c.x_prev).float()), dict(A=cuda(c.A)[:, :8]), dict(A=cuda(c.A).transpose(0, 1)),
                 dict(B=cuda(c.B)[:1]), dict(B=cuda(c.B).float()), dict(y=cuda(c.y)[:3]), dict(y=cuda(c.y).t()), dict(x=cuda(c.x).t().contiguous().t()), dict(adapter=torch.zeros(1, dtype=torch.int64, device="cuda")),
                 dict(scale=torch.ones(1, device="cuda")), dict(ranks=torch.ones(c.n, device="cuda")), dict(mu_image=None), dict(x=cuda(c.x).double()), dict(adapter=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises((ValueError, B.RwkvqError)):
            c.call(listed=False, **over)
