"""Low-rank adapters (rwkvq_lowrank): sequences that have none."""
import pytest
import torch

from paper_2505_03803_b200 import binding as B
from tests.test_lowrank_gpu import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("bf16", "f16"), ("f32", "f16")])
@pytest.mark.parametrize("mix", [None, "first"])
@pytest.mark.parametrize("lens", [[1] * 20, [3, 40, 1, 17, 5], [300, 64, 700, 65, 500]])
def test_tiles_without_an_adapter(x, w, mix, lens):
    """Whether a tile has an adapter is known while its rows are already being read, mixed or brought to a common size: tiles with and without in one call, time after time."""
    n = len(lens)
    c = Case(n + sum(lens), lens, 520, 72, 16, [(-1, 0, 1, -1, 2)[i % 5] for i in range(n)], x, w, "f32", ranks=[16, 0, 16], mix=mix)
    check(c)
    want = c.call()
    for i, (a, t0, t1) in enumerate(zip(c.adapter, c.starts(), c.starts()[1:])):
        if a < 0 or a == 1:
            assert torch.equal(want[t0:t1].cpu(), c.y[t0:t1])
    up = {k: getattr(c, k).cuda() for k in ("x", "A", "B", "ranks", "scale")}
    adapter, starts = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (c.adapter, c.starts()))
    xprev0 = None if c.xprev0 is None else c.xprev0.cuda()
    ys = [c.y.cuda() for _ in range(50)]
    for y in ys:
        B.rwkvq_lowrank(up["x"], up["A"], up["B"], y, adapter, seq_start=starts, ranks=up["ranks"], scale=up["scale"], xprev0=xprev0, mu_desc=c.mu.desc if c.mu else None,
                        mu_image=c.mu.dev if c.mu else None)
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0 and all(torch.equal(y, want) for y in ys)
    none = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    assert torch.equal(c.call(adapter=none).cpu(), c.y) and B.rwkvq_device_status() == 0


@pytest.mark.parametrize("lens", [[5, 30, 4], [500, 3000, 400]])
def test_rows_of_bad_lists(lens):
    """Which rows a list that does not rise, or leaves the rows there are, computes and which it leaves, each of them."""
    c = Case(13, lens, 64, 48, 16, [0, 1, 0])
    want, before = c.call().cpu(), c.y
    n0, n1, T = lens[0], lens[0] + lens[1], sum(lens)
    for starts, ranges in (([0, n0, n1, T + 1], [(0, n1)]),                    # the last ends behind the rows
                           ([0, n0, n0 - 2, T], [(0, n0)]),                    # one ends before it begins, the next begins in front of an earlier entry
                           ([-1, n0, n1, T], [(n0, T)]),
                           ([0, n0, n1, 2 ** 31 - 1], [(0, n1)]),
                           ([0, n1, n0, T], [(0, n1)]),                        # the second is [n1, n0), the third lies inside the first
                           ([n0, n1, n1, n1 - 1], [])):
        got = c.call(seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda")).cpu()
        assert B.rwkvq_device_status() == 1
        if starts[0] > 0:          # the first is [n0, n1) with the adapter of the first, the second is empty, the third ends before it begins
            assert torch.equal(got[:n0], before[:n0]) and torch.equal(got[n1:], before[n1:]) and not torch.equal(got[n0:n1], before[n0:n1])
            continue
        if starts[1] == n1:        # the first takes the second's rows, too, with its own adapter
            assert torch.equal(got[:n0], want[:n0]) and torch.equal(got[n1:], before[n1:]) and not torch.equal(got[n0:n1], before[n0:n1])
            continue
        keep = torch.ones(T, dtype=torch.bool)
        for a, b in ranges:
            assert torch.equal(got[a:b], want[a:b])
            keep[a:b] = False
        assert torch.equal(got[keep], before[keep])
