"""Low-rank adapters (rwkvq_lowrank): the terms that numbers are taken apart into for the tensor cores are all there.  An adapter that is the identity gives x back; what y has in front is
x rounded to fewer bits, the other way round, so that the bits behind those are all that is left, whatever y's type."""
import pytest
import torch

from paper_2505_03803_b200 import binding as B
from tests.test_lowrank_gpu import HALF_ULP, LEAST, TYPES

pytestmark = pytest.mark.gpu

N = 128


@pytest.mark.parametrize("form", ["rows", "list", "wide"])
@pytest.mark.parametrize("x,w,y", [(x, w, y) for x in TYPES for w in ("f16", "bf16") for y in TYPES])
def test_an_identity_gives_back_all_of_x(x, w, y, form):
    T = 2048 if form == "wide" else 40
    g = torch.Generator().manual_seed(T)
    xs = (torch.rand((T, N), generator=g) + 1.0) * torch.pow(2.0, torch.randint(-4, 5, (T, N), generator=g).float()) * (torch.randint(0, 2, (T, N), generator=g) * 2 - 1)
    xs = xs.to(TYPES[x])
    front = -xs.to(torch.bfloat16 if y == "f32" else TYPES[y])
    eye = torch.eye(N).to(TYPES[w]).view(1, N, N).cuda()
    out = front.to(TYPES[y]).cuda()
    adapter = torch.zeros(T if form == "rows" else 2 if form == "list" else 1, dtype=torch.int32, device="cuda")
    B.rwkvq_lowrank(xs.cuda(), eye, eye, out, adapter, seq_start=torch.tensor([0, 33, T], dtype=torch.int32, device="cuda") if form == "list" else None)
    torch.cuda.synchronize()
    assert B.rwkvq_device_status() == 0
    left = xs.double() + front.double()
    # Up to three terms, in each of the two products, are added up by a tensor core that may cut off 2^-23 of what it adds to; beside f16 weights x of 32 bits is off by up to 2^-24, A x
    # by 2^-22.  A term that is missing is 2^-16 of x, or more.
    tol = (6 * 2.0 ** -23 + (2.0 ** -22 + 2.0 ** -24 if w == "f16" else 0.0)) * xs.double().abs()
    tol += HALF_ULP[y] * (left.abs() + tol) + LEAST[y]
    err = (out.double().cpu() - left).abs()
    assert (err <= tol).all(), f"max err/tol {(err / tol).max().item()}, {(err > tol).double().mean().item()} of all"
