"""4-bit products of rows with one value far above the others.

Bound.  With q' = 1 + q/128 and z' = 1 + z/128, at most 1 + 15/128 < 1.12, a group's sum of
x (q' - z') is built in fp32 by at most 8 matrix instructions (two sums of up to 128 rows, 32
each), whose accumulator stays below 1.12 sum |x|.  Four roundings or truncations of 2^-23
in each are 8 * 4 * 2^-23 * 1.12 of sum |x|, times 128 s: 2^-10.8 s sum |x|, here as 2^-11
1.2.  The result is rounded once, 2^-8 of it; one group, so that nothing else is added.
"""
import pytest
import torch

from paper_2606_26344_amd import gmlp, w4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


@pytest.mark.parametrize("T", [4, 8, 32, 64])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_an_outlier_at_a_weight_of_zero(T, group, zeros):
    gen = torch.Generator().manual_seed(T + group)
    K, N = group, 520
    q = torch.randint(0, 16, (K, N), generator=gen, dtype=torch.uint8)
    z = torch.randint(0, 16, (1, N), generator=gen, dtype=torch.uint8) if zeros else torch.full((1, N), 8, dtype=torch.uint8)
    s = ((torch.rand((1, N), generator=gen) + 0.5) * 0.01).to(torch.bfloat16)
    x = torch.randn((T, K), generator=gen).to(torch.bfloat16)
    for t in range(T):
        x[t, t % 16] = 1e4 * (-1) ** t
    q[:16] = z
    y = w4.matmul(x.cuda(), w4.pack(q.cuda(), s.cuda(), z.cuda() if zeros else None, group=group)).cpu().double()
    ref = x.double() @ ((q.double() - z.double()) * s.double())
    bound = 2.0 ** -8 * ref.abs() + 1.2 * 2.0 ** -11 * x.double().abs().sum(1, keepdim=True) * s.double()
    ratio = ((y - ref).abs() / bound).max().item()
    print("T=%d group=%d zeros=%s: max |err|/bound = %.3f" % (T, group, zeros, ratio), flush=True)
    assert ratio <= 1.0
