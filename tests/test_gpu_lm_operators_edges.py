"""The operators around a language model's output where a first set of tests did not look."""

import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = (torch.float32, torch.float16, torch.bfloat16)
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def Bd():
    from paper_2206_07882_b200 import binding
    binding.lib()
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ------------------------------------------------------------------------------------------------------------- norm
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,at", [(3, 1, 0), (5, 64, 63), (4, 1001, 500), (2500, 640, 0), (2400, 1029, 1028), (3, 9001, 17), (2, 8192, 8191), (2, 40001, 40000)])
@pytest.mark.parametrize("gain_at", [NAN, INF, -INF])
def test_norm_with_a_gain_that_is_not_finite(Bd, dtype, rows, k, at, gain_at):
    # y is not finite where the gain is not, over h = 0 too (NaN, and 0 * inf is NaN): such a row has no boundary, its scale is NaN
    # and its codes are 0, whatever its length, its alignment or its number (one warp a row, several, rows from memory)
    g = gen(k)
    x, r = (torch.randn(rows, k, generator=g).to(dtype) for _ in range(2))
    x[1:, at] = 0
    gain = torch.rand(k, generator=g)
    sound = gain.clone()
    gain[at] = gain_at
    for residual in (None, r):
        out = None if residual is None else torch.empty_like(x, device="cuda")
        rd = None if residual is None else residual.cuda()
        codes, scale = Bd.q4_rmsnorm_quantize(x.cuda(), gain.cuda(), 1e-5, residual=rd, sum_out=out)
        assert scale.isnan().all() and (codes == 0).all()
        if residual is not None:
            assert torch.equal(out.cpu(), (x.float() + r.float()).to(dtype))
    codes, scale = Bd.q4_rmsnorm_quantize(x.cuda(), sound.cuda(), 1e-5)     # (the row itself is a sound one)
    assert torch.isfinite(scale).all()
