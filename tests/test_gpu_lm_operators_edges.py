"""The operators around a language model's output where a first set of tests did not look."""
import ctypes as C
from fractions import Fraction

import numpy as np
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


def code_of(h, gain, top):
    """127 h gain / top rounded to the nearest integer, halves to even, in rational numbers (fp32 values are such)."""
    return round(127 * Fraction(h) * Fraction(gain) / top)


def check_codes_in_rationals(Bd, x, gain, pad):
    """x [rows, m] with m gains, in rows of `pad` elements whose others are zeros."""
    rows, m = x.shape
    wide, wide_gain = torch.zeros(rows, pad), torch.ones(pad)
    wide[:, :m], wide_gain[:m] = x, gain
    codes, scale = Bd.q4_rmsnorm_quantize(wide.cuda(), wide_gain.cuda(), 1e-5)
    got = codes.cpu().view(torch.int8)
    xs, gs = x.tolist(), gain.tolist()
    for i in range(rows):
        top = max(abs(Fraction(h) * Fraction(f)) for h, f in zip(xs[i], gs))
        assert got[i, :m].tolist() == [code_of(h, f, top) for h, f in zip(xs[i], gs)]
    assert (got[:, m:] == 0).all() and torch.isfinite(scale).all()


# rows that fit a warp, wider groups, and rows from memory; and rows from memory because squares leave fp32
@pytest.mark.parametrize("pad,factor", [(256, 1.0), (1001, 1.0), (9000, 1.0), (20011, 1.0), (256, 2.0 ** 66)])
def test_norm_of_exact_halves_with_long_mantissas(Bd, pad, factor):
    # h = (2n+1) a beside 254 a: 127 h / max is n + 1/2 whatever the gain, though h gain takes 48 bits and 127 of them 55
    g = gen(pad)
    a = 2 * torch.randint(1 << 14, 1 << 15, (24, 1), generator=g) + 1
    sign = 1 - 2 * torch.randint(0, 2, (24, 127), generator=g)
    x = torch.cat([254 * a, (2 * torch.arange(127) + 1) * a * sign], 1).double()
    assert torch.equal(x.float().double(), x)
    for gain in (1.0580815, 0.70710677, 1.9999999, 3.0):
        check_codes_in_rationals(Bd, x.float() * factor, torch.full((128,), gain), pad)


@pytest.mark.parametrize("pad", [256, 20011])
def test_norm_of_fp32_next_to_halves(Bd, pad):
    # products a step of their last bits beside a half: (y - 1)(y + 1) = y^2 - 1 against y^2
    g = gen(pad)
    y = torch.randint(1 << 14, (1 << 16) - 2, (8, 1), generator=g).double()
    n = 2 * torch.arange(60).double() + 1
    below, above = n * (y - 1), n * y                         # times y + 1 and y
    for row in range(8):
        v = float(y[row])
        # max 254 y^2: n (y^2 - 1) lies below the half, n y^2 on it; max 254 (y^2 - 1): n (y^2 - 1) on it, n y^2 above it
        for top, top_gain in ((254 * v, v), (254 * (v - 1), v + 1)):
            x = torch.cat([torch.tensor([top], dtype=torch.float64), below[row], -above[row]])[None]
            gain = torch.cat([torch.tensor([top_gain], dtype=torch.float64), torch.full((60,), v + 1, dtype=torch.float64),
                              torch.full((60,), v, dtype=torch.float64)])
            assert torch.equal(x.float().double(), x)
            check_codes_in_rationals(Bd, x.float(), gain.float(), pad)
    check_codes_in_rationals(Bd, torch.randn(20, 120, generator=g), torch.randn(120, generator=g), pad)


# ----------------------------------------------------------------------------------------------------------- select
@pytest.mark.parametrize("dtype", DTYPES)
def test_select_adds_many_small_terms_to_a_large_sum(Bd, dtype):
    # A row of 16 turns, one segment: every thread meets terms of 1 first, then 15 turns whose terms are each below half of the last
    # fp32 place of its sum so far, 8e-7 of it together.  Terms of 1 are exact (2^0), the small ones good to 1e-6 of themselves, and
    # what is added to a sum in double stays; the scores lie near 0, where fp32 shows it.
    per, B, W = (2048, 33, 32) if dtype == torch.float32 else (4096, 33, 32)      # elements of a turn; more rows than block slots
    z = torch.full((B, W, 16 * per), -16.75, dtype=dtype, device="cuda")
    z[:, :, :per] = 0
    lse = float(np.log(per + 15 * per * np.exp(-16.75)))
    score = torch.full((B, W), round(lse * 64) / 64, device="cuda") - torch.arange(W, device="cuda") / 64
    r = Bd.q4_lm_beam_select(z, score)
    want = score[0, 0].double().item() - lse
    assert abs(want) < 2.0 ** -6                              # rounded to fp32 by less than 2^-31
    assert (r["parent"] == 0).all() and (r["token"].cpu() == torch.arange(W)).all()
    assert ((r["score"].double() - want).abs() < 1e-9).all(), (r["score"].double() - want).abs().max().item()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gap", [0, 1, 3])
@pytest.mark.parametrize("V", [64, 1024, 9000, 70000])
def test_select_of_beams_that_differ_in_their_tails_only(Bd, dtype, gap, V):
    # Equal scores and equal best labels, but one row holds a little more beside them: 2e-6 of its sum, several times what terms
    # and sums are off by (e^-1 by 2^-22 of itself, a handful of roundings of 2^-24).  Each keeps its own sum, the lighter tail wins.
    W, low = 2, torch.finfo(dtype).min
    for heavy in (0, 1):
        z = torch.full((1, W, V + gap), low, dtype=dtype)
        z[:, :, 3], z[:, :, V - 5] = 0.0, -1.0
        z[0, :, V // 2] = -16.0
        z[0, heavy, V // 2] = -12.75
        score = torch.full((1, W), 0.3125)
        r = Bd.q4_lm_beam_select(z.cuda()[:, :, :V], score.cuda())
        total = score.double() - torch.logsumexp(z[:, :, :V].double(), 2)
        assert (total[0, 1 - heavy] - total[0, heavy]).item() > 1.9e-6
        assert r["parent"].tolist() == [[1 - heavy, heavy]] and r["token"].tolist() == [[3, 3]]
        got = r["score"].cpu().double()[0]
        assert (got - torch.stack([total[0, 1 - heavy], total[0, heavy]])).abs().max() < 8e-7
        assert 1.6e-6 < (got[0] - got[1]).item() < 2.4e-6


@pytest.mark.parametrize("dtype", DTYPES)
def test_select_of_equal_rows_and_of_nearly_equal_ones(Bd, dtype):
    # rows that begin at different places of 16 bytes: equal ones are told apart by their number, one that differs in its last label
    # alone is a row of its own (2e-6 of its sum), whether it comes before, between or behind them
    V, W = 4099, 12
    g = gen(5)
    row = torch.full((V,), -30.0)
    row[torch.randperm(V - 1, generator=g)[:W]] = -torch.arange(W).float() / 8
    for other in ((0,), (5,), (11,), (2, 7), (0, 11)):
        z = row.to(dtype).repeat(1, W, 1)
        for w in other:
            z[0, w, V - 1] = -11.25                           # 1.3e-5 beside a sum of about 6.6
        r = Bd.q4_lm_beam_select(z.cuda(), torch.zeros(1, W, device="cuda"))
        order = [w for w in range(W) if w not in other] + list(other)
        assert r["parent"].tolist() == [order] and len(set(r["token"][0].tolist())) == 1
        got = r["score"].cpu()[0]
        n = W - len(other)
        assert len(set(got[:n].tolist())) == 1 and (len(set(got[n:].tolist())) == 1)
        want = -torch.logsumexp(z[0].double(), 1)[order]
        assert (got.double() - want).abs().max() < 1.3e-6 and got[n - 1] > got[n]


# ---------------------------------------------------------------------------------------------------------- reorder
def test_reorder_of_more_tensors_than_a_launch_is_checked_before_any_moves(Bd):
    B, W = 2, 4
    parent = torch.tensor([[1, 0, 3, 2], [2, 2, -1, 0]], dtype=torch.int32, device="cuda")
    fresh = lambda n: [(torch.randn(B, W, 24, device="cuda"), torch.zeros(B, W, 24, device="cuda")) for _ in range(n)]
    n = Bd.launch_count()
    # the 17th (and the last of 40) reads what the first one writes
    for count, at in ((17, 16), (40, 39), (40, 20)):
        pairs = fresh(count)
        pairs[at] = (pairs[0][1], pairs[at][1])
        with pytest.raises(Bd.Q4Error) as err:
            Bd.q4_beam_reorder(pairs, parent)
        assert err.value.code == -6 and all((d == 0).all() for _, d in pairs)
        pairs = fresh(count)
        pairs[0] = (pairs[at][1][:, :, :], pairs[0][1])       # and the other way round
        with pytest.raises(Bd.Q4Error) as err:
            Bd.q4_beam_reorder(pairs, parent)
        assert err.value.code == -6 and all((d == 0).all() for _, d in pairs)
    # a 17th that is refused by its shape, its type, its device or in place
    for bad in ((torch.zeros(B, W, 3, device="cuda"), torch.zeros(B, W, 4, device="cuda")),
                (torch.zeros(B, W, 3, device="cuda"), torch.zeros(B, W, 3, device="cuda", dtype=torch.int32)),
                (torch.zeros(B, W, 3), torch.zeros(B, W, 3)), (torch.zeros(W, B, 3, device="cuda"),) * 2, (fresh(1)[0][0],) * 2):
        pairs = fresh(16) + [bad]
        with pytest.raises((ValueError, Bd.Q4Error)):
            Bd.q4_beam_reorder(pairs, parent)
        assert all((d == 0).all() for _, d in pairs[:16])
    assert Bd.launch_count() == n
    pairs = fresh(40)
    Bd.q4_beam_reorder(pairs, parent)
    assert Bd.launch_count() == n + 3
    for s, d in pairs:
        for b in range(B):
            for w, p in enumerate(parent[b].tolist()):
                assert torch.equal(d[b, w], s[b, p] if p >= 0 else torch.zeros_like(d[b, w]))


# ------------------------------------------------------------------------------------------------- buffers of a call
def test_select_keeps_its_buffers_where_shapes_alternate(Bd):
    # many counters and little workspace, then the other way round: after one of each nothing is allocated any more
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        a = torch.randn(64, 16, 64, device="cuda"), torch.randn(64, 16, device="cuda")
        b = torch.randn(1, 32, 400000, device="cuda"), torch.randn(1, 32, device="cuda")
        want = [Bd.q4_lm_beam_select(*s) for s in (a, b)]
        key = next(k for k in Bd._select_scratch if k[1] == stream.cuda_stream)
        kept = [t.data_ptr() for t in Bd._select_scratch[key]]
        n = Bd._select_scratch[key][1].numel()
        assert n >= Bd.workspace_bytes(Bd.WS_LM_SELECT, b[0].shape) and Bd._select_scratch[key][0].numel() >= 64 * 17
        for _ in range(3):
            for s, w in zip((a, b), want):
                got = Bd.q4_lm_beam_select(*s)
                assert all(torch.equal(got[k], w[k]) for k in w)
                assert [t.data_ptr() for t in Bd._select_scratch[key]] == kept
    stream.synchronize()


def test_select_with_the_callers_workspace_keeps_none_of_its_own(Bd):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        z, score = torch.randn(1, 32, 400000, device="cuda"), torch.randn(1, 32, device="cuda")
        need = Bd.workspace_bytes(Bd.WS_LM_SELECT, z.shape)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        got = Bd.q4_lm_beam_select(z, score, workspace=ws)
        held = sum(t.numel() * t.element_size() for k, e in Bd._select_scratch.items() if k[1] == stream.cuda_stream for t in e)
        assert held < need                                    # counters alone
        want = Bd.q4_lm_beam_select(z, score)
        assert all(torch.equal(got[k], want[k]) for k in want)
    stream.synchronize()


# ----------------------------------------------------------------------------------------------------------- linear
@pytest.mark.parametrize("M,N,K", [(5, 300, 256), (16, 256, 4096), (1024, 4096, 256)])
def test_linear_tells_of_a_wait_that_ran_out_without_being_asked(Bd, M, N, K):
    # a layer has a status word of its own, which a call without one uses
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda").view(torch.uint8)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w, torch.rand(N, device="cuda"), N, K, K, 8))
    xq, sx = torch.randint(0, 255, (M, K), dtype=torch.uint8, device="cuda"), torch.rand(M, device="cuda")
    want = Bd.q4_linear_token_scales(xq, sx, lin)
    assert Bd.q4_poll_status(lin.status) == 0
    assert Bd.lib().q4_test_wait_expiry_set(C.c_int32(1), C.c_uint32(1 << 12)) == 0
    try:
        Bd.q4_linear_token_scales(xq, sx, lin)
        assert Bd.q4_poll_status(lin.status) == -8
        own = torch.zeros(1, dtype=torch.int32, device="cuda")
        lin.status.zero_()
        Bd.q4_linear_token_scales(xq, sx, lin, status=own)
        assert Bd.q4_poll_status(own) == -8 and Bd.q4_poll_status(lin.status) == 0
    finally:
        Bd.lib().q4_test_wait_expiry_set(C.c_int32(0), C.c_uint32(0))
    assert torch.equal(Bd.q4_linear_token_scales(xq, sx, lin), want) and Bd.q4_poll_status(lin.status) == 0


@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (33, 257, 640), (300, 1001, 1283)])
@pytest.mark.parametrize("x_dtype", [torch.float32, torch.float16])
def test_linear_of_the_frameworks_own_activations_and_weights(Bd, M, N, K, x_dtype):
    # codes of quantize_pack_int4 with one MAX boundary a row, weights of DeviceMat.from_float_max
    g = gen(M + N)
    x, w = torch.randn(M, K, generator=g).to(x_dtype), torch.randn(N, K, generator=g)
    x[M // 2] = 0                                             # (its boundary is 1)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat.from_float_max(w.numpy(), 8), torch.randn(N, generator=g).cuda())
    xq, sx = Bd.quantize_pack_int4(x.cuda(), Bd.Act(1.0, 1.0, 0, 8, 1), mode=1, n_groups=M, k_pad=lin.w.k_pad)
    got = Bd.q4_linear_token_scales(xq, sx, lin).cpu().double()
    values = lambda q, s: q.cpu().view(torch.int8).double() * s.cpu().double()[:, None]
    acc = values(xq, sx) @ values(lin.w.q, lin.w.scale).t()
    want = acc + lin.bias.cpu().double()
    assert ((got - want).abs() <= (3 * 2.0 ** -24 * acc.abs() + 2.0 ** -23 * want.abs()) * 1.01 + 1e-38).all()
    # and both are the real product to what 8 bits leave: half a step an operand and element, and what the rounded scales add
    steps = (sx.cpu().double() / 2 * 1.01)[:, None] * w.double().abs().sum(1) + \
        (lin.w.scale.cpu().double() / 2 * 1.01) * (x.double().abs() + sx.cpu().double()[:, None]).sum(1)[:, None]
    assert ((got - lin.bias.cpu().double() - x.double() @ w.double().t()).abs() <= steps).all()


# -------------------------------------------------------------------------------------------------- rows of nearly 2^31
@pytest.mark.parametrize("with_residual", [False, True])
def test_norm_of_the_longest_row(Bd, with_residual):
    k = 2 ** 31 - 32
    x = torch.ones((1, k), dtype=torch.float16, device="cuda")
    x[0, 0], x[0, -1] = 0.0, -2.0                             # 127 / 2 is a half: 64
    residual = torch.zeros_like(x) if with_residual else None
    codes, scale = Bd.q4_rmsnorm_quantize(x, torch.ones(k, device="cuda"), 1e-5, residual=residual, sum_out=residual)
    codes = codes.view(torch.int8)
    assert codes.shape == (1, k) and codes[0, 0].item() == 0 and codes[0, -1].item() == -127 and bool((codes[0, 1:-1] == 64).all())
    want = 2 / np.sqrt((k + 2) / k + 1e-5) / 127
    assert abs(scale.item() - want) <= 2.0 ** -24 * want * 1.01
    assert residual is None or torch.equal(residual, x)


@pytest.mark.parametrize("level", [0.0, 2097152.0])          # (the latter is summed by differences from the maximum)
def test_select_over_the_longest_row(Bd, level):
    V = 2 ** 31 - 1
    z = torch.full((1, 1, V), level, dtype=torch.bfloat16, device="cuda")
    score = torch.zeros(1, 1, device="cuda")
    tol = 5e-6 + 2.0 ** -24 * np.log(V) * 1.01
    r = Bd.q4_lm_beam_select(z, score)                        # all alike: the first label
    assert r["parent"].item() == 0 and r["token"].item() == 0 and abs(r["score"].item() + np.log(V)) <= tol
    z[0, 0, 0], z[0, 0, V - 1] = -INF, level + 16384 if level else 8.0
    r = Bd.q4_lm_beam_select(z, score)
    want = 0.0 if level else 8 - np.log(V - 2 + np.exp(8.0))
    assert r["token"].item() == V - 1 and abs(r["score"].item() - want) <= tol
