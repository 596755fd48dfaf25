"""The operators around a language model's output against plain 64-bit computations of the same formulas: norm with 8-bit
codes, linear layer with token scales, beam selection over a vocabulary, reordering of states."""
import ctypes as C
import math
import os
import subprocess
import sys

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


def strided(t, gap, fill=NAN):
    """t on the device, its rows `gap` elements further apart than they are long, the elements between them `fill`."""
    wide = torch.full(t.shape[:-1] + (t.shape[-1] + gap,), fill, dtype=t.dtype)
    wide[..., :t.shape[-1]] = t
    return wide.cuda()[..., :t.shape[-1]]


# ------------------------------------------------------------------------------------------------------------- norm
# A scale: sums of squares in fp32 over chains of at most 64 terms, each rounded by 2^-24, halved by the root, and four
# single roundings behind it.
SCALE_RTOL = (64 / 2 + 4) * 2.0 ** -24


def norm_oracle(x, gain, eps, residual=None):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    d = h.double()
    v = d * gain.double()
    top = v.abs().amax(1)
    root = torch.sqrt((d * d).mean(1) + eps)
    none = top == 0
    codes = torch.round(127 * v / torch.where(none, torch.ones_like(top), top)[:, None])
    scale = torch.where(none, torch.ones_like(top), top / torch.where(none, torch.ones_like(root), root)) / 127
    bad = ~torch.isfinite(d).all(1)
    codes[bad], scale[bad] = 0, NAN
    return h, codes, scale


def check_norm(Bd, x, gain, eps=1e-5, residual=None, gap=0, k_pad=None):
    xs, rs = strided(x, gap), None if residual is None else strided(residual, gap + 3)
    out = None if residual is None else strided(torch.zeros_like(x), 1)
    codes, scale = Bd.q4_rmsnorm_quantize(xs, gain.cuda(), eps, residual=rs, sum_out=out, k_pad=k_pad)
    h, want, want_scale = norm_oracle(x, gain, eps, residual)
    k = x.shape[1]
    got = codes.cpu().view(torch.int8)
    assert got.shape[1] == (Bd.pad32(k) if k_pad is None else k_pad)
    assert torch.equal(got[:, :k].double(), want)
    assert (got[:, k:] == 0).all()
    np.testing.assert_allclose(scale.cpu().double().numpy(), want_scale.numpy(), rtol=SCALE_RTOL, atol=0)
    if residual is not None:
        assert torch.equal(torch.nan_to_num(out.cpu()), torch.nan_to_num(h))
        assert torch.equal(out.cpu().isnan(), h.isnan())
        whole = out.as_strided((x.shape[0], k + 1), (k + 1, 1)).cpu()
        assert whole[:-1, k].isnan().all()             # between the rows nothing was written


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,gap", [(1, 1, 0), (3, 31, 0), (5, 32, 8), (16, 1024, 0), (7, 1001, 0), (9, 1280, 1), (33, 640, 64),
                                        (2, 4096, 0), (3, 8192, 8), (2, 20011, 5), (2, 40960, 0), (300, 96, 0)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_norm(Bd, dtype, rows, k, gap, with_residual):
    g = gen(rows * 7919 + k)
    channel = torch.exp(torch.randn(k, generator=g))
    x = (torch.randn(rows, k, generator=g) * channel).to(dtype)
    r = (4 * torch.randn(rows, k, generator=g)).to(dtype) if with_residual else None
    check_norm(Bd, x, 1 + 0.2 * torch.randn(k, generator=g), residual=r, gap=gap)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,k_pad", [(3, 1, 64), (5000, 33, 160), (2500, 640, 1024), (4, 4000, 4096), (2400, 2049, 2112)])
def test_norm_into_longer_rows(Bd, dtype, rows, k, k_pad):
    # few and many rows (a row on a warp, on two, on more), with codes of 0 behind them
    g = gen(k)
    x, r = (torch.randn(rows, k, generator=g).to(dtype) for _ in range(2))
    check_norm(Bd, x, torch.randn(k, generator=g), residual=r, k_pad=k_pad)
    check_norm(Bd, x, torch.randn(k, generator=g), gap=8 - k % 8, k_pad=k_pad)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k", [(2400, 1536), (2400, 2048), (2500, 4096), (2400, 8000), (2400, 1537)])
def test_norm_of_many_rows(Bd, dtype, rows, k):
    g = gen(k)
    x, r = (torch.randn(rows, k, generator=g).to(dtype) for _ in range(2))
    check_norm(Bd, x, torch.randn(k, generator=g), residual=r)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vectors", [1, 32, 66, 97, 129, 160, 192, 193, 256, 257, 320, 380, 385, 448, 512, 514, 640, 760, 770, 896, 1024, 1026, 1280, 1530, 1538, 1700,
                                     2048, 2050, 2560, 3070, 3584, 4096])
def test_norm_of_every_group(Bd, dtype, vectors):
    # rows of so many 16-byte vectors: few rows, enough for one wave of blocks, and many, so that every number of threads of a row
    # and of vectors of a thread is met; rows that begin at a multiple of 16 bytes, and one element behind it
    k = vectors * (4 if dtype == torch.float32 else 8)
    wave = (1900 if dtype == torch.float32 else 3600) if vectors <= 256 else 1300 if vectors <= 512 else 600
    for rows in [5] + ([wave, 7300 if vectors <= 320 else 3600 if vectors <= 512 else 1300] if vectors <= 1024 else [600] if vectors <= 2048 else []):
        g = torch.Generator(device="cuda").manual_seed(rows * 31 + vectors)
        gain = 1 + 0.2 * torch.randn(k, generator=g, device="cuda")
        for odd in (0, 1):
            x, r, out = (torch.randn(rows, k + 8 * odd, generator=g, device="cuda").to(dtype)[:, odd:k + odd] for _ in range(3))
            for residual in (None, r):
                codes, scale = Bd.q4_rmsnorm_quantize(x, gain, 1e-5, residual=residual, sum_out=None if residual is None else out)
                h, want, want_scale = norm_oracle(x, gain, 1e-5, residual)
                assert torch.equal(codes.view(torch.int8)[:, :k].double(), want)
                assert ((scale.double() - want_scale).abs() <= SCALE_RTOL * want_scale).all()
                assert residual is None or torch.equal(out, h)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [64, 1003, 9001])
def test_norm_of_values_next_to_a_half(Bd, dtype, k):
    # a row maximum of 127 (or 254) makes many quotients exact halves, which go to the even neighbour
    g = gen(k)
    x = torch.randint(-254, 255, (6, k), generator=g).float() / 2
    x[:, 0] = torch.tensor([127.0, -127.0, 127.0, 63.5, 31.75, 127.0])
    x = x.clamp(-127, 127)
    for gain in (torch.ones(k), torch.full((k,), 0.25), 1 + torch.randint(-3, 4, (k,), generator=g) / 8):
        check_norm(Bd, x.to(dtype), gain)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_of_rows_at_the_edges(Bd, dtype):
    k, g = 300, gen(3)
    info = torch.finfo(dtype)
    x = torch.randn(12, k, generator=g).to(dtype)
    x[0] = 0
    x[1, 5] = INF
    x[2, 299] = NAN
    x[3] = 0
    x[3, 7] = info.tiny
    x[4] = info.max
    x[5, ::3] = -info.max
    x[6] = x[6] * 1e-4
    x[7, 0] = -INF
    x[8] = info.tiny
    gain = torch.randn(k, generator=g)
    for eps in (1e-5, 1e-30):
        check_norm(Bd, x, gain, eps=eps)
    check_norm(Bd, x, torch.zeros(k))
    check_norm(Bd, x[6:7] * 0, gain, eps=0.0)
    check_norm(Bd, x, gain, eps=0.0)


@pytest.mark.parametrize("k", [320, 333])
def test_norm_adds_in_place(Bd, k):
    g = gen(k)
    x, r = (torch.randn(9, k, generator=g).to(torch.bfloat16) for _ in range(2))
    gain = torch.rand(k, generator=g)
    h, want, _ = norm_oracle(x, gain, 1e-6, r)
    for into in (0, 1):
        xd, rd = x.cuda(), r.cuda()
        codes, _ = Bd.q4_rmsnorm_quantize(xd, gain.cuda(), 1e-6, residual=rd, sum_out=(xd, rd)[into])
        assert torch.equal((xd, rd)[into].cpu(), h)
        assert torch.equal((xd, rd)[1 - into].cpu(), (x, r)[1 - into])
        assert torch.equal(codes.cpu().view(torch.int8)[:, :k].double(), want)


def test_norm_counts_as_one_quantizer_and_takes_no_rows(Bd):
    n = Bd.quantizer_calls()
    x = torch.ones(4, 64, device="cuda")
    Bd.q4_rmsnorm_quantize(x, x[0].clone(), 1e-5)
    assert Bd.quantizer_calls() == n + 1
    codes, scale = Bd.q4_rmsnorm_quantize(x[:0], x[0].clone(), 1e-5)
    assert codes.shape == (0, 64) and scale.shape == (0,)


# ----------------------------------------------------------------------------------------------------------- linear
def linear_inputs(M, N, K, seed, bias=True, most=127):
    g = gen(seed)
    pad = (K + 31) // 32 * 32
    x, w = torch.zeros(M, pad, dtype=torch.int8), torch.zeros(N, pad, dtype=torch.int8)
    x[:, :K] = torch.randint(-most, most + 1, (M, K), generator=g).to(torch.int8)
    w[:, :K] = torch.randint(-most, most + 1, (N, K), generator=g).to(torch.int8)
    sx, sw = 0.01 + 0.05 * torch.rand(M, generator=g), (0.2 + torch.rand(N, generator=g)) / (127 * math.sqrt(K))
    return x, w, sx, sw, torch.randn(N, generator=g) if bias else None


def check_linear(Bd, x, w, sx, sw, b, dtype, gap=0, k=None):
    M, N = x.shape[0], w.shape[0]
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w.cuda().view(torch.uint8), sw.cuda(), N, k or w.shape[1], w.shape[1], 8),
                                   None if b is None else b.cuda())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    wide = torch.full((M + 2, N + gap), 7.0, dtype=dtype, device="cuda")
    got = Bd.q4_linear_token_scales(x.cuda().view(torch.uint8), sx.cuda(), lin, out=wide[1:M + 1, :N], status=status)
    assert Bd.q4_poll_status(status) == 0
    whole = wide.cpu().double()
    assert (whole[0] == 7).all() and (whole[M + 1] == 7).all() and (whole[:, N:] == 7).all()   # nothing beside the output
    acc = x.double() @ w.double().t() * sx.double()[:, None] * sw.double()
    want = acc if b is None else acc + b.double()
    # the sum becomes fp32 and is multiplied by a rounded product of scales; then one rounding to fp32 and one to dtype
    tol = (3 * 2.0 ** -24 * acc.abs() + (2.0 ** -24 + torch.finfo(dtype).eps / 2) * want.abs()) * 1.01 + torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    err = (got.cpu().double() - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 128, 32), (2, 7, 31), (3, 129, 129), (16, 2050, 512), (16, 1024, 4096), (17, 127, 1283),
                                   (33, 1001, 640), (64, 384, 256), (65, 130, 128), (128, 256, 384), (129, 129, 33), (200, 520, 1000),
                                   (257, 1001, 1283), (1000, 96, 64), (1024, 640, 2048), (31, 5000, 96), (5, 20000, 256)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear(Bd, M, N, K, dtype):
    x, w, sx, sw, b = linear_inputs(M, N, K, M + N + K, bias=(M + N) % 2 == 0)
    check_linear(Bd, x, w, sx, sw, b, dtype, gap=(M + K) % 3, k=K)


@pytest.mark.parametrize("M,N,K", [(2048, 2050, 160), (70, 14500, 64), (1800, 2000, 1283), (600, 5000, 31), (9000, 640, 260), (257, 40000, 96)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_of_many_tiles(Bd, M, N, K, dtype):
    x, w, sx, sw, b = linear_inputs(M, N, K, M + N + K, bias=N % 4 == 0)
    check_linear(Bd, x, w, sx, sw, b, dtype, gap=M % 3, k=K)


@pytest.mark.parametrize("M,N,K", [(13, 2000, 4100), (5, 259, 2050), (250, 130, 4100), (400, 130, 9003), (29, 100, 4100), (51, 1021, 14000),
                                   (400, 259, 6000), (250, 130, 14000), (200, 1000, 6000), (128, 512, 8192), (9, 5000, 14000), (30, 5100, 14000),
                                   (16, 4097, 2048), (32, 4100, 4096), (60, 4095, 4096), (128, 1025, 2048), (30, 1021, 2048), (3, 65, 4096)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_of_few_tiles_and_a_long_sum(Bd, M, N, K, dtype):
    # 16, 32 and 64 tokens a tile, each of whose sums is shared by 4 or 8 CTAs
    x, w, sx, sw, b = linear_inputs(M, N, K, M + N + K, bias=N % 4 == 0)
    check_linear(Bd, x, w, sx, sw, b, dtype, gap=M % 3, k=K)


@pytest.mark.parametrize("M", [2, 70, 300])
def test_linear_of_the_longest_rows(Bd, M):
    # every product 2^14: the sum of 131040 of them is just below 2^31
    x, w, sx, sw, _ = linear_inputs(M, 5, 131040, 1, bias=False)
    x[:] = -128
    w[0], w[1] = -128, 127
    check_linear(Bd, x, w, sx, sw, None, torch.float32)


@pytest.mark.parametrize("M,N,K", [(5, 300, 256), (16, 256, 4096), (100, 700, 300), (1024, 4096, 256)])
def test_linear_whose_wait_runs_out_stores_nothing(Bd, M, N, K):
    # one tile a CTA, a split, wider tiles, pairs of CTAs: the producers issue no copy, every thread leaves, the status says so
    x, w, sx, sw, b = linear_inputs(M, N, K, 11)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w.cuda().view(torch.uint8), sw.cuda(), N, w.shape[1], w.shape[1], 8), b.cuda())
    out, status = torch.full((M, N), 3.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    xd, sxd = x.cuda().view(torch.uint8), sx.cuda()
    assert Bd.lib().q4_test_wait_expiry_set(C.c_int32(1), C.c_uint32(1 << 12)) == 0
    try:
        Bd.q4_linear_token_scales(xd, sxd, lin, out=out, status=status)
        assert Bd.q4_poll_status(status) == -8
    finally:
        Bd.lib().q4_test_wait_expiry_set(C.c_int32(0), C.c_uint32(0))
    assert (out == 3.0).all()
    status.zero_()
    Bd.q4_linear_token_scales(xd, sxd, lin, out=out, status=status)
    assert Bd.q4_poll_status(status) == 0
    assert torch.equal(out, Bd.q4_linear_token_scales(xd, sxd, lin)) and not (out == 3.0).all()


@pytest.mark.parametrize("M,N,K", [(300, 11000, 1000), (700, 2050, 4100), (100, 14001, 2048), (129, 9000, 2001), (3000, 700, 5000), (500, 4097, 700)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_linear_of_pairs(Bd, M, N, K, dtype):
    # tiles of 128 and 256 tokens by two CTAs, one round of tiles and several, ragged at both ends
    x, w, sx, sw, b = linear_inputs(M, N, K, M + N + K, bias=N % 2 == 0)
    check_linear(Bd, x, w, sx, sw, b, dtype, gap=M % 3, k=K)


def test_linear_of_a_split_whose_wait_runs_out_stores_nothing(Bd):
    test_linear_whose_wait_runs_out_stores_nothing(Bd, 250, 130, 14000)   # 8 CTAs for 64 tokens
    test_linear_whose_wait_runs_out_stores_nothing(Bd, 400, 259, 6000)    # 4
    test_linear_whose_wait_runs_out_stores_nothing(Bd, 300, 11000, 1000)  # pairs of CTAs, tiles of 128 tokens


def test_linear_rows_without_a_scale_stay_alone(Bd):
    x, w, sx, sw, b = linear_inputs(40, 200, 96, 5)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w.cuda().view(torch.uint8), sw.cuda(), 200, 96, 96, 8), b.cuda())
    want = Bd.q4_linear_token_scales(x.cuda().view(torch.uint8), sx.cuda(), lin)
    sx[7] = NAN
    got = Bd.q4_linear_token_scales(x.cuda().view(torch.uint8), sx.cuda(), lin)
    assert got[7].isnan().all()
    keep = torch.arange(40) != 7
    assert torch.equal(got.cpu()[keep], want.cpu()[keep])
    assert Bd.q4_linear_token_scales(torch.empty((0, 96), dtype=torch.uint8, device="cuda"), sx.cuda()[:0], lin).shape == (0, 200)


def test_linear_agrees_with_the_layer_of_one_scale(Bd):
    # all token scales equal: the same sums and the same roundings as q4_linear_forward's
    x, w, sx, sw, b = linear_inputs(300, 256, 640, 9)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w.cuda().view(torch.uint8), sw.cuda(), 256, 640, 640, 8), b.cuda())
    act = Bd.Act(0.03125, 32.0, 0, 8, 1)
    one = Bd.q4_linear_forward(x.cuda().view(torch.uint8), act, lin)
    two = Bd.q4_linear_token_scales(x.cuda().view(torch.uint8), torch.full((300,), 0.03125, device="cuda"), lin)
    assert torch.equal(one, two)


# ----------------------------------------------------------------------------------------------------------- select
# log-sum-exp: terms with the base-2 unit's 2^-22 and their argument's rounding (t e^-t 2^-24 <= 2^-25), added in fp32 over
# chains of at most 64 terms, the rest in double.
LSE_TOL = 2.0 ** -22 + 2.0 ** -25 + 64 * 2.0 ** -24


def select_oracle(logits, score, done, eos, rho):
    z = logits.double()
    B, W, V = z.shape
    total = torch.full((B, W, V), -INF, dtype=torch.float64)
    for b in range(B):
        for w in range(W):
            s = score[b, w].double()
            if not torch.isfinite(s):
                continue
            if done is not None and done[b, w]:
                total[b, w, eos] = s
                continue
            row = z[b, w]
            if row.isnan().any() or (row == INF).any() or (row == -INF).all():
                continue
            total[b, w] = s + (row - torch.logsumexp(row, 0) + rho)
    total = total.reshape(B, W * V)
    total[~torch.isfinite(total.float())] = -INF
    # score, parent, then the beam's own order, logit and label (where a score of 1e38 takes up a logit's difference)
    label = np.tile(np.arange(V), W)
    index = torch.from_numpy(np.stack([np.lexsort((label, -torch.nan_to_num(z[b], nan=-INF, posinf=INF, neginf=-INF).flatten().numpy(),
                                                   np.repeat(np.arange(W), V), -total[b].numpy()))[:W] for b in range(B)]))
    value = total.gather(1, index)
    empty = value == -INF
    parent, token = torch.where(empty, -1, index // V), torch.where(empty, -1, index % V)
    return parent, token, value, (token == eos) & ~empty


def check_select(Bd, logits, score, done=None, eos=-1, rho=0.0, gap=0):
    r = Bd.q4_lm_beam_select(strided(logits, gap), score.cuda(), done=None if done is None else done.cuda(), eos=eos, rho=rho)
    parent, token, value, ended = select_oracle(logits, score, done, eos, rho)
    assert torch.equal(r["parent"].cpu().long(), parent)
    assert torch.equal(r["token"].cpu().long(), token)
    assert torch.equal(r["done"].cpu().bool(), ended)
    got = r["score"].cpu().double()
    live = torch.isfinite(value)
    assert (got[~live] == -INF).all()
    assert ((got - value).abs()[live] <= LSE_TOL + 2.0 ** -24 * value.abs()[live] * 1.01).all()
    return r


@pytest.mark.parametrize("B,W,V", [(1, 1, 1), (1, 1, 40), (2, 3, 7), (3, 2, 64), (1, 16, 1024), (2, 32, 33), (4, 5, 1001), (1, 32, 5000),
                                   (2, 12, 50257), (1, 7, 130001), (70, 16, 1024), (40, 8, 8192), (3, 31, 16383)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_select(Bd, B, W, V, dtype):
    g = gen(B * 31 + W * 7 + V)
    logits = (2.0 * torch.randn(B, W, V, generator=g)).to(dtype)
    score = 3 * torch.randn(B, W, generator=g) - 20
    check_select(Bd, logits, score, rho=0.25, gap=(0, 3, 8)[V % 3])
    if V > 2:
        done = torch.rand(B, W, generator=g) < 0.3
        score[:, W // 2:] = torch.where(torch.rand(B, W - W // 2, generator=g) < 0.3, -INF, score[:, W // 2:])
        logits[torch.rand(B, W, V, generator=g) < 0.1] = -INF
        logits[0, 0, 1] = 1.0
        check_select(Bd, logits, score, done=done.to(torch.uint8), eos=V // 2, gap=1)


@pytest.mark.parametrize("V", [3, 41, 1001, 9001, 50257])
@pytest.mark.parametrize("dtype", DTYPES)
def test_select_of_equal_beams_in_rows_that_begin_anywhere(Bd, V, dtype):
    # equal beams of equal scores are told apart by their number alone, wherever their rows begin in memory
    g, W = gen(V), 12
    row, other = torch.randn(V, generator=g).to(dtype), torch.randn(V, generator=g).to(dtype)
    logits = torch.stack([row, other, row, row, other, row, row, other, row, row, other, row])[None].contiguous()
    score = torch.tensor([[0.0, 0.1, 0.0, 0.0, 0.1, -0.0, 0.0, 0.1, -0.25, -0.25, 0.1, 0.0]])
    for gap in (0, 1, 2):
        check_select(Bd, logits, score, gap=gap)
        check_select(Bd, logits, torch.zeros(1, W), gap=gap, rho=0.5)


@pytest.mark.parametrize("V", [40, 1024, 9000, 40000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_of_equal_and_ordered_logits(Bd, V, dtype):
    W = 16
    score = torch.zeros(1, W)
    ramp = torch.arange(V, dtype=torch.float32) / 64
    for logits in (torch.zeros(V), ramp, -ramp, torch.where(torch.arange(V) % 3 == 0, 1.0, 0.0),
                   torch.where(torch.arange(V) >= V - 20, 2.0, 0.0)):
        rows = logits.to(dtype).expand(1, W, V).contiguous()
        check_select(Bd, rows, score)                       # equal rows of equal scores: ties between beams too
        check_select(Bd, rows, score - torch.arange(W) * 1e-3)


@pytest.mark.parametrize("W,V", [(32, 300000), (1, 2000000), (16, 131072)])
def test_select_of_long_rows(Bd, W, V):
    # rows of many segments: all equal (more candidates than a list holds, in every segment and over them), and ordinary
    score = torch.linspace(0, -1, W)[None]
    check_select(Bd, torch.zeros(1, W, V, dtype=torch.float16), score)
    g = torch.Generator(device="cuda").manual_seed(V)
    logits = torch.randn(1, W, V, generator=g, device="cuda")
    r = Bd.q4_lm_beam_select(logits, score.cuda())
    total = (torch.log_softmax(logits.double(), 2) + score.cuda().double()[:, :, None]).view(1, -1)
    value, index = total.topk(W)
    assert torch.equal(r["parent"].long(), index // V) and torch.equal(r["token"].long(), index % V)
    assert ((r["score"].double() - value).abs() <= LSE_TOL + 2.0 ** -24 * value.abs() * 1.01).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [50, 3001])
def test_select_of_masked_and_broken_rows(Bd, dtype, V):
    g, W = gen(V), 8
    low = torch.finfo(dtype).min
    logits = torch.randn(3, W, V, generator=g).to(dtype)
    score = torch.randn(3, W, generator=g)
    logits[0, 0] = -INF
    logits[0, 1, 3] = NAN
    logits[0, 2, V - 1] = INF
    logits[0, 3] = low
    logits[0, 4, 5:] = low
    logits[0, 5, 1:] = -INF
    logits[0, 6, :V - 1] = -INF
    logits[1, :, 10:] = -INF
    logits[1, :, :9] = low
    logits[2] = NAN
    done = torch.zeros(3, W, dtype=torch.uint8)
    done[2, 3] = 1
    score[2, 5] = NAN
    done[1, 2] = 1
    logits[1, 2] = NAN                                       # an ended beam's logits are not looked at
    check_select(Bd, logits, score, done=done, eos=4, rho=-0.5)
    score[1] = -3.4e38                                       # below fp32 with a mask's lowest value added
    check_select(Bd, logits, score, done=done, eos=0)
    check_select(Bd, torch.full((2, W, V), -INF).to(dtype), score[:2])
    check_select(Bd, logits, torch.full((3, W), -INF))


def test_select_leaves_the_tail_empty(Bd):
    # the first step of a search: one beam, fewer labels than beams
    logits, score = torch.randn(2, 16, 5, generator=gen(1)), torch.full((2, 16), -INF)
    score[:, 0] = 0
    r = check_select(Bd, logits, score)
    assert (r["parent"][:, 5:] == -1).all() and (r["parent"][:, :5] == 0).all()


def test_select_takes_a_workspace_with_anything_in_it(Bd):
    g = gen(4)
    logits, score = torch.randn(2, 16, 3000, generator=g).cuda(), torch.randn(2, 16, generator=g).cuda()
    want = Bd.q4_lm_beam_select(logits, score)
    need = Bd.workspace_bytes(Bd.WS_LM_SELECT, (2, 16, 3000))
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        got = Bd.q4_lm_beam_select(logits, score, workspace=ws[:need])
        assert all(torch.equal(got[k], want[k]) for k in want)
        assert (ws[need:] == 0xFF).all()
        ws[:need] = 0x7F


# ---------------------------------------------------------------------------------------------------------- reorder
def reorder_oracle(src, dst, parent, dim):
    want = dst.clone()
    B, W = parent.shape
    s, d = src.movedim((dim, dim + 1), (0, 1)), want.movedim((dim, dim + 1), (0, 1))
    for b in range(B):
        for w in range(W):
            p = int(parent[b, w])
            if 0 <= p < W:
                d[b, w] = s[b, p]
    return want


def parents(B, W, seed):
    p = torch.randint(-1, W, (B, W), generator=gen(seed), dtype=torch.int32)
    if W > 3:
        p[0, 1], p[-1, 2] = W, -7                           # out of range: left alone
    return p


@pytest.mark.parametrize("shape,dim,dtype", [((1, 1, 4), 0, torch.uint8), ((1, 16, 2048), 0, torch.float32), ((3, 5, 7), 0, torch.uint8),
                                             ((2, 9), 0, torch.int32), ((64, 16, 96), 0, torch.float16), ((4, 2, 6, 8, 40, 24), 1, torch.bfloat16),
                                             ((2, 3, 8, 1, 33, 5), 1, torch.uint8), ((3, 1, 4, 130), 1, torch.float32), ((2, 2, 2, 5000), 1, torch.bfloat16)])
def test_reorder(Bd, shape, dim, dtype):
    g = gen(len(shape))
    src, dst = (torch.randint(0, 100, shape, generator=g).to(dtype) for _ in range(2))
    parent = parents(*shape[dim:dim + 2], seed=sum(shape))
    out = dst.cuda()
    Bd.q4_beam_reorder([(src.cuda(), out)], parent.cuda(), dim=dim)
    assert torch.equal(out.cpu(), reorder_oracle(src, dst, parent, dim))


@pytest.mark.parametrize("used", [0, 1, 3, 16, 31, 32])
@pytest.mark.parametrize("H", [64, 20, 3])
def test_reorder_moves_the_used_part_of_a_cache(Bd, used, H):
    L, B, W, heads, S = 3, 2, 5, 4, 32
    g = gen(used + H)
    src, dst = (torch.randn(L, B, W, heads, S, H, generator=g).to(torch.bfloat16) for _ in range(2))
    parent = parents(B, W, used)
    want = dst.clone()
    want[:, :, :, :, :used] = reorder_oracle(src[:, :, :, :, :used], dst[:, :, :, :, :used], parent, 1)
    a, b = src.cuda(), dst.cuda()
    Bd.q4_beam_reorder([(a[:, :, :, :, :used], b[:, :, :, :, :used])], parent.cuda(), dim=1)
    assert torch.equal(b.cpu(), want)
    # the same from a cache of another length and another order of layers and beams
    c = torch.zeros(B, W, L, heads, S + 5, H, dtype=torch.bfloat16)
    c[:, :, :, :, :S] = src.permute(1, 2, 0, 3, 4, 5)
    b = dst.cuda()
    Bd.q4_beam_reorder([(c.cuda().permute(2, 0, 1, 3, 4, 5)[:, :, :, :, :used], b[:, :, :, :, :used])], parent.cuda(), dim=1)
    assert torch.equal(b.cpu(), want)


def test_reorder_of_many_tensors_of_different_rows(Bd):
    B, W, g = 3, 7, gen(2)
    shapes = [(B, W, n) for n in (1, 2, 3, 5, 8, 16, 33, 64, 129, 1000, 4096, 10000)] * 2
    pairs = [tuple(torch.randint(0, 256, s, generator=g).to(torch.uint8) for _ in range(2)) for s in shapes]
    parent = parents(B, W, 5)
    dev = [(s.cuda(), d.cuda()) for s, d in pairs]
    n = Bd.launch_count()
    Bd.q4_beam_reorder(dev, parent.cuda())
    assert Bd.launch_count() == n + 2                       # 16 tensors in one launch
    for (s, d), (_, out) in zip(pairs, dev):
        assert torch.equal(out.cpu(), reorder_oracle(s, d, parent, 0))


# -------------------------------------------------------------------------------------------------------- together
def search_step(Bd, s):
    """One step of a search whose network is one residual block and an output layer."""
    codes, scale = Bd.q4_rmsnorm_quantize(s["x"], s["gain"], 1e-5, residual=s["res"], sum_out=s["sum"])
    hidden = Bd.q4_linear_token_scales(codes, scale, s["layer"], out_dtype=torch.bfloat16)
    codes, scale = Bd.q4_rmsnorm_quantize(hidden, s["gain"], 1e-5, residual=s["sum"], sum_out=s["sum2"])
    logits = Bd.q4_linear_token_scales(codes, scale, s["head"])
    r = Bd.q4_lm_beam_select(logits.view(s["B"], s["W"], -1), s["score"], done=s["done"], eos=1, rho=0.1)
    Bd.q4_beam_reorder([(s["sum2"].view(s["B"], s["W"], -1), s["moved"])], r["parent"])
    return dict(r, logits=logits, moved=s["moved"])


def search_state(Bd, B, W, D, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    lin = lambda n, k: Bd.DeviceLinear.from_mat(Bd.DeviceMat(torch.randint(-127, 128, (n, k), generator=g, device="cuda").to(torch.int8).view(torch.uint8),
                                                             torch.rand(n, generator=g, device="cuda") / 500, n, k, k, 8), rand(n))
    bf = lambda *shape: rand(*shape).to(torch.bfloat16)
    return dict(B=B, W=W, x=bf(B * W, D), res=bf(B * W, D), sum=bf(B * W, D), sum2=bf(B * W, D), moved=bf(B, W, D), gain=1 + 0.1 * rand(D),
                layer=lin(D, D), head=lin(V, D), score=rand(B, W), done=(rand(B, W) > 1).to(torch.uint8))


@pytest.mark.parametrize("B,W,D,V", [(1, 4, 64, 100), (2, 16, 640, 5000), (20, 8, 256, 1024)])
def test_a_step_of_a_search_by_itself_and_replayed(Bd, B, W, D, V):
    s = search_state(Bd, B, W, D, V, seed=V)
    r = search_step(Bd, s)
    logits = r["logits"].cpu()
    # the selection and the move on what the layers gave, the layers on what the norms gave
    parent, token, value, _ = select_oracle(logits.view(B, W, V), s["score"].cpu(), s["done"].cpu(), 1, float(np.float32(0.1)))
    assert torch.equal(r["parent"].cpu().long(), parent) and torch.equal(r["token"].cpu().long(), token)
    h, codes, scale = norm_oracle(s["x"].cpu(), s["gain"].cpu(), 1e-5, s["res"].cpu())
    w = s["layer"].w
    hidden = codes @ w.q.cpu().view(torch.int8).double().t() * scale[:, None] * w.scale.cpu().double() + s["layer"].bias.cpu().double()
    near = hidden + h.double()
    assert ((s["sum2"].cpu().double() - near).abs() <= 2.0 ** -8 * (hidden.abs() + near.abs()) * 1.01 + 1e-4).all()
    eager = {k: v.clone() for k, v in r.items()}
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = search_step(Bd, s)
    before = s["moved"].clone()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], eager[k]) for k in eager)
    # other inputs in the same buffers
    other = search_state(Bd, B, W, D, V, seed=V + 1)
    for k in ("x", "res", "score", "done"):
        s[k].copy_(other[k])
    s["moved"].copy_(before)
    graph.replay()
    torch.cuda.synchronize()
    replayed = {k: v.clone() for k, v in out.items()}
    s["moved"].copy_(before)
    with torch.cuda.stream(side):
        again = search_step(Bd, s)
    torch.cuda.synchronize()
    assert all(torch.equal(again[k], replayed[k]) for k in replayed)


def test_steps_on_two_streams_at_once(Bd):
    states = [search_state(Bd, 2, 8, 256, 4000, seed) for seed in (1, 2)]
    want = [{k: v.clone() for k, v in search_step(Bd, s).items()} for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    got = [[], []]
    for _ in range(20):
        for i, (s, st) in enumerate(zip(states, streams)):
            with torch.cuda.stream(st):
                got[i].append(search_step(Bd, s))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(r[k], want[i][k]) for k in want[i])


def shifted(t, at, gap):
    """t on the device as columns `at` and on of a wider tensor that is NaN elsewhere."""
    wide = torch.full(t.shape[:-1] + (at + t.shape[-1] + gap,), NAN, dtype=t.dtype)
    wide[..., at:at + t.shape[-1]] = t
    return wide.cuda()[..., at:at + t.shape[-1]]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [1, 2, 3, 5, 7])
def test_views_that_begin_anywhere(Bd, dtype, at):
    # rows that begin at every place of a 16-byte granule, the first and the last element of a tensor among them
    g = gen(at)
    for rows, k in ((6, 777), (2500, 200), (3, 5), (2400, 1029)):
        x, r = (torch.randn(rows, k, generator=g).to(dtype) for _ in range(2))
        gain = torch.randn(k, generator=g)
        h, want, want_scale = norm_oracle(x, gain, 1e-5, r)
        for gap in (0, 1, 8):
            xd, rd, sd = shifted(x, at, gap), shifted(r, at + 1, gap), shifted(torch.zeros_like(x), 2 * at, gap + 1)
            codes, scale = Bd.q4_rmsnorm_quantize(xd, gain.cuda(), 1e-5, residual=rd, sum_out=sd)
            assert torch.equal(codes.cpu().view(torch.int8)[:, :k].double(), want) and torch.equal(sd.cpu(), h)
            np.testing.assert_allclose(scale.cpu().double().numpy(), want_scale.numpy(), rtol=SCALE_RTOL, atol=0)
            whole = sd.as_strided((rows, k + 2 * at + gap + 1), (k + 2 * at + gap + 1, 1), 0).cpu()
            assert whole[:, :2 * at].isnan().all() and whole[:, 2 * at + k:].isnan().all()
            Bd.q4_rmsnorm_quantize(xd, gain.cuda(), 1e-5, residual=rd, sum_out=rd)      # in place
            assert torch.equal(rd.cpu(), h)
    for B, W, V in ((2, 5, 1003), (1, 3, 6), (3, 16, 20011)):
        logits, score = torch.randn(B, W, V, generator=g).to(dtype), torch.randn(B, W, generator=g)
        near = Bd.q4_lm_beam_select(logits.cuda(), score.cuda())
        for gap in (0, 3):
            got = Bd.q4_lm_beam_select(shifted(logits, at, gap), score.cuda())
            assert all(torch.equal(near[n], got[n]) for n in ("parent", "token", "done"))
            # a row that begins elsewhere is summed in another order: each sum within LSE_TOL, a score rounded once
            assert ((near["score"] - got["score"]).abs() <= 2 * LSE_TOL + 2.0 ** -23 * near["score"].abs()).all()
    x, w, sx, sw, b = linear_inputs(70, 333, 96, at)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w.cuda().view(torch.uint8), sw.cuda(), 333, 96, 96, 8), b.cuda())
    want = Bd.q4_linear_token_scales(x.cuda().view(torch.uint8), sx.cuda(), lin, out_dtype=dtype)
    out = shifted(torch.zeros(70, 333, dtype=dtype), at, 2)
    Bd.q4_linear_token_scales(x.cuda().view(torch.uint8), sx.cuda(), lin, out=out)
    assert torch.equal(out, want)
    src, dst = torch.randn(2, 4, 37, generator=g).to(dtype), torch.randn(2, 4, 37, generator=g).to(dtype)
    parent = parents(2, 4, at)
    to = shifted(dst, 2 * at, 1)
    Bd.q4_beam_reorder([(shifted(src, at, 3), to)], parent.cuda())
    assert torch.equal(to.cpu(), reorder_oracle(src, dst, parent, 0))


def far_rows(t, step):
    """t [rows, k] on the device with rows `step` elements apart (more than 2^31 in all), what lies between them unread."""
    big = torch.empty((t.shape[0] - 1) * step + t.shape[1], dtype=t.dtype, device="cuda")
    view = big.as_strided(t.shape, (step, 1))
    view.copy_(t)
    return view


def test_rows_further_apart_than_32_bits_count(Bd):
    g, step = gen(12), (1 << 30) + 40
    x = torch.randn(4, 96, generator=g).to(torch.float16)
    codes, scale = Bd.q4_rmsnorm_quantize(far_rows(x, step), torch.ones(96, device="cuda"), 1e-5)
    _, want, want_scale = norm_oracle(x, torch.ones(96), 1e-5)
    assert torch.equal(codes.cpu().view(torch.int8).double(), want)
    xi, w, sx, sw, _ = linear_inputs(4, 100, 96, 3, bias=False)
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w.cuda().view(torch.uint8), sw.cuda(), 100, 96, 96, 8))
    out = far_rows(torch.zeros(4, 100, dtype=torch.float16), step)
    Bd.q4_linear_token_scales(xi.cuda().view(torch.uint8), sx.cuda(), lin, out=out)
    assert torch.equal(out.clone(), Bd.q4_linear_token_scales(xi.cuda().view(torch.uint8), sx.cuda(), lin, out_dtype=torch.float16))
    logits = torch.randn(1, 4, 300, generator=g).to(torch.float16)
    score = torch.randn(1, 4, generator=g)
    far = far_rows(logits[0], step).as_strided((1, 4, 300), (4 * step, step, 1))
    near, got = Bd.q4_lm_beam_select(logits.cuda(), score.cuda()), Bd.q4_lm_beam_select(far, score.cuda())
    assert all(torch.equal(near[k], got[k]) for k in near)
    rows = torch.randn(4, 50, generator=g).to(torch.float16)
    src, dst = far_rows(rows, step).as_strided((1, 4, 50), (4 * step, step, 1)), torch.zeros(1, 4, 50, dtype=torch.float16, device="cuda")
    Bd.q4_beam_reorder([(src, dst)], torch.tensor([[3, 2, -1, 0]], dtype=torch.int32, device="cuda"))
    assert torch.equal(dst[0].cpu(), torch.stack([rows[3], rows[2], 0 * rows[0], rows[0]]))


FIRST_CALLS = """
import torch
from paper_2206_07882_b200 import binding as Bd
torch.manual_seed(1)
x, gain = torch.randn(64, 8192, device="cuda"), torch.ones(8192, device="cuda")
wide = torch.randn(2000, 12288, device="cuda")            # (wide groups)
w = torch.randint(-127, 128, (1024, 8192), device="cuda").to(torch.int8).view(torch.uint8)
lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(w, torch.full((1024,), 1e-3, device="cuda"), 1024, 8192, 8192, 8))
score, cells = torch.randn(4, 16, device="cuda"), torch.randn(4, 16, 100, device="cuda")
moved = torch.zeros_like(cells)
torch.cuda.synchronize()

def step():
    q, s = Bd.q4_rmsnorm_quantize(x, gain, 1e-5)
    logits = Bd.q4_linear_token_scales(q, s, lin)
    best = Bd.q4_lm_beam_select(logits.view(4, 16, 1024), score, eos=0)
    Bd.q4_beam_reorder([(cells, moved)], best["parent"])
    return [q, s, logits, best["parent"], best["token"], best["score"], *Bd.q4_rmsnorm_quantize(wide, gain.new_ones(12288), 1e-5)]

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = step()
graph.replay()
graph.replay()
torch.cuda.synchronize()
kept = moved.clone()
want = step()
assert all(torch.equal(g, h) for g, h in zip(got, want)) and torch.equal(kept, moved)
print("same")
"""


def test_first_calls_of_a_process_are_captured(Bd):
    # what a first call asks the device or sets up does not disturb a capture
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and r.stdout.split() == ["same"], r.stderr[-2000:]


# -------------------------------------------------------------------------------------------------------- refusals
def test_refusals_of_the_binding(Bd):
    x = torch.randn(4, 64, device="cuda")
    gain = torch.ones(64, device="cuda")
    for call in (lambda: Bd.q4_rmsnorm_quantize(x.cpu(), gain, 1e-5), lambda: Bd.q4_rmsnorm_quantize(x.double(), gain, 1e-5),
                 lambda: Bd.q4_rmsnorm_quantize(x, gain[:32], 1e-5), lambda: Bd.q4_rmsnorm_quantize(x.t(), gain[:4].contiguous(), 1e-5),
                 lambda: Bd.q4_rmsnorm_quantize(x, gain, 1e-5, residual=x), lambda: Bd.q4_rmsnorm_quantize(x, gain, 1e-5, residual=x.half(), sum_out=x),
                 lambda: Bd.q4_rmsnorm_quantize(x[:1].expand(4, 64), gain, 1e-5), lambda: Bd.q4_rmsnorm_quantize(x, gain.half(), 1e-5)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: Bd.q4_rmsnorm_quantize(x, gain, -1.0), -2), (lambda: Bd.q4_rmsnorm_quantize(x, gain, NAN), -2),
                       (lambda: Bd.q4_rmsnorm_quantize(x, gain, 1e-5, k_pad=72), -3), (lambda: Bd.q4_rmsnorm_quantize(x, gain, 1e-5, k_pad=32), -2)):
        with pytest.raises(Bd.Q4Error) as err:
            call()
        assert err.value.code == code
    lin = Bd.DeviceLinear.from_mat(Bd.DeviceMat(torch.zeros(8, 64, dtype=torch.uint8, device="cuda"), gain[:8].contiguous(), 8, 64, 64, 8))
    xq, sx = torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.ones(4, device="cuda")
    for call in (lambda: Bd.q4_linear_token_scales(xq[:, :32], sx, lin), lambda: Bd.q4_linear_token_scales(xq, sx[:3], lin),
                 lambda: Bd.q4_linear_token_scales(xq.cpu(), sx, lin), lambda: Bd.q4_linear_token_scales(xq, sx, lin, out_dtype=torch.int8),
                 lambda: Bd.q4_linear_token_scales(xq, sx, lin, out=torch.zeros(4, 9, device="cuda")),
                 lambda: Bd.DeviceLinear.from_mat(lin.w, gain)):
        with pytest.raises(ValueError):
            call()
    four = Bd.DeviceLinear.from_mat(Bd.DeviceMat(torch.zeros(8, 32, dtype=torch.uint8, device="cuda"), gain[:8].contiguous(), 8, 64, 64, 4))
    with pytest.raises(Bd.Q4Error) as err:
        Bd.q4_linear_token_scales(xq, sx, four)
    assert err.value.code == -4
    logits, score = torch.zeros(2, 4, 10, device="cuda"), torch.zeros(2, 4, device="cuda")
    done = torch.zeros(2, 4, dtype=torch.uint8, device="cuda")
    for call in (lambda: Bd.q4_lm_beam_select(logits[0], score), lambda: Bd.q4_lm_beam_select(logits, score[:1]),
                 lambda: Bd.q4_lm_beam_select(logits, score.double()), lambda: Bd.q4_lm_beam_select(logits.permute(1, 0, 2), score.t().contiguous()),
                 lambda: Bd.q4_lm_beam_select(logits, score, done=done.float())):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: Bd.q4_lm_beam_select(logits, score, done=done), -2), (lambda: Bd.q4_lm_beam_select(logits, score, eos=10), -2),
                       (lambda: Bd.q4_lm_beam_select(torch.zeros(1, 33, 4, device="cuda"), torch.zeros(1, 33, device="cuda")), -2),
                       (lambda: Bd.q4_lm_beam_select(logits, score, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")), -5)):
        with pytest.raises(Bd.Q4Error) as err:
            call()
        assert err.value.code == code
    parent = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    with pytest.raises(Bd.Q4Error) as err:
        Bd.q4_beam_reorder([(logits, logits)], parent)
    assert err.value.code == -6
    for pair in ((logits, logits[:1]), (logits, logits.half()), (logits.permute(1, 0, 2), logits.permute(1, 0, 2))):
        with pytest.raises(ValueError):
            Bd.q4_beam_reorder([pair], parent)
    with pytest.raises(ValueError):
        Bd.q4_beam_reorder([(logits, logits.clone())], parent.long())
