"""The operators around the output of a quantized language model, each as one pass.

Four kinds of cases, in the order in which a label-synchronous search uses them:

  norm     root-mean-square norm of a row, with the residual's addition in front of it, and 8-bit codes with one
           scale for each row (token) behind it
  linear   product of such codes with 8-bit weights: one scale for each token and one for each output channel
  select   one step of a beam search over beams and vocabulary: log-softmax of every beam's logits, scores, the best W
           of W x V extensions
  reorder  the beams' states, moved to where the selection put their extensions

With `own` false every pass is computed from elementary torch operations, in 32 bits, and in 64 where a rounding decides a
whole number (the codes of a norm, the order of a selection).
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def _pad32(k):
    return (k + 31) // 32 * 32


def listed():
    return [
        # the 16 hypotheses of one utterance between two layers of 1024 cells: a call of a few microseconds at most
        dict(name="norm_16x1024_f32", kind="norm", M=16, K=1024, dtype="f32", residual=True, gap=0),
        # outputs of a bidirectional encoder layer (2 x 640), 32 utterances of 500 frames, nothing to add
        dict(name="norm_16000x1280_f16", kind="norm", M=16000, K=1280, dtype="f16", residual=False, gap=0),
        # a prompt of 4096 tokens at a wide model, rows cut out of wider ones
        dict(name="norm_4096x4096_bf16", kind="norm", M=4096, K=4096, dtype="bf16", residual=True, gap=64),
        # one decoding step of one utterance, beam 16: the weights are the work
        dict(name="linear_16_8192x2048_bf16", kind="linear", M=16, N=8192, K=2048, dtype="bf16", bias=True),
        # the vocabulary of a language model for the same 16 hypotheses, logits in 32 bits
        dict(name="linear_16_32000x2048_f32", kind="linear", M=16, N=32000, K=2048, dtype="f32", bias=False),
        # a ragged batch with widths that fit no tile
        dict(name="linear_333_1001x1283_f16", kind="linear", M=333, N=1001, K=1283, dtype="f16", bias=True),
        # a long prompt or a full batch at a wide layer: the arithmetic is the work
        dict(name="linear_8192_8192x8192_bf16", kind="linear", M=8192, N=8192, K=8192, dtype="bf16", bias=False),
        # one utterance, beam 16, the benchmark's 1024 labels: the shortest step of a search
        dict(name="select_1x16x1024_f32", kind="select", B=1, W=16, V=1024, dtype="f32", gap=0, ended=False),
        # a few utterances in the middle of their search, some beams ended, odd vocabulary in padded rows
        dict(name="select_5x12x50257_f16", kind="select", B=5, W=12, V=50257, dtype="f16", gap=47, ended=True),
        # a full batch at a vocabulary of subwords
        dict(name="select_64x16x32000_f32", kind="select", B=64, W=16, V=32000, dtype="f32", gap=0, ended=True),
        # cell states and packed 4-bit codes of one utterance's beams
        dict(name="reorder_cells_1x16", kind="reorder", B=1, W=16, layers=2, heads=0, S=0, used=0, H=2048),
        # keys of 8 layers and 8 heads of 64, 4 x 16 beams, 333 of 512 places written so far
        dict(name="reorder_cache_4x16", kind="reorder", B=4, W=16, layers=8, heads=8, S=512, used=333, H=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "linear", "linear", "select", "select", "reorder"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    if kind == "norm":
        K = _log_int(rng, 64, 8192)
        return dict(kind=kind, M=_log_int(rng, 1, min(16384, (1 << 24) // K)), K=K, dtype=dtype, residual=rng.random() < 0.6,
                    gap=rng.choice((0, 0, 0, 1, 8, 64)))
    if kind == "linear":
        N, K = _log_int(rng, 32, 16384), _log_int(rng, 32, 8192)
        if rng.random() < 0.5:
            N, K = -(-N // 128) * 128, -(-K // 128) * 128
        return dict(kind=kind, M=_log_int(rng, 1, min(8192, (1 << 39) // (N * K))), N=N, K=K, dtype=dtype,
                    bias=rng.random() < 0.5)
    if kind == "select":
        W, V = rng.randint(1, 32), _log_int(rng, 40, 130000)
        return dict(kind=kind, B=_log_int(rng, 1, max(1, min(64, (1 << 25) // (W * V)))), W=W, V=V, dtype=dtype,
                    gap=rng.choice((0, 0, 3, 48)), ended=rng.random() < 0.5)
    B, W = _log_int(rng, 1, 16), rng.randint(1, 24)
    if rng.random() < 0.5:
        return dict(kind=kind, B=B, W=W, layers=rng.randint(1, 4), heads=0, S=0, used=0, H=32 * rng.randint(1, 64))
    S = _log_int(rng, 16, 512)
    return dict(kind=kind, B=min(B, 4), W=W, layers=rng.randint(1, 8), heads=rng.choice((1, 4, 8)), S=S,
                used=rng.randint(1, S), H=rng.choice((64, 80, 128)))


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def prepare(case, seed):
    return {"norm": _prepare_norm, "linear": _prepare_linear, "select": _prepare_select,
            "reorder": _prepare_reorder}[case["kind"]](case, _generator(seed))


def run(state):
    return {"norm": _run_norm, "linear": _run_linear, "select": _run_select, "reorder": _run_reorder}[state["kind"]](state)


def exact(case, seed):
    state = prepare(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "select": _exact_select,
            "reorder": _exact_reorder}[case["kind"]](state)


def work(case):
    if case["kind"] == "norm":
        M, K, s = case["M"], case["K"], SIZE[case["dtype"]]
        # the row, the residual and their sum; the gain; the values of the codes (32 bits as they are returned here)
        return {"bytes": M * K * s * (3 if case["residual"] else 1) + 4 * K + 4 * M * K + 4 * M, "flops": 4 * M * K}
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + M * N * SIZE[case["dtype"]] + 4 * (M + N * (2 if case["bias"] else 1)),
                "flops": 2 * M * N * K}
    if case["kind"] == "select":
        rows = case["B"] * case["W"]
        return {"bytes": rows * (case["V"] * SIZE[case["dtype"]] + 18), "flops": 3 * rows * case["V"]}
    rows, L, H = case["B"] * case["W"], case["layers"], case["H"]
    row = L * case["heads"] * case["used"] * H * 2 if case["heads"] else L * (4 * H + H // 2)
    return {"bytes": 2 * rows * row + 4 * rows, "flops": 0}


# ---------------------------------------------------------------------------------------------------- norm
def _prepare_norm(case, g):
    M, K, dtype = case["M"], case["K"], DTYPES[case["dtype"]]

    def rows(spread):
        # a few channels carry much larger values than the others, as they do in trained networks
        channel = torch.exp(torch.randn(K, generator=g, device="cuda"))
        wide = torch.zeros((M, K + case["gap"]), dtype=dtype, device="cuda")
        wide[:, :K] = (torch.randn((M, K), generator=g, device="cuda") * channel * spread).to(dtype)
        return wide[:, :K]

    state = dict(kind="norm", x=rows(1.0), gain=1.0 + 0.2 * torch.randn(K, generator=g, device="cuda"),
                 residual=rows(4.0) if case["residual"] else None)
    state["sum"] = torch.empty((M, K), dtype=dtype, device="cuda") if case["residual"] else None
    return state


def _run_norm(s):
    if own:
        from paper_2206_07882_b200 import binding as q4
        codes, scale = q4.q4_rmsnorm_quantize(s["x"], s["gain"], EPS, residual=s["residual"], sum_out=s["sum"])
        values = codes.view(torch.int8)[:, :s["x"].shape[1]] * scale[:, None]
        return (values, scale, s["sum"]) if s["residual"] is not None else (values, scale)
    x, dtype = s["x"].float(), s["x"].dtype
    if s["residual"] is not None:
        stored = (x + s["residual"].float()).to(dtype)
        x = stored.float()
    mean_square = (x * x).mean(dim=1, keepdim=True)
    # codes: nearest integer of 127 v / max |v| of the row; the norm's own factor is in both and cancels, and 64 bits decide
    # values next to a half
    v = x.double() * s["gain"].double()
    top = v.abs().amax(dim=1, keepdim=True)
    none = top == 0
    codes = torch.round(127.0 * v / torch.where(none, torch.ones_like(top), top))
    scale = torch.where(none, torch.ones_like(top).float(), top.float() / torch.sqrt(mean_square + EPS)) / 127.0
    values = codes.float() * scale
    return (values, scale[:, 0], stored) if s["residual"] is not None else (values, scale[:, 0])


def _exact_norm(s):
    h = s["x"].double()
    if s["residual"] is not None:
        h = (h + s["residual"].double()).to(s["x"].dtype).double()
    y = h / (h.pow(2).sum(1) / h.shape[1] + EPS).sqrt()[:, None] * s["gain"].double()
    edge = y.abs().max(1).values
    edge[edge == 0] = 1.0
    # the codes from the values before the division by the root: a factor that is common to a row, and none of its rounding
    u = h * s["gain"].double()
    most = u.abs().max(1).values
    most[most == 0] = 1.0
    scale = edge / 127
    values = (u * 127 / most[:, None]).round() * scale[:, None]
    return (values, scale, h) if s["residual"] is not None else (values, scale)


# -------------------------------------------------------------------------------------------------- linear
def _prepare_linear(case, g):
    M, N, K = case["M"], case["N"], case["K"]

    def codes(rows):
        # bell-shaped around zero with the largest magnitude in use, as a maximum boundary leaves them
        c = torch.zeros((rows, _pad32(K)), dtype=torch.int8, device="cuda")
        c[:, :K] = torch.clamp(torch.round(torch.randn((rows, K), generator=g, device="cuda") * 36.0), -127, 127).to(torch.int8)
        return c

    x, w = codes(M), codes(N)
    state = dict(kind="linear", K=K, dtype=DTYPES[case["dtype"]], x=x, w=w,
                 x_scale=0.01 + 0.05 * torch.rand(M, generator=g, device="cuda"),
                 w_scale=(0.2 + torch.rand(N, generator=g, device="cuda")) / (127.0 * math.sqrt(K)),
                 bias=0.5 * torch.randn(N, generator=g, device="cuda") if case["bias"] else None)
    if own:
        from paper_2206_07882_b200 import binding as q4
        state["layer"] = q4.DeviceLinear.from_mat(q4.DeviceMat(w.view(torch.uint8), state["w_scale"], N, K, _pad32(K), 8),
                                                  state["bias"])
    return state


def _run_linear(s):
    if own:
        from paper_2206_07882_b200 import binding as q4
        return q4.q4_linear_token_scales(s["x"].view(torch.uint8), s["x_scale"], s["layer"], out_dtype=s["dtype"])
    y = s["x"].float() @ s["w"].float().t()
    y = y * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["dtype"])


def _exact_linear(s):
    y = torch.empty((s["x"].shape[0], s["w"].shape[0]), dtype=torch.float64, device="cuda")
    w = s["w"].double().t()
    for m in range(0, y.shape[0], 1024):
        y[m:m + 1024] = s["x"][m:m + 1024].double() @ w
    y *= s["x_scale"].double()[:, None] * s["w_scale"].double()[None, :]
    return y if s["bias"] is None else y.add_(s["bias"].double())


# -------------------------------------------------------------------------------------------------- select
def _prepare_select(case, g):
    B, W, V, dtype = case["B"], case["W"], case["V"], DTYPES[case["dtype"]]
    wide = torch.zeros((B, W, V + case["gap"]), dtype=dtype, device="cuda")
    # a broad floor of unlikely labels and a few that the model finds likely
    z = 1.5 * torch.randn((B, W, V), generator=g, device="cuda")
    z.scatter_(2, torch.randint(0, V, (B, W, 4), generator=g, device="cuda"),
               4.0 + 6.0 * torch.rand((B, W, 4), generator=g, device="cuda"))
    # labels that a search's grammar closes
    z.masked_fill_(torch.rand(V, generator=g, device="cuda") < 0.02, -math.inf)
    z[:, :, V // 2] = 0.5
    wide[:, :, :V] = z.to(dtype)
    score = -40.0 + torch.sort(torch.randn((B, W), generator=g, device="cuda") * 4.0, dim=1, descending=True).values
    done = None
    if case["ended"]:
        done = (torch.rand((B, W), generator=g, device="cuda") < 0.2).to(torch.uint8)
        score[0, W // 2:] = -math.inf            # a search that has just begun: not every beam holds a hypothesis
    return dict(kind="select", logits=wide[:, :, :V], score=score, done=done, eos=2 if case["ended"] else -1, rho=0.2)


def _run_select(s):
    if own:
        from paper_2206_07882_b200 import binding as q4
        r = q4.q4_lm_beam_select(s["logits"], s["score"], done=s["done"], eos=s["eos"], rho=s["rho"])
        return r["parent"], r["token"], r["score"], r["done"]
    logits, score = s["logits"].double(), s["score"].double()
    B, W, V = logits.shape
    lse = torch.logsumexp(logits, dim=2, keepdim=True)
    total = score[:, :, None] + (logits - lse + s["rho"])
    if s["done"] is not None:                    # an ended beam goes on as it is, by one extension with the end's label
        ended = s["done"].bool()[:, :, None]
        total = torch.where(ended, torch.full_like(total, -math.inf), total)
        total[:, :, s["eos"]] = torch.where(ended[:, :, 0], score, total[:, :, s["eos"]])
    total = total.reshape(B, W * V)
    # the W best; of equal values at the end of the list those of the lowest parents and labels
    last = total.topk(W, dim=1).values[:, -1:]
    equal = total == last
    room = W - (total > last).sum(dim=1, keepdim=True)
    keep = (total > last) | (equal & (equal.cumsum(dim=1) <= room))
    place = torch.arange(W * V, 0, -1, device=total.device)
    index = torch.where(keep, place, torch.zeros_like(place)).topk(W, dim=1).indices
    best, order = total.gather(1, index).sort(dim=1, descending=True, stable=True)
    index = index.gather(1, order)
    empty = best == -math.inf
    parent = torch.where(empty, -1, index // V).to(torch.int32)
    token = torch.where(empty, -1, index % V).to(torch.int32)
    done = (token == s["eos"]) & ~empty
    return parent, token, best.float(), done.to(torch.uint8)


def _exact_select(s):
    logits, score = s["logits"].double(), s["score"].double()
    B, W, V = logits.shape
    parent, token, value, done = [], [], [], []
    for b in range(B):
        z = logits[b]
        top = z.max(1, keepdim=True).values
        lp = (z - top) - (z - top).exp().sum(1, keepdim=True).log()
        cand = score[b][:, None] + lp + s["rho"]
        if s["done"] is not None:
            for w in torch.nonzero(s["done"][b]).flatten().tolist():
                cand[w] = -math.inf
                cand[w, s["eos"]] = score[b, w]
        order = torch.sort(cand.flatten(), descending=True, stable=True)
        v, i = order.values[:W], order.indices[:W]
        live = torch.isfinite(v)
        value.append(v)
        parent.append(torch.where(live, i // V, torch.full_like(i, -1)))
        token.append(torch.where(live, i % V, torch.full_like(i, -1)))
        done.append(live & (token[-1] == s["eos"]))
    return (torch.stack(parent).to(torch.int32), torch.stack(token).to(torch.int32), torch.stack(value),
            torch.stack(done).to(torch.uint8))


# ------------------------------------------------------------------------------------------------- reorder
def _prepare_reorder(case, g):
    B, W, L, H = case["B"], case["W"], case["layers"], case["H"]
    parent = torch.sort(torch.randint(0, W, (B, W), generator=g, device="cuda"), dim=1).values.to(torch.int32)
    if W > 2:
        parent[0, W - 1] = -1                    # a beam that holds no hypothesis
    if case["heads"]:
        shape, used = (L, B, W, case["heads"], case["S"], H), case["used"]
        src, dst = (torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        pairs = [(src[:, :, :, :, :used], dst[:, :, :, :, :used], dst)]
    else:
        cells = lambda: torch.randn((B, W, H), generator=g, device="cuda")
        codes = lambda: torch.randint(0, 256, (B, W, H // 2), generator=g, device="cuda").to(torch.uint8)
        pairs = [(make(), to, to) for _ in range(L) for make in (cells, codes) for to in (make(),)]
    return dict(kind="reorder", parent=parent, pairs=pairs, dim=1 if case["heads"] else 0)


def _run_reorder(s):
    if own:
        from paper_2206_07882_b200 import binding as q4
        q4.q4_beam_reorder([(src, dst) for src, dst, _ in s["pairs"]], s["parent"], dim=s["dim"])
        return [whole for _, _, whole in s["pairs"]]
    parent, d = s["parent"].long(), s["dim"]
    B, W = parent.shape
    live = parent >= 0
    rows = torch.arange(B, device="cuda")[:, None] * W + torch.where(live, parent, torch.zeros_like(parent))
    rows = rows.flatten()

    def move(src, dst, whole):
        moved = src.flatten(d, d + 1).index_select(d, rows).unflatten(d, (B, W))
        dst.copy_(torch.where(live.reshape((1,) * d + (B, W) + (1,) * (src.dim() - d - 2)), moved, dst))
        return whole

    return [move(*pair) for pair in s["pairs"]]


def _exact_reorder(s):
    out = []
    where = s["parent"].tolist()
    for src, dst, whole in s["pairs"]:
        if s["dim"]:
            src, dst = src.movedim(0, 2), dst.movedim(0, 2)
        for b, row in enumerate(where):
            for w, p in enumerate(row):
                if p >= 0:
                    dst[b, w] = src[b, p]
        out.append(whole)
    return out
