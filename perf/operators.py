"""The operators around the LM head, as they are measured: token statistics (log-probability, entropy, top alternatives) and
their gradient, 8-bit quantisation of rows and the 8-bit matrix product. With own = False `run` computes them in their plain
form, in elementary torch operations; with own = True by the framework's calls."""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
I8_ROW = 128        # rows of 8-bit operands are padded with zeros to a multiple of this
H_STEP, W_STEP = 2.0 ** -4, 2.0 ** -9


def listed():
    return [
        # the tiny workload's shape: what a call costs when there is next to nothing to compute
        dict(name="stats_f32_tiny", op="stats", dtype="f32", N=170, D=64, V=512, top_k=5, targets=True),
        # one decoded token: its alternatives and entropy, no target yet; reading the vocabulary matrix is all the work
        dict(name="stats_bf16_one", op="stats", dtype="bf16", N=1, D=2560, V=151936, top_k=20, targets=False),
        # entropy monitored over a small training batch, vocabulary of 32000
        dict(name="stats_bf16_small", op="stats", dtype="bf16", N=1501, D=1024, V=32000, top_k=0, targets=True),
        # scoring a packed row of completions with 20 alternatives a token
        dict(name="stats_bf16_score", op="stats", dtype="bf16", N=8191, D=2560, V=151936, top_k=20, targets=True),
        # the same of a policy whose head is quantised to 8 bits, activations quantised within the call
        dict(name="stats_i8_score", op="stats", dtype="i8", N=6001, D=2560, V=151936, top_k=20, targets=True),
        # gradients of log-probability and entropy: the tiny workload, a small batch, a packed row
        dict(name="bwd_f32_tiny", op="bwd", dtype="f32", N=170, D=64, V=512),
        dict(name="bwd_bf16_small", op="bwd", dtype="bf16", N=1501, D=1024, V=32000),
        dict(name="bwd_bf16_row", op="bwd", dtype="bf16", N=4111, D=2560, V=151936),
        # logits of one decoded token, and of a prompt's tokens, from a quantised head
        dict(name="matmul_i8_one", op="matmul", dtype="bf16", N=1, D=4096, V=151936, out="f32"),
        dict(name="matmul_i8_prompt", op="matmul", dtype="bf16", N=2047, D=4096, V=32000, out="bf16"),
        # the activations of a batch and a vocabulary matrix brought to 8 bits
        dict(name="quantize_tokens", op="quantize", dtype="bf16", N=2047, D=4096),
        dict(name="quantize_vocabulary", op="quantize", dtype="bf16", N=151936, D=2560),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["stats", "stats", "stats", "bwd", "bwd", "matmul", "quantize"])
    if op == "quantize":
        case = dict(op=op, dtype=rng.choice(["f32", "bf16"]), N=_spread(rng, 1, 151936), D=_spread(rng, 64, 4096))
        while case["N"] * case["D"] * (4 if case["dtype"] == "f32" else 2) > 151936 * 2560 * 2:
            case["N"] = 1 + case["N"] // 2
        return case
    dtype = "bf16" if op == "matmul" else rng.choice(["f32", "bf16", "bf16", "i8"] if op == "stats" else ["f32", "bf16", "bf16"])
    if dtype == "f32":
        case = dict(op=op, dtype=dtype, N=_spread(rng, 1, 2000), D=_spread(rng, 16, 512), V=_spread(rng, 100, 32000))
    else:
        D = _spread(rng, 64, 4096)
        if dtype == "bf16" and op != "matmul":
            D = (D + 32) // 64 * 64
        case = dict(op=op, dtype=dtype, N=_spread(rng, 1, 8191), D=max(64, D), V=_spread(rng, 500, 151936))
    most = 2.0 * 4111 * 2560 * 151936 if op == "bwd" else 2.0 * 2047 * 4096 * 32000 if op == "matmul" else 2.0 * 8191 * 2560 * 151936
    while 2.0 * case["N"] * case["D"] * case["V"] > most:
        case["N"] = 1 + case["N"] // 2
    if op == "stats":
        case["top_k"] = rng.choice([0, 1, 3, 8, 20, 64])
        case["targets"] = rng.random() < 0.75
    if op == "matmul":
        case["out"] = rng.choice(["f32", "bf16"])
    return case


# -- inputs -------------------------------------------------------------------------------------------------
def _grid(shape, sigma, step, gen, dtype):
    """Normal values on a grid of 8 significant bits, as an 8-bit checkpoint has them that was widened again: sums of their
    products are exact in 32 bits in any order, so it is the logits, not roundings, that decide which alternative is ahead."""
    x = torch.randn(shape, generator=gen, device="cuda")
    return x.mul_(sigma / step).round_().clamp_(-127, 127).mul_(step).to(dtype)


def _loss_pos(N, gen):
    """Rows of N loss tokens among the packed ones, about a fifth of which are prompts; the last token predicts nothing."""
    T = N + N // 4 + 1
    return T, torch.randperm(T - 1, generator=gen, device="cuda")[:N].sort().values.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, N, D = case["op"], case["N"], case["D"]
    s = dict(case)
    if op == "quantize":
        s["X"] = torch.randn((N, D), generator=gen, device="cuda").to(DTYPES[case["dtype"]])
        return s
    V = case["V"]
    dtype = DTYPES.get(case["dtype"], torch.bfloat16)
    if op == "matmul" or case["dtype"] == "i8":
        # weights quantised once, rows padded; the activations come as the model's last norm leaves them
        W = torch.randn((V, D), generator=gen, device="cuda").mul_(0.02)
        q, s["w_scale"] = _quantize(W)
        s["Wq"] = torch.nn.functional.pad(q, (0, -D % I8_ROW))
    else:
        # D = 64: wider weights, so that the distribution is as far from uniform as a model's
        s["W"] = _grid((V, D), 0.05 if D >= 256 else 0.15, W_STEP, gen, dtype)
    if op == "matmul":
        s["X"] = torch.randn((N, D), generator=gen, device="cuda").to(dtype)
        return s
    T, s["loss_pos"] = _loss_pos(N, gen)
    if op == "stats" and not case["targets"]:        # decoding: every row is asked for
        T, s["loss_pos"] = N, None
    s["H"] = torch.randn((T, D), generator=gen, device="cuda").to(dtype) if case["dtype"] == "i8" else _grid((T, D), 1.0, H_STEP, gen, dtype)
    s["ids"] = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    if op == "stats" and not case["targets"]:
        s["ids"] = None
    if op == "bwd":
        # advantages over the batch's tokens, and an entropy bonus that differs from token to token
        s["g_logp"] = torch.randn(N, generator=gen, device="cuda").div_(N)
        s["g_entropy"] = torch.rand(N, generator=gen, device="cuda").mul_(-0.1 / N)
        z = s["H"][s["loss_pos"].long()].float() @ s["W"].float().T
        s["lse"], s["entropy"] = _softmax_stats(z)
    return s


# -- plain forms --------------------------------------------------------------------------------------------
def _quantize(x):
    x = x.float()
    scale = x.abs().amax(dim=1) / 127.0
    q = (x / scale[:, None]).round().clamp(-127, 127)
    return torch.where(scale[:, None] > 0, q, torch.zeros_like(q)).to(torch.int8), scale


def _product_i8(xq, x_scale, wq, w_scale):
    # whole sums of products pass 24 bits: formed in 64, where they are exact, then rounded to 32
    return (xq.double() @ wq.double().T).float().mul_(w_scale).mul_(x_scale[:, None])


def _softmax_stats(z):
    m = z.amax(dim=1, keepdim=True)
    d = z - m
    e = d.exp()
    total = e.sum(dim=1)
    return m[:, 0] + total.log(), total.log() - (d * e).sum(dim=1) / total


def _top(z, k):
    # one whole number a logit that orders like the logit and, among equals, like the lower id
    bits = z.contiguous().add_(0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    key = order * 2 ** 20 + (2 ** 20 - 1 - torch.arange(z.shape[1], device=z.device))
    return 2 ** 20 - 1 - (torch.topk(key, k, dim=1).values & (2 ** 20 - 1))


def _logits(s):
    rows = s["H"] if s["loss_pos"] is None else s["H"][s["loss_pos"].long()]
    if s["dtype"] == "i8":
        q, scale = _quantize(rows)
        return _product_i8(q, scale, s["Wq"][:, :s["D"]], s["w_scale"])
    return rows.float() @ s["W"].float().T


def _run_plain(s):
    if s["op"] == "quantize":
        q, scale = _quantize(s["X"])
        return dict(values=q * scale[:, None], scale=scale)
    if s["op"] == "matmul":
        q, scale = _quantize(s["X"])
        return _product_i8(q, scale, s["Wq"][:, :s["D"]], s["w_scale"]).to(DTYPES[s["out"]])
    z = _logits(s)
    if s["op"] == "stats":
        lse, entropy = _softmax_stats(z)
        out = dict(lse=lse, entropy=entropy)
        if s["ids"] is not None:
            out["logp"] = z.gather(1, s["ids"][s["loss_pos"].long() + 1].long()[:, None])[:, 0] - lse
        if s["top_k"]:
            top = _top(z, s["top_k"])
            out.update(top_ids=top.to(torch.int32), top_logp=z.gather(1, top) - lse[:, None])
        return out
    at = s["loss_pos"].long()
    logp = z - s["lse"][:, None]
    g = logp.exp() * -(s["g_logp"][:, None] + s["g_entropy"][:, None] * (logp + s["entropy"][:, None]))
    g.scatter_add_(1, s["ids"][at + 1].long()[:, None], s["g_logp"][:, None])
    dH = torch.zeros_like(s["H"])
    dH[at] = (g @ s["W"].float()).to(dH.dtype)
    return dict(dH=dH, dW=(g.T @ s["H"][at].float()).to(s["W"].dtype))


# -- the framework's calls ----------------------------------------------------------------------------------
def _run_own(s):
    import paper_2603_04135_amd as P
    if s["op"] == "quantize":
        q, scale = P.dppo_quantize_rows(s["X"])
        return dict(values=q[:, :s["D"]] * scale[:, None], scale=scale)
    if s["op"] == "matmul":
        q, scale = P.dppo_quantize_rows(s["X"])
        return P.dppo_matmul_i8(q, scale, s["Wq"], s["w_scale"], out_dtype=DTYPES[s["out"]])
    if s["op"] == "bwd":
        return P.dppo_token_stats_bwd(s["H"], s["W"], s["ids"], s["loss_pos"], s["lse"], s["entropy"],
                                      g_logp=s["g_logp"], g_entropy=s["g_entropy"], dW_dtype=s["W"].dtype)
    H, scales = s["H"], {}
    W = s.get("W")
    if s["dtype"] == "i8":
        H, h_scale = P.dppo_quantize_rows(H)
        W, scales = s["Wq"], dict(h_scale=h_scale, w_scale=s["w_scale"])
    return P.dppo_token_stats(H, W, s["ids"], s["loss_pos"], top_k=s["top_k"], **scales)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# -- what a pass cannot do without --------------------------------------------------------------------------
def work(case):
    op, N, D = case["op"], case["N"], case["D"]
    es = 4 if case["dtype"] == "f32" else 2
    if op == "quantize":
        return {"bytes": N * D * es + N * D + 4 * N, "flops": 2 * N * D}
    V = case["V"]
    if op == "matmul":
        return {"bytes": N * D * 2 + V * (D + 4) + N * V * (4 if case["out"] == "f32" else 2), "flops": 2 * N * D * V}
    if op == "bwd":
        T = N + N // 4 + 1
        return {"bytes": (N + V) * D * es + 24 * N + (T + V) * D * es, "flops": 6 * N * D * V}
    w_bytes = V * (D + 4) if case["dtype"] == "i8" else V * D * es
    return {"bytes": N * D * es + w_bytes + (16 if case["targets"] else 8) * N + 8 * N * case["top_k"], "flops": 2 * N * D * V}


# -- the same in 64 bits, from the definitions ---------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op, D = case["op"], case["D"]

    def steps(x):
        """Rows in units of their scale, rounded to whole steps in 64 bits as in 32 (the quotient that decides is the 32-bit one)."""
        scale = (x.float().abs().max(dim=1).values / 127).double()
        unit = torch.where(scale > 0, scale, torch.ones_like(scale)).float()
        return torch.round(x.float() / unit[:, None]).double(), scale

    if op == "quantize":
        q, scale = steps(s["X"])
        return dict(values=q * scale[:, None], scale=scale)
    if op == "matmul" or case["dtype"] == "i8":
        Wd = s["Wq"][:, :D].double() * s["w_scale"].double()[:, None]
    else:
        Wd = s["W"].double()
    if op == "matmul":
        q, scale = steps(s["X"])
        return (q * scale[:, None]) @ Wd.T
    at = torch.arange(s["H"].shape[0], device="cuda") if s["loss_pos"] is None else s["loss_pos"].long()
    x = s["H"].index_select(0, at)
    if case["dtype"] == "i8":
        q, scale = steps(x)
        x = q * scale[:, None]
    else:
        x = x.double()
    z = x @ Wd.T
    logp = torch.log_softmax(z, dim=1)
    if op == "stats":
        lse = torch.logsumexp(z, dim=1)
        out = dict(lse=lse, entropy=-(logp.exp() * logp).sum(dim=1))
        if s["ids"] is not None:
            y = s["ids"].index_select(0, at + 1).long()
            out["logp"] = logp[torch.arange(len(y), device="cuda"), y]
        if case["top_k"]:
            out.update(top_ids=None, top_logp=torch.topk(logp, case["top_k"], dim=1).values)
        return out
    del z
    y = s["ids"].index_select(0, at + 1).long()
    p = logp.exp()
    ent = -(p * logp).sum(dim=1, keepdim=True)
    dz = -p * (s["g_logp"].double()[:, None] + s["g_entropy"].double()[:, None] * (logp + ent))
    dz[torch.arange(len(y), device="cuda"), y] += s["g_logp"].double()
    dH = torch.zeros(s["H"].shape, dtype=torch.float64, device="cuda")
    dH[at] = dz @ Wd
    return dict(dH=dH, dW=dz.T @ x)
