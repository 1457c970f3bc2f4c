"""Token statistics of the LM head (log-probability, lse, entropy, top alternatives), their gradient, and the head in 8-bit
integers, against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0 ** -24                     # half a step of float32, relative
U16 = 2.0 ** -8                      # half a step of bfloat16, relative to the value (an upper bound)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def P():
    import paper_2603_04135_amd as P
    P.load()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return P


def grid(shape, sigma, step, gen, dtype):
    """Values of 8 significant bits on a grid: sums of their products are exact in float32."""
    x = torch.randn(shape, generator=gen, device=DEV)
    return (x * (sigma / step)).round().clamp(-127, 127).mul(step).to(dtype)


class Case:
    def __init__(self, dtype, N, D, V, seed=0, extra=None, sigma_w=None, targets=True):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype, self.N, self.D, self.V = dtype, N, D, V
        T = N + (N // 3 + 2 if extra is None else extra)
        self.T = T
        sw = sigma_w or 2.0 / D ** 0.5
        self.loss_pos = None
        if extra is None:
            self.loss_pos = torch.randperm(T - 1, generator=gen, device=DEV)[:N].sort().values.to(torch.int32)
        self.ids = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32) if targets else None
        self.h_scale = self.w_scale = None
        if dtype == "i8":
            self.H = torch.randint(-127, 128, (T, D), generator=gen, device=DEV, dtype=torch.int8)
            self.W = torch.randint(-127, 128, (V, D), generator=gen, device=DEV, dtype=torch.int8)
            self.h_scale = torch.rand(T, generator=gen, device=DEV) * 0.02 + 0.01
            self.w_scale = (torch.rand(V, generator=gen, device=DEV) + 0.5) * 0.03 / D ** 0.5
        else:
            self.H = grid((T, D), 1.0, 2.0 ** -4, gen, DTYPES[dtype])
            self.W = grid((V, D), sw, 2.0 ** -8 if D <= 256 else 2.0 ** -9, gen, DTYPES[dtype])

    def rows(self):
        at = torch.arange(self.N, device=DEV) if self.loss_pos is None else self.loss_pos.long()
        y = None if self.ids is None else self.ids[at if self.loss_pos is None else at + 1].long()
        return at, y

    def logits(self):
        """float64 logits: exact for the grid; for int8 the float32 values that the definition names, widened."""
        at, _ = self.rows()
        if self.dtype == "i8":
            acc = (self.H[at].double() @ self.W.double().T).float()
            return ((acc * self.w_scale) * self.h_scale[at][:, None]).double()
        return self.H[at].double() @ self.W.double().T

    def call(self, P, top_k, **kw):
        return P.dppo_token_stats(self.H, self.W, self.ids, self.loss_pos, top_k=top_k, h_scale=self.h_scale,
                                  w_scale=self.w_scale, **kw)


def reference(z, y):
    m = z.max(dim=1, keepdim=True).values
    lse = torch.logsumexp(z, dim=1)
    lp = z - lse[:, None]
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(dim=1)
    logp = None if y is None else lp.gather(1, y[:, None])[:, 0]
    return lse, ent, logp, (m - z.min(dim=1, keepdim=True).values)[:, 0]


def check_stats(out, z, y, k, z_err=0.0):
    """z_err: bound on the error of the kernel's own logits. Arithmetic behind the tolerances: an exponential's argument is rounded
    twice (relative error of exp(-d): 2 d U32, plus 2 U32 of its own), a sum of exponentials passes at most 64 additions on
    its way from a lane to the result: log S is off by (64 + 2 d) U32, R / S by (1 + d) times that; lse adds its own rounding."""
    lse, ent, logp, d = reference(z, y)
    s_err = (64 + 2 * d) * U32 + 2 * z_err
    tol = s_err + 2 * U32 * (lse.abs() + z.abs().max(dim=1).values)
    assert ((out["lse"].double() - lse).abs() <= tol).all()
    assert ((out["entropy"].double() - ent).abs() <= 2 * (1 + d) * s_err + 4 * U32 * ent.abs()).all()
    if y is not None:
        assert ((out["logp"].double() - logp).abs() <= 2 * tol).all()
    else:
        assert out["logp"] is None
    if k == 0:
        assert out["top_ids"] is None and out["top_logp"] is None
        return
    ids, lp = out["top_ids"].long(), out["top_logp"].double()
    got = z.gather(1, ids)
    assert ((lp - (got - lse[:, None])).abs() <= 2 * tol[:, None]).all()
    if z_err == 0.0:
        want = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids, want)
    else:
        assert ((got - torch.topk(z, k, dim=1).values).abs() <= 2 * z_err).all()
        assert (ids.sort(dim=1).values.diff(dim=1) > 0).all()


# columns of 96, 128, 192 and 256 tokens and their edges; vocabularies around tiles, of one entry, of several parts a row
@pytest.mark.parametrize("dtype,N,D,V,k", [
    ("f32", 1, 1, 1, 1), ("f32", 1, 7, 3, 3), ("f32", 3, 64, 255, 64), ("f32", 170, 64, 512, 5), ("f32", 300, 33, 1001, 20),
    ("f32", 2, 130, 20011, 7), ("f32", 700, 16, 100, 0),
    ("bf16", 1, 64, 1, 1), ("bf16", 1, 128, 20011, 20), ("bf16", 2, 64, 257, 64), ("bf16", 95, 64, 700, 3), ("bf16", 97, 128, 256, 8),
    ("bf16", 128, 192, 1000, 0), ("bf16", 129, 64, 513, 20), ("bf16", 192, 256, 4099, 5), ("bf16", 193, 64, 300, 1),
    ("bf16", 256, 64, 64, 64), ("bf16", 257, 128, 20011, 20), ("bf16", 700, 512, 2049, 33), ("bf16", 520, 64, 33333, 64),
    ("bf16", 5, 1088, 700, 4), ("bf16", 16, 2560, 1003, 20), ("bf16", 3, 4096, 515, 3), ("bf16", 3, 4160, 515, 3), ("bf16", 17, 2560, 300, 3),
    ("i8", 7, 2176, 700, 4), ("i8", 16, 6144, 333, 20), ("i8", 4, 6272, 333, 5), ("i8", 2, 1024, 33000, 64),
    ("bf16", 300, 64, 70001, 20), ("bf16", 300, 128, 20011, 3), ("bf16", 1500, 64, 16700, 1), ("i8", 300, 128, 70001, 20),
    ("i8", 1, 128, 1, 1), ("i8", 1, 128, 20011, 20), ("i8", 50, 256, 1000, 7), ("i8", 100, 128, 300, 0), ("i8", 150, 384, 513, 64),
    ("i8", 192, 128, 4099, 2), ("i8", 193, 128, 255, 20), ("i8", 513, 256, 20011, 20), ("i8", 300, 1152, 257, 9)])
@pytest.mark.parametrize("positions", ["loss_pos", "identity", "no targets"])
def test_statistics(P, dtype, N, D, V, k, positions):
    if dtype == "i8" and D % 128:
        pytest.skip("int8 rows are padded")
    c = Case(dtype, N, D, V, seed=N + V, extra=None if positions == "loss_pos" else 0,
             targets=positions != "no targets")
    status = torch.full((1,), 77, dtype=torch.int32, device=DEV)
    out = c.call(P, k, status=status)
    assert status.item() == 0
    check_stats(out, c.logits(), c.rows()[1], k)


@pytest.mark.parametrize("dtype,N,V", [("bf16", 40, 5000), ("bf16", 600, 5000), ("f32", 300, 5000)])
def test_statistics_of_ordinary_values(P, dtype, N, V):
    """Inputs off the grid: the logits carry the rounding errors of float32 sums, at most D + 2 of them a sum."""
    D = 256
    gen = torch.Generator(device=DEV).manual_seed(5)
    c = Case(dtype, N, D, V, seed=1)
    c.H = torch.randn((c.T, D), generator=gen, device=DEV).to(DTYPES[dtype])
    c.W = (torch.randn((V, D), generator=gen, device=DEV) * 0.3).to(DTYPES[dtype])
    at, y = c.rows()
    z_err = (D + 2) * U32 * float((c.H[at].double().abs() @ c.W.double().abs().T).max())
    check_stats(c.call(P, 20), c.logits(), y, 20, z_err)


@pytest.mark.parametrize("dtype,N", [("f32", 5), ("f32", 300), ("bf16", 5), ("bf16", 150), ("bf16", 600), ("i8", 5), ("i8", 600)])
@pytest.mark.parametrize("kind", ["all equal", "two values", "ascending", "descending", "copies"])
@pytest.mark.parametrize("k", [64, 3])
def test_equal_logits_go_by_id(P, dtype, N, kind, k):
    D, V = 128, 9001
    c = Case(dtype, N, D, V, seed=3)
    i = torch.arange(V, device=DEV)
    c.H.zero_()
    c.H[:, 0] = 1
    c.W.zero_()
    if dtype == "i8":
        c.w_scale.fill_(0.01)
        c.h_scale.fill_(1.0)
    if kind == "two values":                     # the larger one first at the end of a tile, then all over
        c.W[:, 0] = torch.where((i % 250 == 249) & (i > 700), 2, 1).to(c.W.dtype)
    elif kind == "ascending":                    # every alternative seen so far is overtaken by the next ones
        c.W[:, 0] = (i // 100).to(c.W.dtype)
    elif kind == "descending":
        c.W[:, 0] = (90 - i // 100).to(c.W.dtype)
    elif kind == "copies":                       # H at work, every vocabulary row there four times, far apart
        c = Case(dtype, N, D, V, seed=4)
        n = V // 4
        for r in range(1, 4):
            c.W[r * n:(r + 1) * n] = c.W[:n]
            if dtype == "i8":
                c.w_scale[r * n:(r + 1) * n] = c.w_scale[:n]
    out = c.call(P, k)
    check_stats(out, c.logits(), c.rows()[1], k)
    if kind == "all equal":
        assert torch.equal(out["top_ids"], torch.arange(k, device=DEV, dtype=torch.int32).expand(N, k))


@pytest.mark.parametrize("dtype,N", [("f32", 3), ("f32", 300), ("bf16", 3), ("bf16", 150), ("bf16", 600)])
@pytest.mark.parametrize("kind", ["tile", "most", "lowest", "lowest all", "all", "nan", "inf"])
@pytest.mark.parametrize("V,k", [(5001, 20), (9001, 3)])
def test_masked_and_non_finite_logits(P, dtype, N, kind, V, k):
    """Column 0 of W is added to the logits. -infinity and the type's lowest value carry no weight and come last; a NaN or
    +infinity makes the row's statistics NaN and leaves distinct alternatives in range."""
    D = 64
    c = Case(dtype, N, D, V, seed=6)
    c.H[:, 0] = 1
    low = float(torch.finfo(DTYPES[dtype]).min)
    if kind == "tile":
        c.W[256:512, 0] = -np.inf
    elif kind == "most":
        c.W[k // 3:, 0] = -np.inf                # fewer finite entries than alternatives
    elif kind == "lowest":
        c.W[:4000, 0] = low
    elif kind == "lowest all":
        c.W.zero_()
        c.W[:, 0] = low
    elif kind == "all":
        c.W[:, 0] = -np.inf
    elif kind == "nan":
        c.W[V - 3, 0] = np.nan
    elif kind == "inf":
        c.W[V - 2, 0] = np.inf
    out = c.call(P, k)
    at, y = c.rows()
    ids = out["top_ids"].long()
    assert ((ids >= 0) & (ids < V)).all() and (ids.sort(dim=1).values.diff(dim=1) > 0).all()
    if kind in ("all", "nan", "inf"):
        assert not torch.isfinite(out["lse"]).any() and torch.isnan(out["entropy"]).all() and torch.isnan(out["logp"]).all()
        if kind != "all":
            assert torch.isnan(out["lse"]).all() and torch.isnan(out["top_logp"]).all()
        return
    z = c.logits()
    if kind in ("lowest", "lowest all"):
        z = z.float().double()                   # what the sum is in float32
        if dtype == "f32" and kind == "lowest":
            z[:, :4000] = z[:, :4000].clamp(min=low)
    fine = torch.isfinite(z) & (z > -1e30) if kind != "lowest all" else torch.ones_like(z, dtype=torch.bool)
    n_fine = int(fine[0].sum())
    # the reference without the masked entries
    keep = torch.nonzero(fine[0])[:, 0]
    zk = z[:, keep]
    lse, ent, _, d = reference(zk, None)
    tol = (64 + 2 * d) * U32 + 2 * U32 * (lse.abs() + zk.abs().max(dim=1).values)
    assert ((out["lse"].double() - lse).abs() <= tol).all()
    if kind == "lowest all":                     # (V equal logits: uniform)
        assert ((out["entropy"].double() - np.log(V)).abs() <= 128 * U32 * np.log(V)).all()
    else:
        assert ((out["entropy"].double() - ent).abs() <= 2 * (1 + d) * (64 + 2 * d) * U32 + 4 * U32 * ent.abs()).all()
    want = keep[torch.sort(zk, dim=1, descending=True, stable=True).indices[:, :min(k, n_fine)]]
    assert torch.equal(ids[:, :min(k, n_fine)], want)
    if kind == "most":
        assert torch.isneginf(out["top_logp"][:, n_fine:]).all()
        assert torch.equal(ids[:, n_fine:], torch.arange(n_fine, k, device=DEV).expand(N, k - n_fine))


def test_bad_targets_and_positions_are_reported_and_clamped(P):
    for dtype, N in (("f32", 40), ("bf16", 40), ("bf16", 300)):
        c = Case(dtype, N, 64, 500, seed=9)
        good = c.call(P, 4)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        c.ids = c.ids.clone()
        at, _ = c.rows()
        c.ids[int(at[5]) + 1] = 500
        out = c.call(P, 4, status=status)
        assert status.item() == P.HEAD_BAD_TARGET
        same = torch.ones(N, dtype=torch.bool, device=DEV)
        same[5] = False
        assert torch.equal(out["logp"][same], good["logp"][same]) and torch.equal(out["top_ids"], good["top_ids"])
        c.loss_pos = c.loss_pos.clone()
        c.loss_pos[N - 1] = c.T + 100
        c.loss_pos[0] = -7
        c.call(P, 4, status=status)
        assert status.item() & P.HEAD_BAD_POSITION
        # without targets the last packed position is a valid one
        c.ids = None
        c.loss_pos[N - 1], c.loss_pos[0] = c.T - 1, 0
        c.call(P, 4, status=status)
        assert status.item() == 0
        c.loss_pos[3] = c.T
        out = c.call(P, 4, status=status)
        assert status.item() == P.HEAD_BAD_POSITION and torch.isfinite(out["lse"]).all()


@pytest.mark.parametrize("dtype,N,V,k", [("f32", 600, 500, 5), ("bf16", 1000, 3000, 20), ("i8", 1000, 3000, 20), ("bf16", 1000, 3000, 0)])
def test_smallest_workspace(P, dtype, N, V, k):
    """Chunks of 256 tokens, in a workspace full of NaN."""
    c = Case(dtype, N, 128, V, seed=11)
    code = {"f32": 0, "bf16": 1, "i8": 2}[dtype]
    nbytes = P.dppo_token_stats_workspace_min_bytes(c.T, N, 128, V, code, k)
    assert nbytes < P.dppo_token_stats_workspace_bytes(c.T, N, 128, V, code, k)
    ws = P.binding.alloc_workspace(nbytes, DEV).fill_(0xFF)
    check_stats(c.call(P, k, ws=ws), c.logits(), c.rows()[1], k)
    with pytest.raises(P.DppoError) as e:
        c.call(P, k, ws=ws[:nbytes - 1])
    assert e.value.status == 4


# -- gradient -------------------------------------------------------------------------------------------------------
def make_grads(c, seed, which):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    g = {n: torch.randn(c.N, generator=gen, device=DEV) / c.N for n in ("g_logp", "g_lse", "g_entropy")}
    return {n: t for n, t in g.items() if n in which}


def grad_reference(c, g):
    """dz, dH, dW in 64 bits from the formula."""
    at, y = c.rows()
    z = c.logits()
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    lp = z - lse
    p = lp.exp()
    ent = -(p * lp).sum(dim=1, keepdim=True)
    dz = torch.zeros_like(z)
    if "g_logp" in g:
        dz -= g["g_logp"].double()[:, None] * p
        dz.scatter_add_(1, y[:, None], g["g_logp"].double()[:, None])
    if "g_lse" in g:
        dz += g["g_lse"].double()[:, None] * p
    if "g_entropy" in g:
        dz -= g["g_entropy"].double()[:, None] * p * (lp + ent)
    dH = torch.zeros(c.H.shape, dtype=torch.float64, device=DEV)
    dH.index_add_(0, at, dz @ c.W.double())
    return dz, dH, dz.T @ c.H[at].double()


def check_grads(c, g, out, dW0=None):
    """bfloat16: dz rounded once (U16 each, so at most U16 * |dz| @ |W|), the result rounded once more; float32: the entries
    are off by some 64 + 2 d roundings relative to p times their factors, the products by the length of their sums."""
    dz, dH, dW = grad_reference(c, g)
    at, _ = c.rows()
    z = c.logits()
    d = (z.max() - z.min()).item()
    lp = torch.log_softmax(z, dim=1)
    size = sum(t.double().abs()[:, None] for t in g.values()) * lp.exp() * (2 + 2 * lp.abs() + np.log(c.V))
    if "g_logp" in g:
        size.scatter_add_(1, c.rows()[1][:, None], g["g_logp"].double().abs()[:, None])
    e_dz = size * (128 + 4 * d) * U32 + (U16 * dz.abs() if c.dtype == "bf16" else 0)
    absW, absH = c.W.double().abs(), c.H[at].double().abs()
    bH = e_dz @ absW + c.V * U32 * (dz.abs() @ absW)
    bW = e_dz.T @ absH + c.N * U32 * (dz.abs().T @ absH)
    tol_H = torch.zeros(c.H.shape, dtype=torch.float64, device=DEV)
    tol_H[at] = bH
    if c.dtype == "bf16":
        tol_H += U16 * (dH.abs() + tol_H)
    if dW0 is not None:
        dW = dW + dW0.double()
        bW = bW + 2 * U32 * dW.abs()
    if out["dW"].dtype == torch.bfloat16:
        bW = bW + U16 * (dW.abs() + bW)
    assert out["dH"].dtype == c.H.dtype
    assert ((out["dH"].double() - dH).abs() <= tol_H + 1e-30).all()
    assert ((out["dW"].double() - dW).abs() <= bW + 1e-30).all()
    rest = torch.ones(c.T, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert (out["dH"][rest] == 0).all()


def backward(P, c, g, **kw):
    f = c.call(P, 0)
    return P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"], f["entropy"], **g, **kw)


ALL = ("g_logp", "g_lse", "g_entropy")


@pytest.mark.parametrize("dtype,N,D,V", [
    ("f32", 1, 1, 1), ("f32", 1, 3, 700), ("f32", 170, 64, 512), ("f32", 300, 33, 1001), ("f32", 40, 200, 257),
    ("bf16", 1, 64, 1), ("bf16", 1, 128, 20011), ("bf16", 40, 64, 257), ("bf16", 300, 320, 1000), ("bf16", 257, 64, 256),
    ("bf16", 700, 192, 4099), ("bf16", 4200, 64, 300)])
@pytest.mark.parametrize("which", [ALL, ("g_logp",), ("g_lse",), ("g_entropy",)])
def test_gradient(P, dtype, N, D, V, which):
    c = Case(dtype, N, D, V, seed=N + D, extra=None if N % 2 else 0)
    g = make_grads(c, 1, which)
    dH = torch.full_like(c.H, float("nan"))
    check_grads(c, g, backward(P, c, g, dH=dH))
    if dtype == "bf16":
        dW = torch.full(c.W.shape, float("nan"), dtype=torch.bfloat16, device=DEV)
        check_grads(c, g, backward(P, c, g, dW=dW))


@pytest.mark.parametrize("dtype,out", [("f32", torch.float32), ("bf16", torch.float32), ("bf16", torch.bfloat16)])
def test_gradient_in_chunks_and_added(P, dtype, out):
    c = Case(dtype, 1000, 128, 700, seed=2)
    g = make_grads(c, 3, ALL)
    code, what = {"f32": 0, "bf16": 1}[dtype], 2 if out == torch.bfloat16 else 1
    nbytes = P.dppo_token_stats_workspace_min_bytes(c.T, c.N, c.D, c.V, code, 0, what)
    ws = P.binding.alloc_workspace(nbytes, DEV).fill_(0xFF)
    check_grads(c, g, backward(P, c, g, ws=ws, dW_dtype=out))
    with pytest.raises(P.DppoError):
        backward(P, c, g, ws=ws[:nbytes - 1], dW_dtype=out)
    if out == torch.float32:
        dW0 = torch.randn(c.W.shape, device=DEV)
        check_grads(c, g, backward(P, c, g, dW=dW0.clone(), accumulate_dW=True, ws=ws), dW0)
        check_grads(c, g, backward(P, c, g, dW=dW0.clone(), accumulate_dW=True), dW0)
    # no loss tokens: everything is zero, or left as it was
    empty = torch.zeros(0, dtype=torch.int32, device=DEV)
    z = torch.zeros(0, device=DEV)
    o = P.dppo_token_stats_bwd(c.H, c.W, c.ids, empty, z, z, g_logp=z, dW_dtype=out)
    assert (o["dH"] == 0).all() and (o["dW"] == 0).all()


@pytest.mark.parametrize("which", [("g_logp",), ("g_lse",), ("g_entropy",), ALL])
def test_gradient_against_differences(P, which):
    """Central differences of the loss in 64 bits along random directions: error of the differences h^2 times a third derivative
    (of order 1 here), of the kernel U32-sized."""
    c = Case("f32", 60, 32, 200, seed=8)
    g = make_grads(c, 4, which)
    out = backward(P, c, g)
    at, y = c.rows()

    def loss(H, W):
        lp = torch.log_softmax(H[at] @ W.T, dim=1)
        lse = torch.logsumexp(H[at] @ W.T, dim=1)
        terms = dict(g_logp=lp.gather(1, y[:, None])[:, 0], g_lse=lse, g_entropy=-(lp.exp() * lp).sum(dim=1))
        return sum((g[n].double() * terms[n]).sum() for n in g)

    H, W, h = c.H.double(), c.W.double(), 1e-4
    gen = torch.Generator(device=DEV).manual_seed(0)
    for _ in range(4):
        a = torch.randn(H.shape, generator=gen, device=DEV, dtype=torch.float64)
        b = torch.randn(W.shape, generator=gen, device=DEV, dtype=torch.float64)
        num = (loss(H + h * a, W + h * b) - loss(H - h * a, W - h * b)) / (2 * h)
        got = (out["dH"].double() * a).sum() + (out["dW"].double() * b).sum()
        size = (out["dH"].double() * a).abs().sum() + (out["dW"].double() * b).abs().sum()
        assert abs(num - got) <= 1e-5 * size


def test_gradient_of_near_certain_and_impossible_targets(P):
    """p near 1: 1 - p is what is left of the row, not a rounding error; p = 0 in float32: no NaN."""
    for dtype in ("f32", "bf16"):
        c = Case(dtype, 300, 64, 600, seed=12)
        c.H.zero_()
        c.W.zero_()
        c.H[:, 0] = 1
        c.W[3, 0] = 12.0
        c.W[5, 0] = -300.0
        c.ids.fill_(3)
        c.ids[::2] = 5
        g = make_grads(c, 2, ALL)
        check_grads(c, g, backward(P, c, g))


def test_masked_vocabulary_has_no_gradient(P):
    for dtype in ("f32", "bf16"):
        c = Case(dtype, 300, 64, 900, seed=13)
        c.H[:, 0] = 1
        c.W[256:600, 0] = -np.inf
        c.ids.clamp_(max=255)
        g = make_grads(c, 2, ALL)
        o = backward(P, c, g)
        assert torch.isfinite(o["dW"]).all() and (o["dW"][256:600] == 0).all()
        # dH: 0 * -infinity in column 0 alone
        assert torch.isfinite(o["dH"][:, 1:]).all()


# -- 8 bits ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,D", [(1, 1), (1, 4096), (3, 127), (5, 128), (7, 129), (1000, 200), (33, 5000), (257, 2560), (2, 20001)])
def test_quantize_rows(P, dtype, rows, D):
    gen = torch.Generator(device=DEV).manual_seed(D)
    x = torch.randn((rows, D), generator=gen, device=DEV) * torch.exp(torch.randn((rows, 1), generator=gen, device=DEV) * 5)
    x = x.to(DTYPES[dtype])
    if rows > 4:
        x[2] = 0
        x[3] = -0.0
        x[4] = torch.arange(D, device=DEV).remainder(255).sub(127).div(2).to(x.dtype)   # quotients half-way between integers
    q, scale = P.dppo_quantize_rows(x)
    X = x.float().cpu().numpy()
    s = np.abs(X).max(axis=1) * (np.float32(1) / np.float32(127))
    with np.errstate(invalid="ignore", divide="ignore"):
        want = np.where(s[:, None] > 0, np.clip(np.rint(X / s[:, None]), -127, 127), 0).astype(np.int8)
    assert np.array_equal(scale.cpu().numpy(), s)
    assert np.array_equal(q[:, :D].cpu().numpy(), want)
    assert q.shape[1] % 128 == 0 and q.shape[1] - D < 128 and (q[:, D:] == 0).all()


def test_quantize_rows_of_odd_values(P):
    big = float(torch.finfo(torch.float32).max)
    x = torch.zeros((6, 70), device=DEV)
    x[0, 3] = float("inf")
    x[1, 69] = float("nan")
    x[2, 0], x[2, 1] = big, -big
    x[3, 5] = 1e-45                              # the smallest float32: its scale is 0
    x[4, 5], x[4, 6] = 1e-38, -3e-39
    q, scale = P.dppo_quantize_rows(x)
    assert torch.isnan(scale[:2]).all() and (q[:2] == 0).all()
    assert q[2, 0] == 127 and q[2, 1] == -127 and scale[3] == 0 and (q[3] == 0).all() and q[4, 5] == 127
    assert scale[5] == 0 and (q[5] == 0).all()
    with pytest.raises(ValueError):
        P.dppo_quantize_rows(x.T)
    assert P.dppo_quantize_rows(x[:0])[0].shape == (0, 128)


@pytest.mark.parametrize("T,D,V", [(1, 128, 1), (1, 4096, 5000), (16, 6144, 100), (3, 6272, 100), (9, 1152, 70001), (3, 256, 257), (96, 128, 255), (97, 384, 1000), (128, 128, 128),
                                   (129, 128, 513), (192, 640, 300), (193, 128, 1001), (256, 256, 512), (700, 1152, 2001)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_matmul_i8(P, T, D, V, out):
    c = Case("i8", T, D, V, seed=T, extra=0)
    c.H[0] = 127                                 # the largest sum there is
    c.W[0] = 127
    want = (c.H.double() @ c.W.double().T).float() * c.w_scale * c.h_scale[:, None]
    got = P.dppo_matmul_i8(c.H, c.h_scale, c.W, c.w_scale, out_dtype=out)
    assert torch.equal(got, want.to(out))        # exact sums, then the same three roundings
    y = torch.full((T, V), float("nan"), dtype=out, device=DEV)
    assert P.dppo_matmul_i8(c.H, c.h_scale, c.W, c.w_scale, out=y).data_ptr() == y.data_ptr()
    assert torch.equal(y, got)


def test_quantised_head_end_to_end(P):
    """Rows quantised by the library, their product and their statistics: both say the same of the same logits, and are as far
    from the unquantised head's as 8 bits are (each factor half a step of its row's scale)."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    N, D, V = 300, 200, 3000
    H = torch.randn((N, D), generator=gen, device=DEV).to(torch.bfloat16)
    W = torch.randn((V, D), generator=gen, device=DEV) * 0.1
    ids = torch.randint(0, V, (N,), generator=gen, device=DEV, dtype=torch.int32)
    (hq, hs), (wq, ws) = P.dppo_quantize_rows(H), P.dppo_quantize_rows(W)
    z = P.dppo_matmul_i8(hq, hs, wq, ws)
    out = P.dppo_token_stats(hq, wq, ids, top_k=8, h_scale=hs, w_scale=ws)
    check_stats(out, z.double(), ids.long(), 8)
    exact = H.double() @ W.double().T
    bound = (0.5 * hs.double()[:, None] * W.double().abs().sum(dim=1) + 0.5 * ws.double() * H.double().abs().sum(dim=1, keepdim=True)
             + 0.25 * D * hs.double()[:, None] * ws.double()) * 1.001
    assert ((z.double() - exact).abs() <= bound).all()


# -- together, on streams and in graphs --------------------------------------------------------------------------------
def test_statistics_and_their_gradient_are_the_policy_loss(P):
    """Packed sequences: with the log-probabilities as the old ones (ratio 1) and no KL term, the policy loss's gradient is that of
    logp with weights -coef A / C; its log-probabilities are the statistics'."""
    import workloads as WL
    from harness import HeadCase, oracle_select_pack
    rb = WL.make_rollout("tiny")
    sel, pk = oracle_select_pack(rb)
    case = HeadCase(rb.wl, pk, sel, rb.seed, DEV, dtype="bf16", D=128, V=1000)
    f = P.dppo_token_stats(case.H, case.W, case.ids, case.loss_pos, top_k=3)
    old = P.dppo_token_logprob(case.H, case.W, case.ids, case.loss_pos)
    assert (f["logp"] - old[0]).abs().max() <= 1e-4 and (f["lse"] - old[1]).abs().max() <= 1e-4
    assert (f["top_logp"][:, 0] >= f["logp"] - 1e-5).all()
    loss = P.dppo_loss_fwd_bwd(case.H, case.W, case.ids, case.loss_pos, case.loss_cu, case.seq_adv, case.seq_coef, f["logp"], f["logp"],
                               0.2, 0.2, 0.0)
    lengths = case.loss_cu.diff()
    g = torch.repeat_interleave(-case.seq_adv * case.seq_coef / lengths, lengths)
    out = P.dppo_token_stats_bwd(case.H, case.W, case.ids, case.loss_pos, f["lse"], g_logp=g.contiguous())
    for name in ("dH", "dW"):
        a, b = out[name].double(), loss[name].double()
        assert (a - b).norm() <= 4 * U16 * b.norm()


@pytest.mark.parametrize("dtype,N", [("f32", 200), ("bf16", 90), ("bf16", 700), ("i8", 90), ("i8", 700)])
def test_captured_and_replayed(P, dtype, N):
    c = Case(dtype, N, 128, 5003, seed=20)
    k = 20
    g = make_grads(c, 5, ALL)

    def step():
        f = c.call(P, k, ws=ws_f)
        out = [f[n] for n in ("logp", "lse", "entropy", "top_ids", "top_logp")]
        if dtype == "i8":
            out.append(P.dppo_matmul_i8(c.H, c.h_scale, c.W, c.w_scale))
        else:
            out += P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"], f["entropy"], ws=ws_b, **g).values()
        return out

    code = {"f32": 0, "bf16": 1, "i8": 2}[dtype]
    ws_f = P.binding.alloc_workspace(P.dppo_token_stats_workspace_bytes(c.T, N, c.D, c.V, code, k), DEV)
    ws_b = None if dtype == "i8" else P.binding.alloc_workspace(P.dppo_token_stats_workspace_bytes(c.T, N, c.D, c.V, code, 0, 1), DEV)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    gen = torch.Generator(device=DEV).manual_seed(1)
    for r in range(3):
        if dtype == "i8":
            c.H.copy_(torch.randint(-127, 128, c.H.shape, generator=gen, device=DEV, dtype=torch.int8))
        else:
            c.H.copy_(grid(c.H.shape, 1.0, 2.0 ** -4, gen, c.H.dtype))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b)


def test_on_another_stream(P):
    c = Case("bf16", 400, 128, 5003, seed=21)
    want = c.call(P, 20)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = c.call(P, 20)
    s.synchronize()
    for n in want:
        assert torch.equal(want[n], got[n])


def test_arguments_that_are_refused(P):
    c = Case("bf16", 40, 64, 500, seed=1)
    f = c.call(P, 0)
    with pytest.raises(ValueError):
        P.dppo_token_stats(c.H, c.W.float(), c.ids, c.loss_pos)
    with pytest.raises(ValueError):
        P.dppo_token_stats(c.H.T, c.W, c.ids, c.loss_pos)
    with pytest.raises(ValueError):
        P.dppo_token_stats(c.H, c.W, c.ids[:-1], c.loss_pos)
    with pytest.raises(ValueError):
        P.dppo_token_stats(c.H, c.W, c.ids.long(), c.loss_pos)
    with pytest.raises(ValueError):
        P.dppo_token_stats(c.H.cpu(), c.W.cpu())
    for k in (-1, 65):
        with pytest.raises(P.DppoError):
            c.call(P, k)
    with pytest.raises(ValueError):
        P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"][:-1], g_logp=f["lse"])
    with pytest.raises(P.DppoError):
        P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"])
    with pytest.raises(P.DppoError):
        P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"], g_entropy=f["lse"])
    with pytest.raises(P.DppoError):
        P.dppo_token_stats_bwd(c.H, c.W, None, c.loss_pos, f["lse"], g_logp=f["lse"])
    with pytest.raises(ValueError):
        P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"], g_logp=f["lse"], accumulate_dW=True)
    with pytest.raises(P.DppoError):
        P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"], g_logp=f["lse"], accumulate_dW=True,
                               dW=torch.zeros_like(c.W))
    i = Case("i8", 40, 128, 500, seed=1)
    with pytest.raises(P.DppoError):
        P.dppo_token_stats(i.H, i.W, i.ids, i.loss_pos)
    with pytest.raises(ValueError):
        P.dppo_token_stats_bwd(i.H, i.W, i.ids, i.loss_pos, f["lse"], g_logp=f["lse"])
    with pytest.raises(P.DppoError):
        P.dppo_matmul_i8(i.H[:, :64].contiguous(), i.h_scale, i.W[:, :64].contiguous(), i.w_scale)
    with pytest.raises(ValueError):
        P.dppo_matmul_i8(i.H, i.h_scale, i.W, i.w_scale[:-1])


@pytest.mark.parametrize("dtype,N,V", [("f32", 3, 20011), ("f32", 90, 600), ("bf16", 3, 9001), ("bf16", 90, 9001), ("bf16", 300, 9001),
                                       ("bf16", 600, 30001), ("bf16", 4000, 45001), ("i8", 3, 9001), ("i8", 600, 30001)])
@pytest.mark.parametrize("k", [1, 20, 64])
def test_a_token_of_nan_only(P, dtype, N, V, k):
    """A NaN in a token's row of H (in its scale) makes all its logits NaN: distinct alternatives in range all the same, and the other
    tokens are what they were."""
    c = Case(dtype, N, 128 if dtype == "i8" else 64, V, seed=30)
    want = c.call(P, k)
    at, _ = c.rows()
    bad = torch.tensor([0, N - 1], device=DEV).unique()
    if dtype == "i8":
        c.h_scale[at[bad]] = float("nan")
    else:
        c.H[at[bad], 5] = float("nan")
    out = c.call(P, k)
    good = torch.ones(N, dtype=torch.bool, device=DEV)
    good[bad] = False
    for n in want:
        assert torch.equal(out[n][good], want[n][good]), n
    for n in ("logp", "lse", "entropy", "top_logp"):
        assert torch.isnan(out[n][bad]).all(), n
    ids = out["top_ids"][bad].long().sort(dim=1).values
    assert (ids >= 0).all() and (ids < V).all() and (ids.diff(dim=1) > 0).all()


@pytest.mark.parametrize("dtype,N", [("f32", 50), ("bf16", 9), ("bf16", 150), ("bf16", 600), ("i8", 9), ("i8", 600)])
def test_positions_in_any_order_and_more_than_once(P, dtype, N):
    """The forward pass only reads H: loss positions may repeat, in any order."""
    c = Case(dtype, N, 128, 3001, seed=31)
    want = c.call(P, 7)
    gen = torch.Generator(device=DEV).manual_seed(1)
    pick = torch.randint(0, N, (N,), generator=gen, device=DEV)
    c.loss_pos = c.loss_pos[pick].contiguous()
    out = c.call(P, 7)
    for n in want:
        assert torch.equal(out[n], want[n][pick]), n


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_matmul_i8_of_many_tokens(P, out):
    """More than 32768 tokens go in chunks; results on odd addresses and lengths, and nothing behind them."""
    T, D, V = 33001, 128, 77
    gen = torch.Generator(device=DEV).manual_seed(32)
    X = torch.randint(-127, 128, (T, D), generator=gen, device=DEV, dtype=torch.int8)
    W = torch.randint(-127, 128, (V, D), generator=gen, device=DEV, dtype=torch.int8)
    xs, ws = torch.rand(T, generator=gen, device=DEV) + 0.5, torch.rand(V, generator=gen, device=DEV) + 0.5
    room = torch.full((T * V + 2,), 7.0, dtype=out, device=DEV)
    P.dppo_matmul_i8(X, xs, W, ws, out=room[1:-1].view(T, V))
    acc = (X.double() @ W.double().T).float()
    assert torch.equal(room[1:-1].view(T, V), (acc * ws * xs[:, None]).to(out))
    assert room[0] == 7 and room[-1] == 7


@pytest.mark.parametrize("dtype,T,N", [("f32", 90, 41), ("bf16", 90, 41), ("bf16", 700, 513), ("i8", 90, 41), ("i8", 700, 513)])
def test_first_tokens_without_positions(P, dtype, T, N):
    """loss_pos NULL and N < T: the first N rows, and dH of the others is zero."""
    import ctypes
    B = P.binding
    c = Case(dtype, T, 128, 1001, seed=33, extra=0)
    want = P.dppo_token_stats(c.H[:N], c.W, c.ids[:N], None, top_k=5, h_scale=None if c.h_scale is None else c.h_scale[:N], w_scale=c.w_scale)
    code = {"f32": 0, "bf16": 1, "i8": 2}[dtype]
    shape = B.HeadShape(T, N, c.D, c.V, code)
    ws = B.alloc_workspace(P.dppo_token_stats_workspace_bytes(T, N, c.D, c.V, code, 5), DEV)
    got = {n: torch.empty_like(t) for n, t in want.items()}
    ptr = lambda t: None if t is None else t.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    lib = P.load()
    assert lib.dppo_token_stats(ctypes.byref(shape), 5, ptr(c.H), ptr(c.W), ptr(c.h_scale), ptr(c.w_scale), ptr(c.ids), None,
                                *[ptr(got[n]) for n in ("logp", "lse", "entropy", "top_ids", "top_logp")], None, ptr(ws), ws.numel(), stream) == 0
    for n in want:
        assert torch.equal(got[n], want[n]), n
    if dtype == "i8":
        return
    g = [torch.randn(N, device=DEV) for _ in range(3)]
    ref = P.dppo_token_stats_bwd(c.H[:N], c.W, c.ids[:N], None, want["lse"], want["entropy"], *g)
    wb = B.alloc_workspace(P.dppo_token_stats_workspace_bytes(T, N, c.D, c.V, code, 0, 1), DEV)
    dH, dW = torch.full_like(c.H, float("nan")), torch.full(c.W.shape, float("nan"), device=DEV)
    assert lib.dppo_token_stats_bwd(ctypes.byref(shape), ctypes.byref(B.StatsGradParams(0, 0)), ptr(c.H), ptr(c.W), ptr(c.ids), None,
                                    ptr(want["lse"]), ptr(want["entropy"]), *[ptr(t) for t in g], ptr(dH), ptr(dW), None, ptr(wb),
                                    wb.numel(), stream) == 0
    assert torch.equal(dH[:N], ref["dH"]) and (dH[N:] == 0).all() and torch.equal(dW, ref["dW"])


def test_two_calls_at_once(P):
    """On two streams, each with a workspace of its own."""
    cases = [Case("bf16", 700, 128, 9001, seed=34), Case("i8", 700, 128, 9001, seed=35)]
    grads = [make_grads(c, 6, ALL) if c.dtype != "i8" else None for c in cases]

    def both(c, g):
        f = c.call(P, 9)
        out = [f[n] for n in ("logp", "lse", "entropy", "top_ids", "top_logp")]
        if g is not None:
            out += P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, f["lse"], f["entropy"], dW_dtype=torch.bfloat16, **g).values()
        return out

    want = [both(c, g) for c, g in zip(cases, grads)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(both(cases[i], grads[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            for a, b in zip(out, want[i]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("N,D,V,out", [(600, 64, 520, torch.float32), (600, 64, 520, torch.bfloat16), (2100, 128, 300, torch.bfloat16),
                                       (30, 576, 1500, torch.bfloat16), (65, 64, 40000, torch.float32), (1300, 320, 7000, torch.bfloat16)])
def test_gradient_in_parts(P, N, D, V, out):
    """Few tiles with a long sum: dH and dW are cut along it. A workspace full of NaN, nothing outside dH and dW is written."""
    c = Case("bf16", N, D, V, seed=36)
    g = make_grads(c, 7, ALL)
    ws = P.binding.alloc_workspace(P.dppo_token_stats_workspace_bytes(c.T, N, D, V, 1, 0, 2 if out == torch.bfloat16 else 1), DEV).fill_(0xFF)
    pad = 512
    room_h = torch.full((c.T * D + 2 * pad,), 7.0, dtype=torch.bfloat16, device=DEV)
    room_w = torch.full((V * D + 2 * pad,), 7.0, dtype=out, device=DEV)
    r = backward(P, c, g, ws=ws, dH=room_h[pad:-pad].view(c.T, D), dW=room_w[pad:-pad].view(V, D))
    check_grads(c, g, r)
    for room in (room_h, room_w):
        assert (room[:pad] == 7).all() and (room[-pad:] == 7).all()


@pytest.mark.parametrize("N,D,V", [(3, 64, 70001), (64, 320, 3001), (65, 320, 3001), (100, 64, 60001), (70, 1024, 16001), (1500, 64, 20001),
                                   (129, 128, 127), (1025, 448, 130)])
@pytest.mark.parametrize("positions", [True, False])
def test_gradient_of_every_tile(P, N, D, V, positions):
    """Small and large tiles, one or several along every side, with and without positions; what is beside dH and dW stays."""
    c = Case("bf16", N, D, V, seed=37, extra=None if positions else 0)
    g = make_grads(c, 8, ALL)
    pad = 512
    first = None
    for out in (torch.float32, torch.bfloat16):
        room_h = torch.full((c.T * D + 2 * pad,), 7.0, dtype=torch.bfloat16, device=DEV)
        room_w = torch.full((V * D + 2 * pad,), 7.0, dtype=out, device=DEV)
        r = backward(P, c, g, dH=room_h[pad:-pad].view(c.T, D), dW=room_w[pad:-pad].view(V, D))
        check_grads(c, g, r)
        for room in (room_h, room_w):
            assert (room[:pad] == 7).all() and (room[-pad:] == 7).all()
        again = backward(P, c, g, dW_dtype=out)
        assert torch.equal(r["dH"], again["dH"]) and torch.equal(r["dW"], again["dW"])
        if first is not None:                    # (the same float32 sums, rounded once)
            assert torch.equal(first["dH"], r["dH"]) and torch.equal(first["dW"].to(torch.bfloat16), r["dW"])
        first = r
    dW0 = torch.randn(c.W.shape, device=DEV)
    check_grads(c, g, backward(P, c, g, dW=dW0.clone(), accumulate_dW=True), dW0)


@pytest.mark.parametrize("dtype,N,D,V,k", [("bf16", 384, 64, 100001, 20), ("bf16", 384, 64, 100001, 1), ("i8", 384, 128, 100001, 5),
                                           ("bf16", 1100, 64, 60001, 64), ("bf16", 250, 64, 151936, 20), ("bf16", 1501, 64, 70001, 20),
                                           ("i8", 1025, 128, 40001, 3)])
def test_statistics_of_leading_tiles_and_columns_of_192(P, dtype, N, D, V, k):
    """Sizes at which the bound from leading tiles keeps logits from being stored, with either width of columns."""
    c = Case(dtype, N, D, V, seed=40)
    out = c.call(P, k)
    _, y = c.rows()
    check_stats(out, c.logits(), y, k)


@pytest.mark.parametrize("T,D,V", [(3, 256, 70), (40, 384, 300), (300, 128, 1000), (2, 130944, 5)])
def test_matmul_i8_of_the_lowest_value(P, T, D, V):
    """-128 everywhere: the largest sums there are."""
    X, W = (torch.full((n, D), -128, dtype=torch.int8, device=DEV) for n in (T, V))
    W[0] = 127
    xs, ws = torch.ones(T, device=DEV), torch.ones(V, device=DEV)
    Y = P.dppo_matmul_i8(X, xs, W, ws)
    assert (Y[:, 1:] == 16384.0 * D).all() and (Y[:, 0] == float(np.float32(-128.0 * 127.0 * D))).all()


@pytest.mark.parametrize("N", [3, 20, 300])
def test_matrices_of_more_than_4_GiB(P, N):
    """Byte offsets past 32 bits in W, in the result and in dW: the last rows are found, and nothing else."""
    D = 4096
    V = 1_200_011
    X, W = torch.ones((N, D), dtype=torch.int8, device=DEV), torch.zeros((V, D), dtype=torch.int8, device=DEV)
    W[-1], W[V // 2] = 1, 2
    Y = P.dppo_matmul_i8(X, torch.ones(N, device=DEV), W, torch.ones(V, device=DEV))
    assert (Y[:, -1] == D).all() and (Y[:, V // 2] == 2 * D).all() and (Y.count_nonzero(dim=1) == 2).all()
    del X, W, Y
    V = 600_011
    H, W = torch.full((N, D), 1 / 64, dtype=torch.bfloat16, device=DEV), torch.zeros((V, D), dtype=torch.bfloat16, device=DEV)
    W[-1] = 1
    ids = torch.full((N,), V - 1, dtype=torch.int32, device=DEV)
    f = P.dppo_token_stats(H, W, ids, None, top_k=3)
    want = np.log(np.exp(64.0) + V - 1)
    assert (f["top_ids"] == torch.tensor([V - 1, 0, 1], device=DEV, dtype=torch.int32)).all()
    assert ((f["lse"].double() - want).abs() <= 4 * U32 * want).all() and (f["logp"].abs() <= 4 * U32 * want).all()
    g = torch.ones(N, device=DEV)
    b = P.dppo_token_stats_bwd(H, W, ids, None, f["lse"], g_lse=g, dW_dtype=torch.bfloat16)
    assert ((b["dH"].float() - 1).abs() <= 0.01).all() and ((b["dW"][-1].float() - N / 64).abs() <= 0.01 * N / 64).all()
    assert b["dW"][:-1].abs().max() <= 1e-20


def test_quantize_more_rows_than_a_launch_has_threads_for(P):
    """2^26 rows by four rows a workgroup of 256 threads are 2^32 threads: the rows go in ranges, and every one is answered."""
    rows = 2 ** 26 + 2 ** 25 + 3
    x = (torch.arange(rows, device=DEV, dtype=torch.int32) % 251 - 125).to(torch.bfloat16)[:, None]
    q, scale = P.dppo_quantize_rows(x)
    assert torch.equal(scale, x[:, 0].float().abs() * (np.float32(1) / np.float32(127)))
    assert torch.equal(q[:, 0], x[:, 0].sign().mul(127).to(torch.int8))
    words = q.view(torch.int64)                  # (a row's first word holds its one value, the other fifteen nothing)
    assert torch.equal(words[:, 0] & 255, q[:, 0].to(torch.int64) & 255) and (words[:, 0] >> 8 == 0).all()
    assert words[:, 1:].count_nonzero() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "i8"])
def test_status_of_a_call_without_loss_tokens(P, dtype):
    """The status word is cleared where there is nothing to do, too: what an earlier call reported is gone."""
    c = Case(dtype, 5, 128, 300, seed=41)
    none, word = torch.zeros(0, dtype=torch.int32, device=DEV), torch.full((1,), 77, dtype=torch.int32, device=DEV)
    at, c.loss_pos = c.loss_pos, none
    for k in (0, 3):
        out = c.call(P, k, status=word.fill_(77))
        assert word.item() == 0 and out["lse"].shape == (0,)
    if dtype == "i8":
        return
    z = torch.zeros(0, device=DEV)
    P.dppo_token_stats_bwd(c.H, c.W, c.ids, none, z, z, g_logp=z, status=word.fill_(77))
    assert word.item() == 0
    P.dppo_token_logprob(c.H, c.W, c.ids, none, status=word.fill_(77))
    assert word.item() == 0
    P.dppo_token_logprob_noalloc(c.H, c.W, c.ids, none, z, status=word.fill_(77))
    assert word.item() == 0
    c.loss_pos = at                              # (and no error is left behind)
    c.call(P, 3, status=word.fill_(77))
    assert word.item() == 0


# 8-bit operands by each of the wide tiles, neither tokens nor vocabulary a multiple of them (tests/test_stats_plan.py holds these to their tiles)
I8_TILES = [("256x256", 1100, 128, 60001), ("256x256", 700, 384, 40001), ("256x192", 300, 128, 70001), ("256x192", 513, 256, 20011)]


@pytest.mark.parametrize("tile,N,D,V", I8_TILES)
@pytest.mark.parametrize("positions", ["loss_pos", "identity", "no targets"])
@pytest.mark.parametrize("k", [0, 20])
def test_statistics_of_8_bit_operands_by_wide_tiles(P, tile, N, D, V, positions, k):
    c = Case("i8", N, D, V, seed=42, extra=None if positions == "loss_pos" else 0, targets=positions != "no targets")
    check_stats(c.call(P, k), c.logits(), c.rows()[1], k)


@pytest.mark.parametrize("tile,T,D,V", I8_TILES)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_matmul_i8_by_wide_tiles(P, tile, T, D, V, out):
    c = Case("i8", T, D, V, seed=43, extra=0)
    room = torch.full((T * V + 64,), 7.0, dtype=out, device=DEV)
    P.dppo_matmul_i8(c.H, c.h_scale, c.W, c.w_scale, out=room[:T * V].view(T, V))
    want = (c.H.double() @ c.W.double().T).float() * c.w_scale * c.h_scale[:, None]
    assert torch.equal(room[:T * V].view(T, V), want.to(out)) and (room[T * V:] == 7).all()


# more than 4096 + D tokens and no small gradient: dH reads a transposed copy of W
GRADIENT_BY_A_COPY = [(4200, 64, 4099), (4300, 128, 5003)]


@pytest.mark.parametrize("N,D,V", GRADIENT_BY_A_COPY)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_gradient_by_a_transposed_copy_of_the_vocabulary(P, N, D, V, out):
    """In one chunk, in a workspace full of NaN, and in chunks that share the copy."""
    c = Case("bf16", N, D, V, seed=44)
    g = make_grads(c, 9, ALL)
    what = 2 if out == torch.bfloat16 else 1
    most = P.dppo_token_stats_workspace_bytes(c.T, N, D, V, 1, 0, what)
    least = P.dppo_token_stats_workspace_min_bytes(c.T, N, D, V, 1, 0, what)
    assert least < most
    for nbytes in (most, (least + most) // 2, least):
        ws = P.binding.alloc_workspace(nbytes, DEV).fill_(0xFF)
        check_grads(c, g, backward(P, c, g, ws=ws, dW_dtype=out))


@pytest.mark.parametrize("N", [256, 257, 512, 513, 2048, 2049])
def test_statistics_on_both_sides_of_the_joins(P, N):
    """1, 4, 8 and 16 tokens a workgroup of the join."""
    for dtype, k in (("bf16", 20), ("bf16", 0), ("i8", 3)):
        c = Case(dtype, N, 128, 9001, seed=45)
        check_stats(c.call(P, k), c.logits(), c.rows()[1], k)


@pytest.mark.parametrize("D", [500, 640, 2047, 2553, 2568, 3001, 4096, 4097])
def test_quantize_rows_on_both_sides_of_every_rule(P, D):
    """A wavefront or a workgroup per row, with registers for 512 to 4096 elements, at lengths that are multiples of 8 and not."""
    gen = torch.Generator(device=DEV).manual_seed(D)
    most = torch.randn((16385, D), generator=gen, device=DEV) * torch.exp(torch.randn((16385, 1), generator=gen, device=DEV) * 3)
    for dtype in DTYPES.values():
        for rows in (2048, 2049, 16384, 16385):
            x = most[:rows].to(dtype)
            q, scale = P.dppo_quantize_rows(x)
            top = x.float().abs().amax(dim=1)
            assert torch.equal(scale, top * torch.tensor(1 / 127, dtype=torch.float32, device=DEV))
            want = (x.double() / scale.double()[:, None]).float().round()    # (a quotient that 64 bits round to 32 is the 32-bit quotient)
            assert torch.equal(q[:, :D], want.to(torch.int8)) and (q[:, D:] == 0).all()


def raw_stats(P, c, k, outputs, status=None, chunk_bytes=None):
    """dppo_token_stats through the C entry, with only the given outputs (the others NULL)."""
    import ctypes
    B = P.binding
    shape = B.HeadShape(c.T, c.N, c.D, c.V, {"f32": 0, "bf16": 1, "i8": 2}[c.dtype])
    ws = B.alloc_workspace(chunk_bytes or P.dppo_token_stats_workspace_bytes(c.T, c.N, c.D, c.V, shape.dtype, k), DEV).fill_(0xFF)
    f32 = dict(dtype=torch.float32, device=DEV)
    out = {n: torch.full((c.N,), float("nan"), **f32) for n in outputs}
    if k:
        out["top_ids"] = torch.full((c.N, k), -1, dtype=torch.int32, device=DEV)
        out["top_logp"] = torch.full((c.N, k), float("nan"), **f32)
    ptr = lambda t: None if t is None else t.data_ptr()
    lib = P.load()
    assert lib.dppo_token_stats(ctypes.byref(shape), k, ptr(c.H), ptr(c.W), ptr(c.h_scale), ptr(c.w_scale), ptr(c.ids), ptr(c.loss_pos),
                                *[ptr(out.get(n)) for n in ("logp", "lse", "entropy", "top_ids", "top_logp")], ptr(status), ptr(ws),
                                ws.numel(), torch.cuda.current_stream().cuda_stream) == 0, lib.dppo_last_error()
    return out


@pytest.mark.parametrize("dtype,N,V", [("f32", 3, 20011), ("f32", 90, 600), ("bf16", 3, 9001), ("bf16", 90, 9001), ("bf16", 300, 9001),
                                       ("bf16", 1100, 60001), ("i8", 3, 9001), ("i8", 1100, 60001)])
def test_each_output_by_itself(P, dtype, N, V):
    """What is not asked for may be NULL, in any combination, and changes nothing else."""
    c = Case(dtype, N, 128, V, seed=50)
    want = c.call(P, 5)
    for k, outputs in ((0, ["logp"]), (0, ["lse"]), (0, ["entropy"]), (5, []), (5, ["entropy"]), (0, ["logp", "entropy"])):
        out = raw_stats(P, c, k, outputs)
        assert set(out) == set(outputs) | ({"top_ids", "top_logp"} if k else set())
        for n in out:
            assert torch.equal(out[n], want[n]), (n, k, outputs)


@pytest.mark.parametrize("dtype,N,D,V,k", [("f32", 40001, 16, 300, 3), ("bf16", 40001, 64, 300, 3), ("i8", 40001, 128, 300, 0), ("bf16", 3000, 128, 5003, 20),
                                           ("f32", 3000, 33, 1003, 20), ("i8", 3000, 128, 5003, 20)])
@pytest.mark.parametrize("positions", ["loss_pos", "identity"])
def test_statistics_in_chunks_of_any_size(P, dtype, N, D, V, k, positions):
    """More tokens than one chunk holds, and workspaces between the smallest and the recommended one."""
    c = Case(dtype, N, D, V, seed=51, extra=None if positions == "loss_pos" else 0)
    code = {"f32": 0, "bf16": 1, "i8": 2}[dtype]
    least, most = (f(c.T, N, D, V, code, k) for f in (P.dppo_token_stats_workspace_min_bytes, P.dppo_token_stats_workspace_bytes))
    z, y = c.logits(), c.rows()[1]
    for part in (0.0, 0.3, 0.77, 1.0):
        ws = P.binding.alloc_workspace(least + int((most - least) * part), DEV).fill_(0xFF)
        check_stats(c.call(P, k, ws=ws), z, y, k)


@pytest.mark.parametrize("dtype,N,D,V", [("f32", 40001, 8, 100), ("bf16", 40001, 64, 100), ("bf16", 9000, 128, 3001)])
@pytest.mark.parametrize("positions", ["loss_pos", "identity"])
def test_gradient_of_more_than_a_chunk(P, dtype, N, D, V, positions):
    c = Case(dtype, N, D, V, seed=52, extra=None if positions == "loss_pos" else 0)
    g = make_grads(c, 53, ALL)
    check_grads(c, g, backward(P, c, g))
    dW0 = torch.randn(c.W.shape, device=DEV)
    check_grads(c, g, backward(P, c, g, dW=dW0.clone(), accumulate_dW=True), dW0)
    if dtype == "bf16":
        check_grads(c, g, backward(P, c, g, dW_dtype=torch.bfloat16))


@pytest.mark.parametrize("N", [0, 5, 300])
def test_float32_operands_at_any_address(P, N):
    """float32 needs no more than 4-byte alignment, of any matrix."""
    c = Case("f32", max(N, 1), 64, 513, seed=54)
    if N == 0:
        c.N, c.loss_pos = 0, c.loss_pos[:0]

    def moved(t, fill=None):
        room = torch.full((t.numel() + 8,), 7.0, device=DEV)
        m = room[1:1 + t.numel()].view(t.shape)
        m.copy_(t) if fill is None else m.fill_(fill)
        return room, m

    want = c.call(P, 5)
    g = make_grads(c, 1, ALL) if N else dict(g_logp=torch.zeros(0, device=DEV))
    ref = P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, want["lse"], want["entropy"], **g)
    H, W = c.H, c.W
    (_, c.H), (_, c.W) = moved(H), moved(W)
    got = c.call(P, 5)
    for n in want:
        assert torch.equal(got[n], want[n]), n
    (room_h, dH), (room_w, dW) = moved(H, float("nan")), moved(W, float("nan"))
    P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, want["lse"], want["entropy"], dH=dH, dW=dW, **g)
    assert torch.equal(dH, ref["dH"]) and torch.equal(dW, ref["dW"])
    for room in (room_h, room_w):
        assert room[0] == 7 and (room[-7:] == 7).all()
    if N == 0:
        dW.fill_(3.0)
        P.dppo_token_stats_bwd(c.H, c.W, c.ids, c.loss_pos, want["lse"], want["entropy"], dH=dH, dW=dW, accumulate_dW=True, **g)
        assert (dW == 3).all() and (dH == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,D", [(5, 640), (3000, 333), (3, 5000)])
def test_quantize_rows_at_any_address(P, dtype, rows, D):
    gen = torch.Generator(device=DEV).manual_seed(55)
    room = torch.randn(rows * D + 9, generator=gen, device=DEV).to(DTYPES[dtype])
    x = room[1:1 + rows * D].view(rows, D)
    q, scale = P.dppo_quantize_rows(x)
    q0, scale0 = P.dppo_quantize_rows(x.clone())
    assert torch.equal(q, q0) and torch.equal(scale, scale0)


@pytest.mark.parametrize("dtype,N,V", [("bf16", 3, 9001), ("i8", 16, 9001), ("bf16", 1100, 60001), ("i8", 1100, 60001), ("f32", 2, 20011)])
def test_every_kernel_of_the_statistics_captured(P, dtype, N, V):
    """Few tokens, and leading tiles with their bound, replayed with other inputs."""
    c = Case(dtype, N, 128, V, seed=56)
    ws = P.binding.alloc_workspace(P.dppo_token_stats_workspace_bytes(c.T, N, 128, V, {"f32": 0, "bf16": 1, "i8": 2}[dtype], 20), DEV)
    c.call(P, 20, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = c.call(P, 20, ws=ws)
    gen = torch.Generator(device=DEV).manual_seed(2)
    for _ in range(3):
        if dtype == "i8":
            c.H.copy_(torch.randint(-127, 128, c.H.shape, generator=gen, device=DEV, dtype=torch.int8))
        else:
            c.H.copy_(grid(c.H.shape, 1.0, 2.0 ** -4, gen, c.H.dtype))
        want = {n: t.clone() for n, t in c.call(P, 20).items()}
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(captured[n], want[n]), n


def test_no_loss_tokens_captured(P):
    """All that such a call does is to clear its status word, on replays too."""
    c = Case("bf16", 5, 64, 300, seed=57)
    c.loss_pos = c.loss_pos[:0]
    word, ws = torch.zeros(1, dtype=torch.int32, device=DEV), P.binding.alloc_workspace(1 << 20, DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(P, 3, ws=ws, status=word)
    for _ in range(3):
        word.fill_(77)
        torch.cuda.synchronize()
        graph.replay()
        assert word.item() == 0
