"""The operators that the shared head is trained with, against 64-bit evaluations of their formulas.

Tolerances are bounds from arithmetic.  u = 2^-24 is the half step of fp32, H that of an output's type (bf16: 2^-8).  A sum of k terms
in whatever order is off by at most k u times the sum of the terms' absolute values; a rounding by H times the value."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def half(dtype):
    return torch.finfo(dtype).eps / 2


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, std=1.0, mean=0.0):
    return torch.empty(*shape, device="cuda").normal_(mean, std, generator=g)


def check(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, what
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float(((got - want).abs() / tol).max()):.3g} of the bound"


def strided(t, pad):
    """The same rows in a wider matrix."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


# ---- RMSNorm ---------------------------------------------------------------------------------------------------
NORM_SHAPES = [(1, 16), (3, 48), (1, 4096), (5, 1024), (7, 1040), (2, 2048), (33, 5120), (130, 4096), (9, 6160), (3, 10240), (3, 16400),
               (1300, 64), (2100, 1040)]


def norm_reference(x, gain, eps):
    x, gain = x.double(), gain.double()
    r = 1 / torch.sqrt(x.square().mean(1, keepdim=True) + eps)
    return x, gain, r, x * r * gain


@pytest.mark.parametrize("x_type, dtype", [("f32", "bf16"), ("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("n, d", NORM_SHAPES)
def test_rms_norm_and_its_gradients(n, d, x_type, dtype):
    from paper_2404_16710_amd import rms_norm, rms_norm_grad
    g = gen(n * 7 + d)
    x = (normal(g, n, d) * 4).to(TYPES[x_type])
    if n > 2:
        x[1] = 0                                     # r = 1 / sqrt(eps)
        x[2] *= 1e-4                                 # eps matters
    gain = normal(g, d, std=0.2, mean=1.0).to(TYPES[dtype])
    dy = normal(g, n, d).to(TYPES[dtype])
    if n % 2:
        x, dy = strided(x, 16), strided(dy, 32)
    eps = 1e-5
    xd, gd, r, y = norm_reference(x, gain, eps)
    T, XT = TYPES[dtype], TYPES[x_type]
    # sums of squares: a thread adds d / 64 + 8 terms at most (a wave a row up to d = 1024, then 256 threads) and 8 levels follow;
    # half of that reaches r, and five more roundings y
    k = d / 64 + 16
    rel_r = (k / 2 + 3) * U
    check(rms_norm(x, gain, eps), y, (rel_r + 3 * U + half(T)) * y.abs() + 1e-30, "y")
    dyd = dy.double()
    dot = (gd * dyd * xd).mean(1, keepdim=True)
    dot_abs = (gd * dyd * xd).abs().mean(1, keepdim=True)
    dx = r * gd * dyd - xd * r ** 3 * dot
    tol = (rel_r + 4 * U) * (r * gd * dyd).abs() + xd.abs() * r ** 3 * ((3 * rel_r + 6 * U) * dot.abs() + k * U * dot_abs) + half(XT) * dx.abs()
    dgain = (dyd * xd * r).sum(0)
    # a row's product has r and two roundings, a sum of n terms follows
    tol_g = ((rel_r + 3 * U) + n * U) * (dyd * xd * r).abs().sum(0) + half(T) * dgain.abs()
    got_dx, got_dg = rms_norm_grad(x, gain, dy, eps)
    check(got_dx, dx, tol + 1e-30, "dx")
    check(got_dg, dgain, tol_g + 1e-30, "dgain")
    none, again = rms_norm_grad(x, gain, dy, eps, need_dx=False)
    assert none is None and torch.equal(again, got_dg)


def test_rms_norm_passes_on_what_is_not_finite_in_its_row_alone():
    from paper_2404_16710_amd import rms_norm
    x = normal(gen(3), 5, 2048)
    want = rms_norm(x, torch.ones(2048, device="cuda"), 1e-5)
    x[1, 7], x[3, 100] = float("nan"), float("inf")
    got = rms_norm(x, torch.ones(2048, device="cuda"), 1e-5)
    assert got[1].isnan().all() and got[3, 100].isnan()
    assert torch.equal(got[[0, 2, 4]], want[[0, 2, 4]])


# ---- Softmax cross entropy through the head ----------------------------------------------------------------------
def head_case(n, d, vocab, dtype, seed, pad=0):
    g = gen(seed)
    w = normal(g, vocab, d, std=0.3 / d ** 0.5 * 4).to(TYPES[dtype])
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    h = (normal(g, n, d) + torch.rand(n, 1, generator=g, device="cuda") * w[t].float()).to(TYPES[dtype])
    t = t.to(torch.int32)
    if n > 3:
        t[1] = -1                                    # no loss, no gradient
        t[2] = -100
    weight = torch.rand(n, generator=g, device="cuda") + 0.1
    if n > 4:
        weight[3] = 0
    return (strided(h, pad) if pad else h), w, t, weight


def head_reference(h, w, t, weight):
    """Everything in 64 bits, and the bounds of the logits' and their statistics' errors."""
    h, w, t = h.double(), w.double(), t.long()
    n, d, vocab = h.shape[0], h.shape[1], w.shape[0]
    l = h @ w.T
    lse = torch.logsumexp(l, 1)
    kept = t >= 0
    rows = torch.arange(n, device="cuda")
    loss = torch.where(kept, lse - l[rows, t.clamp(min=0)], 0.0)
    # products are exact (16-bit operands) or kept to 24 bits, then a sum of d terms (fp32 operands: of 6 d)
    dl = (6 * d + 8) * U * (h.abs() @ w.abs().T).amax(1)
    # exponentials: their argument is rounded twice (3 u of at most 90, below which they vanish), exp2 and log to 2 u; sums of up to
    # `vocab` positive terms are off by a u for each of the at most 128 + vocab / 128 steps of a chain
    dlse = dl + (270 + 128 + vocab / 128 + 8) * U + 2 * U * lse.abs()
    q = torch.softmax(l, 1)
    p = q.clone()
    p[rows, t.clamp(min=0)] -= 1
    wt = torch.where(kept, weight.double(), 0.0)[:, None]
    return h, w, loss, lse, dl, dlse, p * wt, q * wt, wt


def check_head(h, w, t, weight, dtype):
    from paper_2404_16710_amd import head_loss, head_loss_grad
    hd, wd, loss, lse, dl, dlse, p, q, wt = head_reference(h, w, t, weight)
    got_loss, got_lse = head_loss(h, w, t)
    tol = dl + dlse + 2 * U * loss.abs()
    check(got_lse, lse, dlse, "lse")
    check(got_loss, loss, torch.where(t.long() >= 0, tol, 0.0), "loss")
    loss2, dh, dw = head_loss_grad(h, w, t, weight)
    check(loss2, loss, torch.where(t.long() >= 0, tol, 0.0), "loss with gradients")
    T = TYPES[dtype]
    n, vocab = p.shape
    # p: the exponential with the errors above, the subtraction, and in 16 bits its rounding (fp32: three planes, 2^-24)
    dp = q * (dl + dlse + 290 * U)[:, None] + 2 * U * (q + p.abs()) + half(T) * p.abs()
    planes = 6 if dtype == "f32" else 1
    want = p @ wd
    tol = dp @ wd.abs() + (planes * vocab + 20) * U * (p.abs() @ wd.abs()) + half(T) * want.abs()
    check(dh, want, tol + 1e-30, "dh")
    want = p.T @ hd
    tol = dp.T @ hd.abs() + (planes * n + 20) * U * (p.T.abs() @ hd.abs()) + half(T) * want.abs()
    check(dw, want, tol + 1e-30, "dW")
    skipped = t.long() < 0
    assert (dh[skipped] == 0).all() and (loss2[skipped] == 0).all()


HEAD_SHAPES = [(1, 16, 1), (1, 16, 17), (2, 48, 31), (1, 256, 1024), (16, 80, 100), (17, 64, 64), (45, 256, 1024), (5, 2048, 333), (64, 208, 1000),
               (65, 128, 2064), (77, 1040, 4099), (130, 384, 257), (300, 96, 511), (333, 512, 1234), (513, 272, 8200), (1100, 64, 96)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, d, vocab", HEAD_SHAPES)
def test_head_loss_and_gradients(n, d, vocab, dtype):
    check_head(*head_case(n, d, vocab, dtype, n + d + vocab, pad=24 if n % 2 else 0), dtype)
