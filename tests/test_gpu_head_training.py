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


@pytest.mark.parametrize("d", [64, 1040, 5120, 16400])
def test_rows_whose_dy_is_zero_throughout_add_nothing_whatever_they_hold(d):
    """Padding: skipped rows of a loss come back as zeros, and their states may be anything."""
    from paper_2404_16710_amd import rms_norm_grad
    g = gen(d)
    n = 9
    x, gain, dy = normal(g, n, d), normal(g, d, std=0.2, mean=1.0), normal(g, n, d)
    dy[[0, 4, 8]] = 0
    dy[4, 5] = -0.0
    dx, dgain = rms_norm_grad(x, gain, dy, 1e-5)
    bad = x.clone()
    bad[0, 3], bad[4], bad[8, d - 1] = float("nan"), float("inf"), float("-inf")
    got_dx, got_dgain = rms_norm_grad(bad, gain, dy, 1e-5)
    assert torch.equal(got_dgain, dgain) and torch.equal(got_dx, dx) and (dx[[0, 4, 8]] == 0).all()


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
    # (16 bits and at most 64 rows: two parts, 2^-17)
    dp = q * (dl + dlse + 290 * U)[:, None] + 2 * U * (q + p.abs()) + (half(T) if dtype == "f32" or len(p) > 64 else 2.0 ** -17) * p.abs()
    planes = 6 if dtype == "f32" else 2
    want = p @ wd
    tol = dp @ wd.abs() + (planes * vocab + 20) * U * (p.abs() @ wd.abs()) + half(T) * want.abs()
    check(dh, want, tol + 1e-30, "dh")
    want = p.T @ hd
    tol = dp.T @ hd.abs() + (planes * n + 20) * U * (p.T.abs() @ hd.abs()) + half(T) * want.abs()
    check(dw, want, tol + 1e-30, "dW")
    skipped = t.long() < 0
    assert (dh[skipped] == 0).all() and (loss2[skipped] == 0).all()


HEAD_SHAPES = [(1, 16, 1), (1, 16, 17), (2, 48, 31), (1, 256, 1024), (16, 80, 100), (17, 64, 64), (45, 256, 1024), (5, 2048, 333), (64, 208, 1000),
               (65, 128, 2064), (77, 1040, 4099), (97, 144, 777), (128, 272, 130), (130, 384, 257), (300, 96, 511), (333, 512, 1234), (513, 272, 8200), (1100, 64, 96)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, d, vocab", HEAD_SHAPES)
def test_head_loss_and_gradients(n, d, vocab, dtype):
    check_head(*head_case(n, d, vocab, dtype, n + d + vocab, pad=24 if n % 2 else 0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_targets_outside_the_vocabulary(dtype):
    from paper_2404_16710_amd import head_loss, head_loss_grad
    h, w, t, weight = head_case(40, 64, 200, dtype, 5)
    t[7] = 200
    loss, lse = head_loss(h, w, t)
    assert loss[7].isnan() and not lse[7].isnan() and not loss[torch.arange(40) != 7].isnan().any()
    loss, dh, dw = head_loss_grad(h, w, t, weight)
    assert loss[7].isnan() and dh[7].isnan().all() and dw.isnan().all() and not dh[torch.arange(40) != 7].isnan().any()
    t[:] = -1                                        # nothing counts
    loss, dh, dw = head_loss_grad(h, w, t, weight)
    assert (loss == 0).all() and (dh == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_rows_are_independent_of_what_else_is_not_finite(dtype):
    from paper_2404_16710_amd import head_loss
    for n in (9, 150):
        h, w, t, _ = head_case(n, 128, 700, dtype, n)
        want = head_loss(h, w, t)
        h2 = h.clone()
        h2[5, 3] = float("nan")
        got = head_loss(h2, w, t)
        keep = torch.arange(n, device="cuda") != 5
        assert got[1][5].isnan() and torch.equal(got[0][keep], want[0][keep]) and torch.equal(got[1][keep], want[1][keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, d, vocab", [(4, 64, 100), (40, 208, 700), (70, 144, 300), (100, 1040, 515), (150, 128, 700), (333, 272, 1030)])
def test_skipped_rows_may_hold_anything(n, d, vocab, dtype):
    """Padding: what stands in a row without a target reaches neither the other rows nor dW."""
    from paper_2404_16710_amd import head_loss_grad
    h, w, t, weight = head_case(n, d, vocab, dtype, n, pad=16)
    t[n - 1] = -1
    want = head_loss_grad(h, w, t, weight)
    for bad in (float("nan"), float("inf")):
        h2, weight2 = h.clone(), weight.clone()
        h2[1, 2], h2[n - 1], weight2[n - 1] = bad, bad, bad
        got = head_loss_grad(h2, w, t, weight2)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n, shift", [(3, 1000.0), (100, 1000.0), (100, -1000.0)])
def test_head_loss_of_large_logits(n, shift):
    """Logits of a thousand and more: exponentials are taken of differences only.  A shared shift of all logits changes no loss."""
    from paper_2404_16710_amd import head_loss
    g = gen(n)
    d, vocab = 64, 300
    h, w = normal(g, n, d), normal(g, vocab, d)
    h[:, 0], w[:, 0] = 1.0, shift
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda").to(torch.int32)
    check(head_loss(h, w, t)[0], *head_reference(h, w, t, torch.ones(n, device="cuda"))[2:3],
          sum(head_reference(h, w, t, torch.ones(n, device="cuda"))[4:6]), "loss")


def test_head_gradients_in_chunks_of_rows():
    """More rows than 4 GB of logits and p hold: dW is added up over chunks, the last of them shorter."""
    from paper_2404_16710_amd import head_loss_grad
    n, d, vocab = 20011, 32, 100003
    h, w, t, weight = head_case(n, d, vocab, "bf16", 11)
    loss, dh, dw = head_loss_grad(h, w, t, weight)
    sum_p, sum_h = torch.zeros(vocab, d, dtype=torch.float64, device="cuda"), 0.0
    tol = torch.zeros_like(sum_p)
    for a in range(0, n, 2048):
        sl = slice(a, a + 2048)
        hd, wd, ls, lse, dl, dlse, p, q, wt = head_reference(h[sl], w, t[sl], weight[sl])
        check(loss[sl], ls, dl + dlse + 2 * U * ls.abs(), "loss")
        dp = q * (dl + dlse + 290 * U)[:, None] + 2 * U * (q + p.abs()) + half(torch.bfloat16) * p.abs()
        want = p @ wd
        check(dh[sl], want, dp @ wd.abs() + (vocab + 20) * U * (p.abs() @ wd.abs()) + half(torch.bfloat16) * want.abs() + 1e-30, "dh")
        sum_p += p.T @ hd
        tol += dp.T @ hd.abs() + (n + 20) * U * (p.T.abs() @ hd.abs())
    check(dw, sum_p, tol + half(torch.bfloat16) * sum_p.abs() + 1e-30, "dW")


def test_head_gradients_agree_with_differences():
    """Central differences of the loss itself, in a direction: (f(x + s) - f(x - s)) / 2 against <gradient, s>."""
    from paper_2404_16710_amd import head_loss, head_loss_grad
    h, w, t, weight = head_case(70, 64, 500, "f32", 21)
    _, dh, dw = head_loss_grad(h, w, t, weight)
    g = gen(22)
    for x, grad, i in ((h, dh, 0), (w, dw, 1)):
        step = normal(g, *x.shape) * 2 ** -8
        up, down = x + step, x - step                # (the differences below use the steps as fp32 took them)
        step = (up.double() - down.double()) / 2
        f = [(head_loss(*((y, w) if i == 0 else (h, y)), t)[0].double() * weight).sum() for y in (up, down)]
        slope = (grad.double() * step).sum()
        # third order of the loss: |s . x|^3 / 6 with |s . x| of at most 2^-8 * 6 * 16; fp32 losses to 1e-6 of their sum
        assert abs((f[0] - f[1]) / 2 - slope) <= 2e-2 * abs(slope) + 1e-4 * float(weight.sum()), (i, f, slope)


# ---- AdamW -----------------------------------------------------------------------------------------------------------
def adam_reference(p, g, m, v, step, lr, betas, eps, decay):
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    return p * (1 - lr * decay) - lr * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + eps), m, v


def decoded(codes, scale):
    n = codes.numel()
    return codes.double() * scale.double().repeat_interleave(256)[:n]


SIZES = [1, 3, 4, 255, 256, 257, 0, 1000, 4096, 4097, 20001]


@pytest.mark.parametrize("param", ["f32", "bf16", "master"])
@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_steps(bits, param):
    from paper_2404_16710_amd import AdamW
    g = gen(bits)
    dtype = torch.float32 if param == "f32" else torch.bfloat16
    sizes = SIZES * 8                                # more tensors than a launch takes
    params = [normal(g, k, std=0.1).to(dtype) for k in sizes]
    grads = [torch.empty(k, dtype=torch.float32 if i % 3 == 0 else dtype, device="cuda") for i, k in enumerate(sizes)]
    masters = [p.float() for p in params] if param == "master" else None
    hyper = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    opt = AdamW(params, grads, masters=masters, bits=bits, **hyper)
    names = ("m", "v") if bits == 32 else ("m", "r")
    for step in range(1, 4):
        for i, x in enumerate(grads):
            x.copy_(normal(g, x.numel()) * 10.0 ** ((i + step) % 5 - 3))
            if x.numel() > 200:
                x[17::3] = 0                         # (with state zero: nothing but decay)
        before = []
        for i in range(len(sizes)):
            st = opt.states[i]
            m = st["m"].double() if bits == 32 else decoded(st["m"], st["m_scale"])
            v = st["v"].double() if bits == 32 else decoded(st["r"], st["r_scale"]) ** 2
            before.append(((masters or params)[i].double(), grads[i].double(), m, v))
        opt.step()
        for i, k in enumerate(sizes):
            if k == 0:
                continue
            st = opt.states[i]
            p, m, v = adam_reference(*before[i], step, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"])
            p0, g0, m0, v0 = before[i]
            # decoding, and three roundings of each product and sum; then a dozen of the step
            dm, dv = 6 * U * (0.9 * m0.abs() + 0.1 * g0.abs()), 8 * U * v
            near = (p - p0 * (1 - 1e-3)).abs()
            rel = dm / m.abs().clamp(min=1e-300) + dv / v.clamp(min=1e-300)
            dp = 4 * U * p0.abs() + near * (14 * U + rel)
            if masters is not None:
                check(masters[i], p, dp + 1e-30, "master")
                assert torch.equal(params[i], masters[i].to(dtype))
            else:
                check(params[i], p, dp + half(dtype) * p.abs() + 1e-30, "param")
            if bits == 32:
                check(st["m"], m, dm + 1e-30, "m")
                check(st["v"], v, dv + 1e-30, "v")
                continue
            # e4m3: half a step is 2^-4 of the value, 2^-10 of a scale below 2^-6; a root is never rounded to zero
            for name, x, dx in (("m", m, dm), ("r", v.sqrt(), dv / v.sqrt().clamp(min=1e-300))):
                scale = st[name + "_scale"].double()
                top = torch.zeros(2, scale.numel() * 256, dtype=torch.float64, device="cuda")
                top[0, :k], top[1, :k] = x.abs(), dx
                want_scale, off = top.view(2, -1, 256).amax(2) / 448
                check(scale, want_scale, 2 * U * want_scale + off + 1e-30, name + "_scale")
                each = scale.repeat_interleave(256)[:k]
                low = 2.0 ** -9 if name == "r" else 2.0 ** -10
                check(decoded(st[name], scale), x, x.abs() * (2.0 ** -4 + 40 * U) + dx + low * each + 1e-30, name)
                assert (decoded(st["r"], st["r_scale"])[v > 0] > 0).all()


def test_adamw_codes_are_those_of_torch():
    """The states as e4m3 hold exactly what rounding to torch.float8_e4m3fn gives."""
    from paper_2404_16710_amd import AdamW
    g = gen(4)
    grad = normal(g, 1 << 16) * torch.exp(2 * normal(g, 1 << 16))
    grad[0::256] = 448.0                             # scales of exactly 2^0 * 0.5: the products with their inverses are exact
    grad.clamp_(-448.0, 448.0)
    opt = AdamW([torch.zeros(1 << 16, device="cuda")], [grad], bits=8, betas=(0.5, 0.5), eps=1e-8)
    opt.step()
    st = opt.states[0]
    assert (st["m_scale"] == 0.5).all()
    assert torch.equal(st["m"].float(), (0.5 * grad / 0.5).to(torch.float8_e4m3fn).float())


def test_adamw_with_gradients_that_are_not_finite():
    from paper_2404_16710_amd import AdamW
    for bits, hit in ((32, 1), (8, 256)):
        p, g = torch.ones(1024, device="cuda"), torch.ones(1024, device="cuda")
        g[300] = float("inf")
        opt = AdamW([p], [g], bits=bits, lr=1e-2)
        opt.step()
        g[300] = 1.0
        opt.step()
        assert int(p.isnan().sum()) == hit and p[256:512].isnan().sum() == hit


# ---- together ------------------------------------------------------------------------------------------------------------
def tiny(dtype, ffn=1088, d=384):
    import workloads as W
    m = W.ModelConfig(name="fit", n_layers=3, n_q_heads=4, n_kv_heads=2, head_dim=128, d_model=d, ffn_dim=ffn, vocab=1040,
                      rope_base=10000.0, rms_eps=1e-5, dtype=dtype)
    return W.Workload(m, exit_layer=1, draft_len=5, n_prompt=70, n_new=8, resid_scale=0.1, gain_jitter=0.1)


@pytest.mark.parametrize("dtype, n, ffn", [("bf16", 70, 1088), ("bf16", 70, 1040), ("bf16", 9, 1088), ("f32", 70, 1040), ("f32", 1, 1040)])
def test_exit_loss_of_a_text_and_a_step_of_the_head(dtype, n, ffn):
    """States as the debug capture shows them, then norm, head, gradients and update, each against its formula on those states."""
    import workloads as W
    from paper_2404_16710_amd import LsModel, rms_norm
    w = tiny(dtype, ffn)
    ws, prompt = W.make_weights(w), [int(t) for t in W.make_prompt(w)][:n]
    gm = LsModel(w.model, ws, max_seq=96)
    hidden = gm.debug_capture()
    argmax, _ = gm.score(prompt)
    states = hidden[:, :n].clone()
    gm.debug_capture(False)
    head, gain = (gm._dev_weights.by_name[(k, -1)] for k in ("lm_head", "final_norm"))
    targets = [*prompt[1:], -1] if n > 1 else [5]
    counted = max(1, sum(t >= 0 for t in targets))
    scales = {1: 0.25, 3: 1.0}
    h = torch.cat([rms_norm(states[e - 1], gain, w.model.rms_eps) for e in scales])
    t = torch.tensor(targets * 2, dtype=torch.int32, device="cuda")
    weight = torch.tensor([s / counted for s in scales.values() for _ in range(n)], device="cuda")
    hd, wd, loss, lse, dl, dlse, p, q, wt = head_reference(h, head, t, weight)
    losses = gm.exit_loss(prompt, scales, targets)
    tol = torch.where(t.long() >= 0, dl + dlse + 2 * U * loss.abs(), 0.0)
    check(torch.from_numpy(losses).cuda().view(-1), loss, tol, "loss")

    opt = gm.head_optimizer(lr=1e-2, betas=(0.9, 0.95))
    before = [(m if opt.masters else x).double() for x, m in zip(opt.params, opt.masters or opt.params)]
    again = gm.fit_exits(prompt, scales, opt, targets)
    assert (again == losses).all() or abs(again - losses).max() <= 2 * float(tol.max())
    T = TYPES[dtype]
    # (16 bits and at most 64 rows: two parts, 2^-17)
    dp = q * (dl + dlse + 290 * U)[:, None] + 2 * U * (q + p.abs()) + (half(T) if dtype == "f32" or len(p) > 64 else 2.0 ** -17) * p.abs()
    planes = 6 if dtype == "f32" else 2
    want = p.T @ hd
    d_head = opt.grads[0]
    check(d_head, want, dp.T @ hd.abs() + (planes * 2 * n + 20) * U * (p.T.abs() @ hd.abs()) + half(T) * want.abs() + 1e-30, "dW")
    # the gain's gradient from dh, which is rounded to the model's type on the way
    x = torch.cat([states[e - 1] for e in scales]).double()
    r = 1 / torch.sqrt(x.square().mean(1, keepdim=True) + w.model.rms_eps)
    dh = p @ wd
    ddh = dp @ wd.abs() + (planes * p.shape[1] + 20) * U * (p.abs() @ wd.abs()) + half(T) * dh.abs()
    want = (dh * x * r).sum(0)
    tol = (ddh * (x * r).abs()).sum(0) + (2 * n + 40) * U * (dh * x * r).abs().sum(0) + half(T) * want.abs()
    check(opt.grads[1], want, tol + 1e-30, "dgain")
    for i, x in enumerate(opt.params):
        g = opt.grads[i].double()
        new, _, _ = adam_reference(before[i], g, torch.zeros_like(g), torch.zeros_like(g), 1, 1e-2, (0.9, 0.95), 1e-8, 0.0)
        check((opt.masters or opt.params)[i], new, 4 * U * before[i].abs() + 40 * U * 1e-2 + 1e-30, "step")
    # the stepped head is the one that answers: its own losses are those of the formula with the new weights
    h = torch.cat([rms_norm(states[e - 1], gain, w.model.rms_eps) for e in scales])
    hd, wd, loss, lse, dl, dlse, *_ = head_reference(h, head, t, weight)
    tol = torch.where(t.long() >= 0, dl + dlse + 2 * U * loss.abs(), 0.0)
    check(torch.from_numpy(gm.exit_loss(prompt, scales, targets)).cuda().view(-1), loss, tol, "loss of the new head")
    gm.close()


def test_every_replay_of_captured_operators_repeats_them():
    from paper_2404_16710_amd import AdamW, head_loss_grad, rms_norm, rms_norm_grad
    g = gen(31)
    n, d, vocab = 90, 256, 1500
    x, gain = normal(g, n, d), normal(g, d, std=0.1, mean=1.0).bfloat16()
    w = normal(g, vocab, d, std=0.1).bfloat16()
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda").to(torch.int32)
    weight = torch.rand(n, generator=g, device="cuda")

    def step():
        h = rms_norm(x, gain, 1e-5)
        loss, dh, dw = head_loss_grad(h, w, t, weight)
        return loss, dw, *rms_norm_grad(x, gain, dh, 1e-5)

    want = [y.clone() for y in step()]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(4):
        head_loss_grad(normal(g, 40, d).bfloat16(), w, t[:40], weight[:40])        # other work, eager
        for y in got:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    # on another stream, with the inputs made there
    with torch.cuda.stream(side):
        x2 = x.clone()
        got = rms_norm(x2, gain, 1e-5), *rms_norm_grad(x2, gain, normal(g, n, d).bfloat16(), 1e-5)
    torch.cuda.synchronize()
    assert torch.equal(got[0], rms_norm(x, gain, 1e-5))
    p, grad = normal(g, 5000), normal(g, 5000)
    opt = AdamW([p], [grad], bits=8, lr=1e-3)
    opt.step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
        opt.step(step=2)
    saved = [x.clone() for x in (p, *opt.states[0].values())]
    opt.step(step=2)
    want = [x.clone() for x in (p, *opt.states[0].values())]
    for _ in range(3):
        for a, b in zip((p, *opt.states[0].values()), saved):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a, b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)
                   for a, b in zip((p, *opt.states[0].values()), want))


def test_fp32_products_keep_24_bits():
    """One product a sum: x = hi + mid + lo to 2^-25 of it, six of nine products of planes, what is left out is below 2^-24 of the product,
    and six additions round."""
    from paper_2404_16710_amd import head_loss, head_loss_grad
    g = gen(41)
    for n in (3, 70, 200):
        h, w = torch.zeros(n, 64, device="cuda"), torch.zeros(1, 64, device="cuda")
        h[:, 37], w[0, 37] = normal(g, n), 1.2345678
        _, lse = head_loss(h, w, torch.zeros(n, dtype=torch.int32, device="cuda"))
        want = h[:, 37].double() * w[0, 37].double()
        check(lse, want, 9 * U * want.abs(), "lse")
    # a single row with a weight: dW[v] = p[v] h, so every element over its h is the same p; dh[:, k] = p[0] (W[0, k] - W[1, k]) over two rows
    n, d = 90, 64
    h, w = normal(g, n, d), normal(g, 2, d)
    weight = torch.zeros(n, device="cuda")
    weight[57] = 1.0
    _, dh, dw = head_loss_grad(h, w, torch.zeros(n, dtype=torch.int32, device="cuda"), weight)
    p = dw.double() / h[57].double()
    check(p, p[:, :1].expand_as(p), 18 * U * p.abs(), "dW / h")
    want = p[:1, :1] * w[0].double() + p[1:, :1] * w[1].double()
    check(dh[57], want[0], 18 * U * (p[:1, :1] * w[0].double()).abs()[0] + 18 * U * (p[1:, :1] * w[1].double()).abs()[0], "dh")


def c_call(name, *args):
    from paper_2404_16710_amd import binding as B
    code = getattr(B.lib(), name)(*args, torch.cuda.current_stream().cuda_stream)
    assert code == 0, (name, code)


class Guarded:
    """A buffer between two strips of a pattern, for writes that miss it."""

    def __init__(self, nbytes, fill=0xA5):
        self.all = torch.full((nbytes + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
        self.all[4096:4096 + nbytes] = fill
        self.nbytes = nbytes

    @property
    def ptr(self):
        return self.all.data_ptr() + 4096

    def view(self, dtype, *shape):
        return self.all[4096:4096 + self.nbytes].view(dtype).view(*shape)

    def check(self):
        assert (self.all[:4096] == 0x5A).all() and (self.all[4096 + self.nbytes:] == 0x5A).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n, d, vocab", [(1, 16, 1), (3, 80, 77), (20, 208, 515), (70, 144, 1001), (130, 1040, 300), (300, 528, 65)])
def test_nothing_is_written_outside_outputs_and_workspace(n, d, vocab, dtype):
    """Through the C interface, with a workspace of exactly the size asked for that holds NaN, outputs in wider rows, and rows behind
    the last one left as they were."""
    from paper_2404_16710_amd import binding as B
    T, code = TYPES[dtype], B.LS_BF16 if dtype == "bf16" else B.LS_F32
    size = 2 if dtype == "bf16" else 4
    h, w, t, weight = head_case(n, d, vocab, dtype, n + vocab)
    loss, dh, dw, lse = Guarded(4 * n), Guarded(size * n * (d + 16)), Guarded(size * vocab * d), Guarded(4 * n)
    nbytes = B.lib().ls_head_loss_workspace(n, d, vocab, code, 1)
    ws = Guarded(nbytes, 0xFF)
    c_call("ls_head_loss_grad", h.data_ptr(), d, w.data_ptr(), code, t.data_ptr(), weight.data_ptr(), n, d, vocab, loss.ptr, lse.ptr, dh.ptr,
           d + 16, dw.ptr, ws.ptr, nbytes)
    torch.cuda.synchronize()
    for g in (loss, dh, dw, lse, ws):
        g.check()
    assert (dh.view(T, n, d + 16)[:, d:].view(torch.uint8) == 0xA5).all()
    hd, wd, want, want_lse, dl, dlse, p, q, wt = head_reference(h, w, t, weight)
    check(lse.view(torch.float32, n), want_lse, dlse, "lse")
    assert not dh.view(T, n, d + 16)[:, :d].isnan().any() and not dw.view(T, vocab, d).isnan().any()
    nbytes = B.lib().ls_head_loss_workspace(n, d, vocab, code, 0)
    ws, again = Guarded(nbytes, 0xFF), Guarded(4 * n)
    c_call("ls_head_loss", h.data_ptr(), d, w.data_ptr(), code, t.data_ptr(), n, d, vocab, again.ptr, None, ws.ptr, nbytes)
    x, gain, y, dx, dgain = h.float(), w[0].contiguous(), Guarded(size * n * (d + 16)), Guarded(4 * n * (d + 16)), Guarded(size * d)
    c_call("ls_rms_norm", x.data_ptr(), B.LS_F32, d, gain.data_ptr(), code, n, d, 1e-5, y.ptr, d + 16)
    nbytes = B.lib().ls_rms_norm_grad_workspace(n, d)
    ws2 = Guarded(nbytes, 0xFF)
    c_call("ls_rms_norm_grad", x.data_ptr(), B.LS_F32, d, gain.data_ptr(), code, h.data_ptr(), d, n, d, 1e-5, dx.ptr, d + 16, dgain.ptr, ws2.ptr, nbytes)
    torch.cuda.synchronize()
    for g in (ws, again, y, dx, dgain, ws2):
        g.check()
    check(again.view(torch.float32, n), want, torch.where(t.long() >= 0, dl + dlse + 2 * U * want.abs(), 0.0), "loss")
    assert (y.view(T, n, d + 16)[:, d:].view(torch.uint8) == 0xA5).all() and (dx.view(torch.float32, n, d + 16)[:, d:].view(torch.uint8) == 0xA5).all()


def test_calls_on_two_streams_at_once():
    from paper_2404_16710_amd import head_loss_grad, rms_norm_grad
    cases = [head_case(n, 512, 3001, "bf16", n) for n in (40, 300)]
    x = [normal(gen(i), 700, 1040) for i in range(2)]
    gain = torch.ones(1040, device="cuda")
    want = [[*head_loss_grad(*c), *rms_norm_grad(y, gain, y, 1e-5)] for c, y in zip(cases, x)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append([*head_loss_grad(*cases[i]), *rms_norm_grad(x[i], gain, x[i], 1e-5)])
    torch.cuda.synchronize()
    for i in range(2):
        for run in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[i]))
