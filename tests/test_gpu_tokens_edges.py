"""Operators on token tables on the GPU where their paths part: small tables with many
scores, offsets of the type's lowest value, rows and tokens that take no part, gradients
of sizes far apart.  References in 64 bits, bounds from the roundings."""
from __future__ import annotations

import pytest
import torch

import tokens_ref as ref
from test_gpu_tokens import BF, F16, F32, INF, LOWEST, grid_rows, ids, rows, tk, within  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- the k best of small tables with many scores --------------------------------------
@pytest.mark.parametrize("B,M,V", [(1, 4_096, 4_096), (1, 8_192, 2_048), (8, 512, 4_096), (1, 8_200, 1_793),
                                   (1, 4_100, 3_841)])
@pytest.mark.parametrize("k", [1, 2])
@pytest.mark.parametrize("dt", [BF, F16])
def test_best_of_small_tables_with_many_scores(tk, B, M, V, k, dt):
    """From a workspace full of large scores, and then of another call's."""
    D, scale = 32, 0.125
    n = tk.logprobs_workspace_bytes(B, M, V, D, k, dt)
    ws = (rows((n // 4 + 1,), F32, 300).abs() * 1e30).view(torch.uint8)
    for seed in (301, 311):
        X, W, t = grid_rows((B, M, D), dt, seed), grid_rows((B, V, D), dt, seed + 1), ids(B, M, V, seed + 2)
        for masked in (False, True):
            bias = None
            if masked:
                bias = torch.zeros((B, V), device="cuda")
                bias[rows((B, V), F32, seed + 3) > 0.3] = -INF
                bias[:, :V // 3] = -INF  # no token of the first columns
            got = tk.tokens_logprobs(X, W, t, k=k, scale=scale, bias=bias, ws=ws)
            want = ref.logprobs(X, W, t, scale, bias, k)
            what = f"{B, M, V} k={k} masked={masked}"
            assert torch.equal(got[3], want[3]), f"alternatives {what}"
            within(got[4], want[4], ref.logprob_bound(X, W, scale, bias).unsqueeze(-1), f"top logprob {what}")
            again = tk.tokens_logprobs(X, W, t, k=k, scale=scale, bias=bias,
                                       ws=torch.full_like(ws, 0x42))
            assert torch.equal(got[3], again[3]) and torch.equal(got[4], again[4])


# ---- gradients ------------------------------------------------------------------------
# What tokens_ref.grads allows, with less slack: dz rounds to fp16 for either storage type
# (half a step, 2^-11, or half the smallest step 2^-24 of what is stored 2048 times larger
# over the row's scale, which is at most 4 times the larger gradient), and the errors of
# scores are given per token.
U, H16 = 2.0 ** -24, 2.0 ** -11


def sharp_grads(z, zerr, X, W, t, g, h, scale):
    """dX, dW and their bounds from the scores z in 64 bits (-inf: forbidden), off by zerr."""
    dt, (B, M, V) = X.dtype, z.shape
    lse = torch.logsumexp(z, -1, keepdim=True)
    logp = z - lse
    p = torch.exp(logp)
    plogp = torch.where(p > 0, p * logp, 0.0)
    ent = -plogp.sum(-1, keepdim=True)
    has = (t >= 0) & (t < V)
    at = torch.where(has, t, 0).long().unsqueeze(-1)
    has = has & (torch.gather(z, 2, at).squeeze(-1) > -INF)
    g = torch.where(has, g.double(), 0.0).unsqueeze(-1)
    h = torch.zeros_like(g) if h is None else h.double().unsqueeze(-1)
    active = (g != 0) | (h != 0)
    keep = active & (z > -INF)
    hot = torch.zeros_like(z).scatter_(2, at, 1.0)
    dz = torch.where(keep, g * (hot - p) - h * (plogp + p * ent), 0.0)
    # p's error: of its score, of the lse (the row's largest), of exponentials and their sums
    dp = 2 * zerr + 2 * torch.where(z > -INF, zerr, 0.0).amax(-1, keepdim=True) + (128 + V / 256) * 4 * U
    mag = (g.abs() + h.abs() * (2 + logp.clamp(min=-100).abs() + ent)) * p
    e = torch.where(keep, dp * mag + H16 * (dz.abs() + dp * mag), 0.0)
    gs = torch.where(active, torch.maximum(g.abs(), h.abs()), 0.0) * 4
    e = torch.where(keep, e + gs * 2.0 ** -25 / 2048, 0.0)
    Xd = torch.where(active, X.double(), 0.0)
    Wd = torch.where((z > -INF).any(1).unsqueeze(-1), W.double(), 0.0)
    dzt, et = dz.transpose(1, 2).contiguous(), e.transpose(1, 2).contiguous()
    dX, dW = torch.matmul(dz, Wd) * scale, torch.matmul(dzt, Xd) * scale
    eX = torch.matmul(e + V * U * (dz.abs() + e), Wd.abs()) * abs(scale)
    eW = torch.matmul(et + M * U * (dzt.abs() + et), Xd.abs()) * abs(scale)
    # the copies of W and X below 2^-28 of the largest (X's times their rows' scales)
    eX += dz.abs().sum(-1, keepdim=True) * Wd.abs().amax((1, 2), keepdim=True) * 2.0 ** -38 * abs(scale)
    per = torch.where(gs > 0, dz.abs() / gs.clamp(min=1e-300), 0.0).sum(1).unsqueeze(-1)
    eW += per * gs.amax(1, keepdim=True) * Xd.abs().amax((1, 2), keepdim=True) * 2.0 ** -38 * abs(scale)
    if dt == F16 and B * M <= 64:  # X times a row's scale, no power of two here
        eW += H16 * torch.matmul(dzt.abs() + et, Xd.abs()) * abs(scale)
    tiny = torch.finfo(dt).smallest_normal * ref.half(dt) * 2
    eX = eX + ref.half(dt) * (dX.abs() + eX) + tiny
    eW = eW + ref.half(dt) * (dW.abs() + eW) + tiny
    return dX, dW, eX, eW


def check_sharp(tk, X, W, t, g, h, scale, bias, z, zerr, what):
    _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=scale, bias=bias)
    got = tk.tokens_logprobs_grad(X, W, t, lse, g, entropy=ent if h is not None else None, grad_entropy=h,
                                  scale=scale, bias=bias)
    wX, wW, eX, eW = sharp_grads(z, zerr, X, W, t, g, h, scale)
    for a, want, bound, n in ((got[0], wX, eX, "dX"), (got[1], wW, eW, "dW")):
        within(a, want, bound, f"{n} {what}")
        # nothing written, or a twentieth of it left out, would show
        assert not (want.abs().amax() > 0) or (bound.norm() < 0.05 * want.norm()), f"{n} {what}: a loose bound"
    return got


def half_rows(shape, dt, seed):
    """Halves: products are quarters."""
    return (rows(shape, F32, seed).round() / 2).to(dt)


@pytest.mark.parametrize("M,V,D", [(300, 700, 64), (40, 500, 128), (500, 600, 250), (60, 700, 300),
                                   (200, 500, 320), (3_000, 4_500, 264)])
@pytest.mark.parametrize("dt", [BF, F16])
def test_gradients_under_offsets_that_all_tokens_share(tk, M, V, D, dt):
    """Offsets of the type's lowest value on every token (all alike) or on the only allowed
    one, and of -2^20: the lse does not hold the logarithm of the sum there."""
    X, W, t = half_rows((3, M, D), dt, 401), half_rows((3, V, D), dt, 402), ids(3, M, V, 403)
    g = rows((3, M), F32, 404)
    bias = torch.full((3, V), -INF, device="cuda")
    bias[0] = LOWEST
    bias[1, V // 2] = LOWEST
    t[1, ::2] = V // 2
    bias[2, 3:] = -2.0 ** 20 - 100
    W[1, 0], W[2, 1] = INF, float("nan")  # forbidden
    z = ref.scores(X, W, 0.5, None)  # eighths, which stay eighths below 2^21
    z[0] = 0
    z[1], z[1, :, V // 2] = -INF, 0
    z[2, :, :3] = -INF
    g[:, ::7] = 0
    for h in (None, rows((3, M), F32, 405, 0.3)):
        _, dW = check_sharp(tk, X, W, t, g, h, 0.5, bias, z, torch.zeros_like(z),
                            f"{M, V, D, dt} {h is not None}")
        assert not dW[1, :V // 2].any() and not dW[1, V // 2 + 1:].any() and not dW[2, :3].any()


def test_gradients_under_lowest_offsets_beside_others(tk):
    """The lowest value on some tokens, 0 on the rest: the same gradients as forbidden ones."""
    for M, V, D in ((300, 700, 64), (60, 700, 300), (3_000, 4_500, 264)):
        X, W, t = rows((1, M, D), BF, 411), rows((1, V, D), BF, 412), ids(1, M, V, 413)
        t[0, ::3] = 1
        g, h = rows((1, M), F32, 414), rows((1, M), F32, 415, 0.3)
        off = rows((1, V), F32, 416) > 0.3
        off[:, 1] = False
        scale = 1 / D ** 0.5
        bias = torch.where(off, LOWEST, 0.0)
        z = ref.scores(X, W, scale, None) + torch.where(off, -1e30, 0.0).double().unsqueeze(1)
        mag = torch.matmul(X.double().abs(), W.double().abs().transpose(1, 2).contiguous()) * scale
        g = torch.where(off[0, t[0].clamp(0, V - 1).long()], 0.0, g)  # (such a target's dz is g)
        for e in (None, h):
            check_sharp(tk, X, W, t, g, e, scale, bias, z, (D + 2) * U * mag, f"{M, V, D} {e is not None}")


@pytest.mark.parametrize("M,V,D", [(300, 700, 64), (500, 600, 250), (60, 700, 300), (60, 700, 299),
                                   (3_000, 4_500, 264), (200, 5_000, 512)])
def test_rows_that_take_no_part_beside_nan(tk, M, V, D):
    """Idle positions get dX 0 whatever an allowed token's row holds, forbidden tokens dW 0
    whatever an active position's row holds."""
    for dt in (BF, F16):
        X, W, t = rows((1, M, D), dt, 421), rows((1, V, D), dt, 422), ids(1, M, V, 423)
        g = rows((1, M), F32, 424)
        g[:, ::3] = 0
        bias = torch.zeros((1, V), device="cuda")
        bias[:, 5::7] = -INF
        for b in (None, bias):
            _, _, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.1, bias=b)
            Y, Z = X.clone(), W.clone()
            Z[0, 3, 1] = float("nan")
            dX, _ = tk.tokens_logprobs_grad(X, Z, t, lse, g, scale=0.1, bias=b)
            assert not dX[:, ::3].any() and dX[0, t[0] == 3].isnan().any(-1).sum() >= (g[0, t[0] == 3] != 0).sum()
            Y[0, 1, 2] = float("nan")
            g[0, 1], t[0, 1] = 1.0, 4
            _, dW = tk.tokens_logprobs_grad(Y, W, t, lse, g, scale=0.1, bias=b)
            assert dW[0, 4].isnan().any()
            if b is not None:
                assert not dW[:, 5::7].any()


def test_instances_and_blocks_that_start_on_odd_elements(tk):
    """dz past what is stored at once: instances one by one, blocks of table rows, each
    with odd sizes, so that every other one's results begin in the middle of a pair."""
    for B, M, V, D in ((2, 12_001, 12_001, 257), (1, 9_001, 40_003, 259)):
        X, W, t = rows((B, M, D), BF, 431), rows((B, V, D), BF, 432), ids(B, M, V, 433)
        g = rows((B, M), F32, 434)
        _, _, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.06)
        dX, dW = tk.tokens_logprobs_grad(X, W, t, lse, g, scale=0.06)
        for b in range(B):
            i = slice(b, b + 1)
            wX, wW, eX, eW = ref.grads(X[i], W[i], t[i], g[i], None, 0.06)
            within(dX[i], wX, eX, f"dX {B, M, V, D} {b}")
            within(dW[i], wW, eW, f"dW {B, M, V, D} {b}")


@pytest.mark.parametrize("M,V,D", [(300, 700, 64), (500, 600, 250), (60, 700, 300), (3_000, 4_500, 264)])
@pytest.mark.parametrize("down", [13, 24, 30, 40])
def test_faint_positions_of_their_own_tokens(tk, M, V, D, down):
    """Half of the positions have gradients 2^down times smaller, and tokens that the other
    half gives no probability: those tokens' gradients are as precise as the others'."""
    X, W = rows((1, M, D), BF, 441), rows((1, V, D), BF, 442)
    faint = torch.arange(M, device="cuda") % 2 == 1
    far = torch.arange(V, device="cuda") % 2 == 1
    X[:, :, :2], W[:, :, :2] = 0, 0  # 400 apart: the products below add a few
    X[0, faint, 0], X[0, ~faint, 1] = 20, 20
    W[0, far, 0], W[0, ~far, 1] = 20, 20
    t = torch.randint(0, V // 2, (1, M), device="cuda") * 2 + faint.int()
    t = t.to(torch.int32)
    g = rows((1, M), F32, 444).abs().clamp(min=0.25)
    h = rows((1, M), F32, 445, 0.1)
    small = torch.where(faint, 2.0 ** -down, 1.0)
    scale = 1.0 if D <= 64 else 0.5
    for ent in (False, True):
        _, e, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=scale)
        kw = dict(entropy=e, scale=scale) if ent else dict(scale=scale)
        even = tk.tokens_logprobs_grad(X, W, t, lse, g, grad_entropy=h if ent else None, **kw)
        got = tk.tokens_logprobs_grad(X, W, t, lse, g * small, grad_entropy=h * small if ent else None, **kw)
        # the same numbers times a power of two, but for what the copies of X and dz round
        # off their smaller values (at most half a step, 2^-11 of a product) and the
        # results' own rounding, half a step of bf16 (2^-8) on both sides
        for a, b, part in ((got[0], even[0], faint), (got[1], even[1], far)):
            x, y = a[0, part].double() * 2.0 ** down, b[0, part].double()
            assert (x - y).norm() <= 2.0 ** -8 * y.norm(), ((x - y).norm() / y.norm()).item()
            assert (x - y).abs().amax() <= 2.0 ** -7 * y.abs().amax()
            assert torch.equal(a[0, ~part], b[0, ~part])


@pytest.mark.parametrize("M,V,D", [(5_000, 700, 64), (5_000, 700, 200), (40, 3_000, 300), (3_000, 4_500, 264)])
@pytest.mark.parametrize("entropy", [False, True])
def test_bf16_gradients_take_dz_in_11_bits(tk, M, V, D, entropy):
    """How many results are not the rounding of the exact ones.  A dz that is off by up to
    2^-11 (2^-12 in the mean) moves a result by no more than that, relative to the root of
    its products' squares, and a result of at least that size (here: of the root mean square
    of all) has steps of 2^-8 of itself or more: at most a sixteenth of them round to
    another value.  With a dz of 8 bits it would be a quarter."""
    X, W, t = rows((1, M, D), BF, 461), rows((1, V, D), BF, 462), ids(1, M, V, 463)
    g = rows((1, M), F32, 464)
    h = rows((1, M), F32, 465, 0.3) if entropy else None
    scale = 1 / D ** 0.5
    _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=scale)
    got = tk.tokens_logprobs_grad(X, W, t, lse, g, entropy=ent if entropy else None, grad_entropy=h, scale=scale)
    want = ref.grads(X, W, t, g, h, scale)

    def off(a, b):
        large = b.abs() >= (b * b).mean().sqrt()
        return (a != b.to(BF))[large].double().mean().item()
    assert off(got[0], want[0]) <= 1 / 16 and off(got[1], want[1]) <= 1 / 16, \
        (off(got[0], want[0]), off(got[1], want[1]))


@pytest.mark.parametrize("M,V,D", [(5_000_000, 40, 264), (6_000_001, 70, 250)])
def test_table_gradients_of_millions_of_positions(tk, M, V, D):
    """dW of sums that do not cancel: every position has the same target and gradient, and
    column d of X the mean 1 + d % 7.  At least 128 shares of M / 128 positions: a running
    sum is off by at most M / 128 steps of 2^-24 of its magnitude, dz by 2^-11, a result by
    half a step of bf16, 2^-8.  Left out, one of 256 shares shows in the mean of all."""
    X = rows((1, M, D), BF, 471, 0.25)
    X += 1 + torch.arange(D, device="cuda").to(BF) % 7
    W = rows((1, V, D), BF, 472)
    t = torch.full((1, M), 3, dtype=torch.int32, device="cuda")
    g, scale = torch.ones((1, M), device="cuda"), 0.02
    _, _, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=scale)
    _, dW = tk.tokens_logprobs_grad(X, W, t, lse, g, scale=scale)
    want = torch.zeros((V, D), dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(want)
    for m in range(0, M, 500_000):
        x, w = X[0, m:m + 500_000].double(), W[0].double()
        dz = -torch.softmax(x @ w.t().contiguous() * scale, -1)
        dz[:, 3] += 1
        dz = dz.t().contiguous()
        want += dz @ x * scale
        mag += dz.abs() @ x.abs() * scale
    sums = M / 128 * U + H16 + 1e-4  # (1e-4: p's error)

    def right(a):
        a = a.double()
        err = (a - want).abs() <= sums * mag + 2.0 ** -8 * (1 + sums) * want.abs()
        # the roundings' mean over V D results: 2^-8 / sqrt(3 V D), five times that
        mean = (a / want - 1).mean().abs() <= sums + 5 * 2.0 ** -8 / (3 * V * D) ** 0.5
        return err.all() and mean
    assert right(dW[0])
    assert not right(torch.zeros_like(want)) and not right(want * (1 - 1 / 256)) and not right(want.roll(1, 1))


# ---- refusals ---------------------------------------------------------------------------
def test_refusals_say_what_is_wrong(tk):
    """The library's own status: sizes and numbers that no call takes are invalid, those
    beyond this build's limits unsupported."""
    from paper_2608_12629_amd.kmeans import ERR_INVALID_ARG, ERR_UNSUPPORTED
    X, W, t = rows((1, 10, 64), BF, 501), rows((1, 50, 64), BF, 502), ids(1, 10, 50, 503)
    none, f = t[:, :0], torch.zeros((1, 10), device="cuda")
    wide = torch.zeros((1, 1, 8_200), dtype=BF, device="cuda")

    def status(want, call, *a, **kw):
        with pytest.raises(tk.KMeansError) as e:
            call(*a, **kw)
        assert e.value.status == want, e.value

    status(ERR_INVALID_ARG, tk.tokens_logprobs, X, W, t, k=-1)
    status(ERR_INVALID_ARG, tk.tokens_logprobs, X, W, t, k=51)
    status(ERR_UNSUPPORTED, tk.tokens_logprobs, X, W, t, k=33)
    status(ERR_INVALID_ARG, tk.tokens_logprobs, X[:, :0], W, none)
    status(ERR_INVALID_ARG, tk.tokens_logprobs, X, W[:, :0], t)
    status(ERR_UNSUPPORTED, tk.tokens_logprobs, X.float(), W.float(), t)
    status(ERR_UNSUPPORTED, tk.tokens_logprobs, wide, wide)
    status(ERR_INVALID_ARG, tk.tokens_embed, W, none)
    status(ERR_INVALID_ARG, tk.tokens_embed_grad, X[:, :0], none, 50)
    status(ERR_INVALID_ARG, tk.tokens_embed_grad, X, t, 0)
    status(ERR_UNSUPPORTED, tk.tokens_embed_grad, X, t, (1 << 20) + 1)
    status(ERR_INVALID_ARG, tk.tokens_logprobs_grad, X[:, :0], W, none, f[:, :0], f[:, :0])
    status(ERR_UNSUPPORTED, tk.tokens_logprobs_grad, X.float(), W.float(), t, f, f)


@pytest.mark.parametrize("B,M,V,D", [(1, 1, 300, 64), (1, 999, 700, 64), (1, 9_001, 500, 40), (1, 300, 900, 320),
                                     (2, 301, 4_001, 24)])
def test_values_that_start_at_any_element(tk, B, M, V, D):
    """Tokens, offsets, statistics and gradients one element into an allocation (the next
    tokens of a sequence) give what copies of them give."""
    def late(x):
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        assert y.data_ptr() % 16 == 4
        return y.copy_(x)

    X, W, t = grid_rows((B, M, D), BF, 511), grid_rows((B, V, D), BF, 512), ids(B, M, V, 513)
    bias, g, h = rows((B, V), F32, 514), rows((B, M), F32, 515), rows((B, M), F32, 516)
    assert torch.equal(tk.tokens_embed(W, late(t)), tk.tokens_embed(W, t))
    assert torch.equal(tk.tokens_embed_grad(X, late(t), V), tk.tokens_embed_grad(X, t, V))
    want = tk.tokens_logprobs(X, W, t, k=3, scale=0.125, bias=bias)
    outs = dict(zip(("logprob", "entropy", "lse", "top_idx", "top_logprob"), (late(a) for a in want)))
    for a in outs.values():
        a.zero_()
    got = tk.tokens_logprobs(X, W, late(t), k=3, scale=0.125, bias=late(bias), **outs)
    for a, b, o in zip(got, want, outs.values()):
        assert a is o and torch.equal(a, b)
    _, ent, lse, _, _ = want
    dX, dW = tk.tokens_logprobs_grad(X, W, t, lse, g, entropy=ent, grad_entropy=h, scale=0.125, bias=bias)
    dX2, dW2 = tk.tokens_logprobs_grad(X, W, late(t), late(lse), late(g), entropy=late(ent), grad_entropy=late(h),
                                       scale=0.125, bias=late(bias))
    assert torch.equal(dX, dX2) and torch.equal(dW, dW2)
