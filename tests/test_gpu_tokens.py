"""Operators on token tables on the GPU against their definitions in 64 bits, within
bounds that tokens_ref.py derives."""
from __future__ import annotations

import sys

import pytest
import torch

import tokens_ref as ref

pytestmark = pytest.mark.gpu
BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")
LOWEST = torch.finfo(torch.float32).min


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def tk():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    from paper_2608_12629_amd import tokens
    return tokens


def within(got, want, bound, what):
    got, want = got.double(), want.double()
    inf = ~want.isfinite()
    assert torch.equal(got[inf], want[inf]), f"{what}: values that are not finite"
    err = torch.where(inf, 0.0, (got - want).abs())
    over = err > torch.where(inf, INF, bound.expand_as(err))
    worst = (err / bound.expand_as(err).clamp(min=1e-300)).amax().item() if err.numel() else 0.0
    say(f"{what}: worst error {worst:.3f} of the bound")
    assert not (over | got.isnan()).any(), f"{what}: {int(over.sum())} outside, worst {worst:.2f}"


def ids(B, M, V, seed, none=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, V, (B, M), device="cuda", generator=g)
    r = torch.rand((B, M), device="cuda", generator=g)
    t = torch.where(r < 0.3, t % max(1, V // 50 + 1), t)  # some tokens often
    t = torch.where(r > 1 - none, torch.where(r > 1 - none / 2, -1, V), t)  # none, on both sides
    return t.to(torch.int32)


def rows(shape, dt, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) * std).to(dt)


def grid_rows(shape, dt, seed):
    """Sixteenths of at most 8 bits: sums of products are exact, equal scores real ties."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) * 16).round().clamp(-127, 127).div(16).to(dt)


# ---- lookup --------------------------------------------------------------------------
EMBED = [(1, 1, 1, 1, F32), (1, 1, 300, 1024, BF), (2, 5, 257, 8, F16), (1, 1000, 1000, 33, BF),
         (3, 77, 64, 100, F32), (1, 4097, 50, 512, F16), (2, 3, 9, 8192, BF), (1, 130, 7, 6, F32),
         (1, 2, 1 << 20, 16, BF)]


@pytest.mark.parametrize("B,M,V,D,dt", EMBED)
def test_embed(tk, B, M, V, D, dt):
    W, t = rows((B, V, D), dt, 1), ids(B, M, V, 2)
    for scale in (1.0, 11.3137085, -0.3):
        assert torch.equal(tk.tokens_embed(W, t, scale), ref.embed(W, t, scale))


def test_embed_offsets_past_32_bits(tk):
    V, D = 1 << 20, 4096  # 8 GiB of bf16
    W = torch.empty((V, D), dtype=BF, device="cuda")
    W[-3:] = rows((3, D), BF, 3)
    W[:2] = rows((2, D), BF, 4)
    t = torch.tensor([V - 1, 0, V - 3, 1, V - 2], dtype=torch.int32, device="cuda")
    assert torch.equal(tk.tokens_embed(W, t)[0], W[t.long()])


@pytest.mark.parametrize("B,M,V,D,dt", EMBED + [(1, 20_000, 70_000, 24, BF), (2, 9_000, 3, 40, F32),
                                                (1, 5_000, 300_000, 8, F16), (1, 70_001, 900, 64, BF)])
def test_embed_grad(tk, B, M, V, D, dt):
    G, t = rows((B, M, D), dt, 5), ids(B, M, V, 6)
    G = torch.where(((t < 0) | (t >= V)).unsqueeze(-1), float("nan"), G)  # rows that are not read
    for out in {dt, F32}:
        into = rows((B, V, D), out, 7)
        for scale in (1.0, 5.6568542):
            want, bound = ref.embed_grad(G, t, V, scale, dt=out)
            got = tk.tokens_embed_grad(G, t, V, scale, out=torch.full_like(into, float("nan")))
            within(got, want, bound, f"embed_grad {B, M, V, D, dt, out}")
            again = tk.tokens_embed_grad(G, t, V, scale, out=torch.empty_like(into))
            assert torch.equal(got, again)
        want, bound = ref.embed_grad(G, t, V, 0.5, into=into, dt=out)
        got = tk.tokens_embed_grad(G, t, V, 0.5, out=into.clone(), accumulate=True)
        within(got, want, bound, "accumulated")
        untouched = torch.ones((B, V), dtype=torch.bool, device="cuda")
        for b in range(B):
            untouched[b, t[b][(t[b] >= 0) & (t[b] < V)].long()] = False
        assert torch.equal(got[untouched], into[untouched])


def test_embed_grad_of_no_tokens_and_of_one(tk):
    G = rows((1, 3_000, 72), BF, 8)
    t = torch.full((1, 3_000), -1, dtype=torch.int32, device="cuda")
    assert not tk.tokens_embed_grad(G, t, 11).any()
    keep = rows((1, 11, 72), BF, 9)
    assert torch.equal(tk.tokens_embed_grad(G, t, 11, out=keep.clone(), accumulate=True), keep)
    t.fill_(10)  # one token everywhere: a run over every slice
    want, bound = ref.embed_grad(G, t, 11, 1.0)
    within(tk.tokens_embed_grad(G, t, 11), want, bound, "one token")


# ---- log probabilities ---------------------------------------------------------------
SCORES = [(1, 1, 1, 8, BF), (1, 1, 300, 64, BF), (2, 5, 257, 40, F16), (1, 300, 256, 33, BF),
          (3, 257, 1000, 200, F16), (1, 64, 5000, 256, BF), (1, 1025, 513, 1000, BF),
          (1, 2, 70_001, 96, BF), (1, 17, 3_000, 2048, F16), (1, 700, 20_000, 128, BF),
          (2, 33, 40_000, 64, F16), (1, 1, 12_345, 8192, BF), (1, 40, 999, 7, BF)]


def check_logprobs(tk, X, W, t, scale, bias, k, what):
    got = tk.tokens_logprobs(X, W, t, k=k, scale=scale, bias=bias)
    want = ref.logprobs(X, W, t, scale, bias, k)
    tol = ref.logprob_bound(X, W, scale, bias)
    V = W.shape[1]
    within(got[0], want[0], tol, f"logprob {what}")
    # dH = -sum dp (log p + H): a score's error times at most 2 (log V + 1)
    within(got[1], want[1], tol * 2 * (1 + torch.log(torch.tensor(float(V + 1)))), f"entropy {what}")
    within(got[2], want[2], tol, f"lse {what}")
    if k:
        assert torch.equal(got[3], want[3]), f"alternatives {what}"
        within(got[4], want[4], tol.unsqueeze(-1), f"top logprob {what}")
    again = tk.tokens_logprobs(X, W, t, k=k, scale=scale, bias=bias)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)
    return got


@pytest.mark.parametrize("B,M,V,D,dt", SCORES)
def test_logprobs(tk, B, M, V, D, dt):
    X, W, t = rows((B, M, D), dt, 11), rows((B, V, D), dt, 12), ids(B, M, V, 13)
    check_logprobs(tk, X, W, t, 1.7 / D ** 0.5, None, 0, f"{B, M, V, D, dt}")
    bias = rows((B, V), F32, 14)
    bias[rows((B, V), F32, 15) > 0.7] = -INF
    check_logprobs(tk, X, W, t, -2.1 / D ** 0.5, bias, 0, f"{B, M, V, D, dt} masked")


@pytest.mark.parametrize("B,M,V,D,dt", SCORES)
@pytest.mark.parametrize("k", [1, 5, 32])
def test_alternatives(tk, B, M, V, D, dt, k):
    k = min(k, V)
    X, W, t = grid_rows((B, M, D), dt, 21), grid_rows((B, V, D), dt, 22), ids(B, M, V, 23)
    W[:, V // 2:V // 2 * 2] = W[:, :V // 2].clone()  # every row twice: ties
    check_logprobs(tk, X, W, t, 0.125, None, k, f"{B, M, V, D, dt} k={k}")
    bias = torch.zeros((B, V), device="cuda")
    bias[rows((B, V), F32, 25) > -0.7] = -INF
    bias[:, V // 3:V // 3 + 100] = 0.5
    check_logprobs(tk, X, W, t, 0.125, bias, k, f"{B, M, V, D, dt} k={k} masked")


def test_alternatives_in_increasing_and_equal_scores(tk):
    V, D = 9_000, 64
    X = torch.ones((1, 3, D), dtype=BF, device="cuda")
    X[0, 1] = -1
    W = torch.zeros((1, V, D), dtype=BF, device="cuda")
    n = torch.arange(V, device="cuda")
    for j in range(14):  # scores 0 .. V - 1: the bits of the row's number
        W[0, :, j] = ((n >> j) & 1).to(BF) * 2.0 ** j
    t = torch.tensor([[0, 0, V - 1]], dtype=torch.int32, device="cuda")
    got = check_logprobs(tk, X, W, t, 2.0 ** -7, None, 20, "increasing")
    assert got[3][0, 0].tolist() == list(range(V - 1, V - 21, -1))
    assert got[3][0, 1].tolist() == list(range(20))
    W.zero_()
    got = check_logprobs(tk, X, W, t, 1.0, None, 32, "equal")
    assert got[3][0, 2].tolist() == list(range(32))


def test_largest_table(tk):
    V = 1 << 20
    X, W = grid_rows((1, 2, 8), BF, 26), grid_rows((1, V, 8), BF, 27)
    t = torch.tensor([[V - 1, 7]], dtype=torch.int32, device="cuda")
    check_logprobs(tk, X, W, t, 0.25, None, 32, "largest table")


def test_masks(tk):
    """Masks that leave one token or none, masks of the type's lowest value, and NaN and
    infinities in what is masked."""
    B, M, V, D = 3, 70, 600, 48
    X, W, t = grid_rows((B, M, D), BF, 31), grid_rows((B, V, D), BF, 32), ids(B, M, V, 33)
    bias = torch.zeros((B, V), device="cuda")
    bias[0] = -INF
    bias[1] = -INF
    bias[1, 411] = 3.0
    got = check_logprobs(tk, X, W, t, 0.25, bias, 5, "none and one")
    assert (got[2][0] == -INF).all() and (got[3][0] == -1).all() and (got[1][:2] == 0).all()
    assert (got[3][1, :, 0] == 411).all() and (got[3][1, :, 1:] == -1).all()
    bias[0] = LOWEST  # every token at the lowest value: they are all alike
    bias[1, 411] = LOWEST
    bias[2, ::2] = LOWEST
    got = tk.tokens_logprobs(X, W, t, scale=0.25, bias=bias)
    has = (t[0] >= 0) & (t[0] < V)
    logv = torch.log(torch.tensor(float(V))).item()
    assert (got[1][0] - logv).abs().max() < 1e-5
    assert (got[0][0][has] + logv).abs().max() < 1e-5 and (got[2][0] == LOWEST).all()
    even = torch.where(torch.arange(V, device="cuda") % 2 == 0, -INF, 0.0)
    bias[2] = even
    want = tk.tokens_logprobs(X, W, t, scale=0.25, bias=bias)
    assert torch.equal(got[1][2], want[1][2]) and torch.equal(got[2][2], want[2][2])
    clean = [a.clone() for a in tk.tokens_logprobs(X, W, t, k=5, scale=0.25, bias=bias)]
    W[2, ::4] = float("nan")
    W[2, 2::4] = INF
    for a, b in zip(clean, tk.tokens_logprobs(X, W, t, k=5, scale=0.25, bias=bias)):
        assert torch.equal(a, b)


def test_a_row_with_nan_stays_alone(tk):
    X, W, t = grid_rows((1, 300, 64), BF, 35), grid_rows((1, 900, 64), BF, 36), ids(1, 300, 900, 37)
    clean = [a.clone() for a in tk.tokens_logprobs(X, W, t, k=4, scale=0.25)]
    X[0, 17, 3] = float("nan")
    X[0, 290, 60] = INF
    got = tk.tokens_logprobs(X, W, t, k=4, scale=0.25)
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[17] = keep[290] = False
    for a, b in zip(clean, got):
        assert torch.equal(a[0, keep], b[0, keep])
    assert got[2][0, 17].isnan() and got[1][0, 17].isnan()
    assert (got[3] < 900).all() and (got[3] >= -1).all()


def test_blocks_of_rows(tk):
    """So many scores that the rows are taken in blocks (k > 0)."""
    M, V, D = 2_700, 131_072, 32
    X, W, t = grid_rows((1, M, D), F16, 38), grid_rows((1, V, D), F16, 39), ids(1, M, V, 40)
    got = tk.tokens_logprobs(X, W, t, k=3, scale=0.25)
    for r in (slice(0, 40), slice(2_030, 2_070), slice(2_660, 2_700)):
        want = ref.logprobs(X[:, r], W, t[:, r], 0.25, None, 3)
        tol = ref.logprob_bound(X[:, r], W, 0.25, None)
        within(got[0][:, r], want[0], tol, "logprob")
        assert torch.equal(got[3][:, r], want[3])


def test_outputs_passed_in_and_left_out(tk):
    X, W, t = rows((2, 50, 64), BF, 41), rows((2, 333, 64), BF, 42), ids(2, 50, 333, 43)
    full = tk.tokens_logprobs(X, W, t, k=3, scale=0.1)
    assert tk.tokens_logprobs(X, W, scale=0.1)[0] is None
    assert torch.equal(tk.tokens_logprobs(X, W, k=3, scale=0.1)[3], full[3])
    outs = dict(logprob=torch.empty((2, 50), device="cuda"), entropy=torch.empty((2, 50), device="cuda"),
                lse=torch.empty((2, 50), device="cuda"),
                top_idx=torch.empty((2, 50, 3), dtype=torch.int32, device="cuda"),
                top_logprob=torch.empty((2, 50, 3), device="cuda"),
                ws=torch.empty(tk.logprobs_workspace_bytes(2, 50, 333, 64, 3, BF), dtype=torch.uint8,
                               device="cuda"))
    got = tk.tokens_logprobs(X, W, t, k=3, scale=0.1, **outs)
    for a, b, n in zip(got, full, ("logprob", "entropy", "lse", "top_idx", "top_logprob")):
        assert a is outs[n] and torch.equal(a, b)


# ---- gradients -----------------------------------------------------------------------
def check_grads(tk, X, W, t, g, h, scale, bias, what):
    _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=scale, bias=bias)
    kw = dict(entropy=ent if h is not None else None, grad_entropy=h, scale=scale, bias=bias)
    B, M, D = X.shape
    dX = torch.full((B, M, D), float("nan"), dtype=X.dtype, device="cuda")
    dW = torch.full(W.shape, float("nan"), dtype=X.dtype, device="cuda")
    tk.tokens_logprobs_grad(X, W, t, lse, g, dX=dX, dW=dW, **kw)
    wX, wW, eX, eW = ref.grads(X, W, t, g, h, scale, bias)
    within(dX, wX, eX, f"dX {what}")
    within(dW, wW, eW, f"dW {what}")
    dX2, dW2 = tk.tokens_logprobs_grad(X, W, t, lse, g, **kw)
    assert torch.equal(dX, dX2) and torch.equal(dW, dW2)
    return dX, dW


@pytest.mark.parametrize("B,M,V,D,dt", SCORES + [(1, 5_000, 300, 64, BF), (2, 3_000, 257, 320, F16),
                                                 (1, 64, 30_000, 512, BF)])
def test_logprobs_grad(tk, B, M, V, D, dt):
    X, W, t = rows((B, M, D), dt, 51), rows((B, V, D), dt, 52), ids(B, M, V, 53)
    g = rows((B, M), F32, 54)
    check_grads(tk, X, W, t, g, None, 1.7 / D ** 0.5, None, f"{B, M, V, D, dt}")
    bias = rows((B, V), F32, 55)
    bias[rows((B, V), F32, 56) > 0.7] = -INF
    check_grads(tk, X, W, t, g, rows((B, M), F32, 57, 0.3), -2.1 / D ** 0.5, bias,
                f"{B, M, V, D, dt} masked, entropy")


def test_grads_of_rows_and_tokens_that_take_no_part(tk):
    B, M, V, D = 2, 300, 700, 64
    for dt in (BF, F16):
        X, W, t = rows((B, M, D), dt, 61), rows((B, V, D), dt, 62), ids(B, M, V, 63)
        g, h = rows((B, M), F32, 64), rows((B, M), F32, 65, 0.1)
        bias = torch.zeros((B, V), device="cuda")
        bias[:, 5::7] = -INF
        bias[1, 200:] = -INF
        idle = torch.arange(M, device="cuda") % 3 == 0
        g[:, idle] = 0
        h[:, idle] = 0
        want = check_grads(tk, X, W, t, g, h, 0.2, bias, "some rows idle")
        X2, W2 = X.clone(), W.clone()
        X2[:, idle] = float("nan")
        W2[:, 5::7] = INF
        _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.2, bias=bias)
        got = tk.tokens_logprobs_grad(X2, W2, t, lse, g, entropy=ent, grad_entropy=h, scale=0.2, bias=bias)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert not got[0][:, idle].any() and not got[1][:, 5::7].any()
        bias.fill_(-INF)  # no token is allowed
        _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.2, bias=bias)
        got = tk.tokens_logprobs_grad(X, W, t, lse, g, entropy=ent, grad_entropy=h, scale=0.2, bias=bias)
        assert not got[0].any() and not got[1].any()


def test_gradients_of_very_different_sizes(tk):
    """fp16: positions whose gradients are six orders apart, and large and tiny losses."""
    X, W, t = rows((1, 200, 96), F16, 71), rows((1, 500, 96), F16, 72), ids(1, 200, 500, 73, none=0)
    for top in (1.0, 3e4, 1e-4):
        g = rows((1, 200), F32, 74) * torch.logspace(0, -6, 200, device="cuda") * top
        check_grads(tk, X, W, t, g, None, 0.1, None, f"up to {top}")


def test_blocks_of_table_rows(tk):
    """dz past what is stored at once: several blocks of table rows, instances one by one."""
    for B, M, V, D in ((1, 6_000, 50_000, 40), (2, 3_000, 50_000, 32)):
        X, W, t = rows((B, M, D), BF, 81), rows((B, V, D), BF, 82), ids(B, M, V, 83)
        check_grads(tk, X, W, t, rows((B, M), F32, 84), None, 0.3, None, f"{B, M, V, D}")


def test_gradients_against_differences(tk):
    """Central differences of the 64-bit loss in a direction, from 16-bit points: the
    gradient's component off by at most its bound plus the difference's own h^2 term."""
    B, M, V, D = 1, 24, 60, 16
    X, W, t = rows((B, M, D), BF, 91), rows((B, V, D), BF, 92), ids(B, M, V, 93)
    g, h = rows((B, M), F32, 94), rows((B, M), F32, 95)
    dX, dW = check_grads(tk, X, W, t, g, h, 0.4, None, "small")
    _, _, eX, eW = ref.grads(X, W, t, g, h, 0.4, None)

    def loss(x, w):
        lp, ent, _ = ref.logprobs(x, w, t, 0.4)
        return (lp * g + ent * h).sum().item()

    for seed in range(4):
        a = rows((B, M, D), torch.float64, 96 + seed)
        b = rows((B, V, D), torch.float64, 196 + seed)
        step = 1e-4
        for u, v in ((a, 0 * b), (0 * a, b)):
            num = (loss(X.double() + step * u, W.double() + step * v) -
                   loss(X.double() - step * u, W.double() - step * v)) / (2 * step)
            ana = ((dX.double() * u).sum() + (dW.double() * v).sum()).item()
            bound = ((eX * u.abs()).sum() + (eW * v.abs()).sum()).item()
            assert abs(num - ana) <= bound + 1e-4 * (1 + abs(num)), (num, ana, bound)


# ---- together, streams, graphs ---------------------------------------------------------
def test_codes_of_k_means_learned_with_one_table(tk):
    """Points clustered and encoded, their codes looked up in a table, scored against the
    same table, and the table's gradient from both ends in one buffer."""
    from paper_2608_12629_amd import kmeans as km
    N, D, K = 4_096, 64, 500
    X = rows((1, N, D), BF, 101)
    C = X[:, :K].float().contiguous()
    km.kmeans_lloyd(X, C, 3)
    codes, _ = km.kmeans_assign(X, C)
    W, scale = C.to(BF), 0.3
    emb = tk.tokens_embed(W, codes, 2.0)
    assert torch.equal(emb, ref.embed(W, codes, 2.0))
    nxt = torch.roll(codes, -1, 1)
    lp, ent, lse, top, toplp = tk.tokens_logprobs(emb, W, nxt, k=5, scale=scale)
    want = ref.logprobs(emb, W, nxt, scale)
    within(lp, want[0], ref.logprob_bound(emb, W, scale, None), "logprob")
    assert (toplp[..., 0] >= lp).all()
    g = torch.full((1, N), -1.0 / N, device="cuda")
    dE, dW = tk.tokens_logprobs_grad(emb, W, nxt, lse, g, scale=scale)
    wE, wW, eE, eW = ref.grads(emb, W, nxt, g, None, scale)
    within(dE, wE, eE, "d rows")
    total = tk.tokens_embed_grad(dE, codes, K, 2.0, out=dW.clone(), accumulate=True)
    want, bound = ref.embed_grad(dE, codes, K, 2.0, into=dW)
    within(total, want, bound, "d table")


def test_captured_and_replayed(tk):
    """All four calls in one graph: replays on new inputs equal eager calls, with eager
    work of the same sizes in between; two graphs with a workspace each do not mix."""
    B, M, V, D, k = 2, 300, 3_000, 96, 4

    def fresh(seed):
        return dict(X=rows((B, M, D), BF, seed), W=rows((B, V, D), BF, seed + 1), t=ids(B, M, V, seed + 2),
                    g=rows((B, M), F32, seed + 3), h=rows((B, M), F32, seed + 4))

    def make_ws():
        n = max(tk.logprobs_workspace_bytes(B, M, V, D, k, BF), tk.embed_grad_workspace_bytes(B, M, V, D, BF),
                tk.logprobs_grad_workspace_bytes(B, M, V, D, BF))
        return torch.empty(n, dtype=torch.uint8, device="cuda")

    def go(s, ws):
        lp, ent, lse, ti, tl = tk.tokens_logprobs(s["X"], s["W"], s["t"], k=k, scale=0.1, ws=ws)
        dX, dW = tk.tokens_logprobs_grad(s["X"], s["W"], s["t"], lse, s["g"], entropy=ent,
                                         grad_entropy=s["h"], scale=0.1, ws=ws)
        tk.tokens_embed_grad(dX, s["t"], V, 2.0, out=dW, accumulate=True, ws=ws)
        fresh_grad = tk.tokens_embed_grad(dX, s["t"], V, 2.0, ws=ws)
        return [lp, ent, lse, ti, tl, dX, dW, fresh_grad, tk.tokens_embed(s["W"], s["t"], 3.0)]

    go(fresh(1), make_ws())
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        s, ws = fresh(10 + 10 * i), make_ws()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs = go(s, ws)
        graphs.append((gr, s, ws, outs))
    for r in range(3):
        for i, (gr, s, ws, outs) in enumerate(graphs):
            for n, v in fresh(100 + 20 * r + 10 * i).items():
                s[n].copy_(v)
        for gr, *_ in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for i, (gr, s, ws, outs) in enumerate(graphs):
            want = go(fresh(100 + 20 * r + 10 * i), make_ws())
            for a, b in zip(outs, want):
                assert torch.equal(a, b), (r, i)


def test_two_streams(tk):
    a = (rows((1, 500, 128), BF, 111), rows((1, 5_000, 128), BF, 112), ids(1, 500, 5_000, 113))
    b = (rows((1, 400, 64), F16, 114), rows((1, 7_000, 64), F16, 115), ids(1, 400, 7_000, 116))
    want = [tk.tokens_logprobs(*s, k=3, scale=0.1) for s in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for st, s in zip(streams, (a, b)):
            with torch.cuda.stream(st):
                got.append(tk.tokens_logprobs(*s, k=3, scale=0.1))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        for x, y in zip(r, want[i % 2]):
            assert torch.equal(x, y)


def test_the_binding_refuses(tk):
    X, W, t = rows((2, 10, 64), BF, 121), rows((2, 30, 64), BF, 122), ids(2, 10, 30, 123)
    lse, g = torch.zeros((2, 10), device="cuda"), torch.zeros((2, 10), device="cuda")
    with pytest.raises(ValueError, match="contiguous"):
        tk.tokens_embed(W.transpose(0, 1), t)
    with pytest.raises(ValueError, match="current GPU"):
        tk.tokens_embed(W.cpu(), t)
    with pytest.raises(TypeError, match="idx must be"):
        tk.tokens_embed(W, t.long())
    with pytest.raises(ValueError, match="idx has shape"):
        tk.tokens_embed(W, t[:1])
    with pytest.raises(ValueError, match="out has"):
        tk.tokens_embed(W, t, out=torch.empty((2, 10, 63), dtype=BF, device="cuda"))
    with pytest.raises(TypeError, match="out must be"):
        tk.tokens_embed_grad(X, t, 30, out=torch.empty((2, 30, 64), dtype=F16, device="cuda"))
    with pytest.raises(ValueError, match="pass it in"):
        tk.tokens_embed_grad(X, t, 30, accumulate=True)
    with pytest.raises(ValueError, match="idx has"):
        tk.tokens_embed_grad(X, t[:, :9].contiguous(), 30)
    with pytest.raises(TypeError, match="share a dtype"):
        tk.tokens_logprobs(X, W.half(), t)
    with pytest.raises(ValueError, match="want"):
        tk.tokens_logprobs(X, W[:, :, :32].contiguous(), t)
    with pytest.raises(ValueError, match="bias has"):
        tk.tokens_logprobs(X, W, t, bias=torch.zeros(30, device="cuda"))
    with pytest.raises(tk.KMeansError):
        tk.tokens_logprobs(X, W, t, k=31)
    with pytest.raises(tk.KMeansError):
        tk.tokens_logprobs(X.float(), W.float(), t)
    with pytest.raises(tk.KMeansError):
        tk.tokens_logprobs(X, W, t, scale=float("nan"))
    with pytest.raises(ValueError, match="entropy of the forward"):
        tk.tokens_logprobs_grad(X, W, t, lse, g, grad_entropy=g)
    with pytest.raises(ValueError, match="dW has"):
        tk.tokens_logprobs_grad(X, W, t, lse, g, dW=torch.empty((2, 29, 64), dtype=BF, device="cuda"))
    torch.cuda.synchronize()


# ---- sizes and masks at which the kernels' paths part -----------------------------------
@pytest.mark.parametrize("B,M,V,D,dt", [(1, 200, 40, 64, BF), (1, 256, 300, 1000, F16), (8, 100, 60, 72, BF),
                                        (2, 1000, 33, 16, BF), (1, 65, 64, 8, F16), (5, 4096, 31, 128, BF)])
def test_many_rows_of_small_tables(tk, B, M, V, D, dt):
    X, W, t = grid_rows((B, M, D), dt, 131), grid_rows((B, V, D), dt, 132), ids(B, M, V, 133)
    W[:, V // 2:V // 2 * 2] = W[:, :V // 2].clone()
    for k in (0, min(V, 7)):
        check_logprobs(tk, X, W, t, 0.125, None, k, f"{B, M, V, D, dt} k={k}")
    bias = torch.where(rows((B, V), F32, 134) > 0.5, -INF, rows((B, V), F32, 135).round())
    check_logprobs(tk, X, W, t, -0.25, bias, min(V, 32), "masked")


@pytest.mark.parametrize("k", [1, 20, 32])
def test_alternatives_outside_a_head(tk, k):
    """Many scores: the best ones of the first columns bound the rest.  Those first ones
    forbidden, fewer than k left anywhere, all forbidden, all equal, and every one twice."""
    M, V, D = 300, 70_000, 32
    X, W, t = grid_rows((1, M, D), BF, 141), grid_rows((1, V, D), BF, 142), ids(1, M, V, 143)
    W[:, V // 2:] = W[:, :V // 2].clone()
    check_logprobs(tk, X, W, t, 0.25, None, k, "twice")
    bias = torch.zeros((1, V), device="cuda")
    bias[:, :V // 2] = -INF
    check_logprobs(tk, X, W, t, 0.25, bias, k, "first half forbidden")
    bias[:, 5::3] = -INF
    bias[:, V - 300:] = 2.0
    check_logprobs(tk, X, W, t, -0.25, bias, k, "best last")
    bias.fill_(-INF)
    bias[0, torch.tensor([3, 40_000, 69_999], device="cuda")] = torch.tensor([1.0, 0.0, 1.0], device="cuda")
    got = check_logprobs(tk, X, W, t, 0.25, bias, k, "three left")
    assert (got[3][..., 3:] == -1).all()
    bias.fill_(-INF)
    got = check_logprobs(tk, X, W, t, 0.25, bias, k, "none left")
    assert (got[3] == -1).all()
    got = check_logprobs(tk, X, W, t, 0.0, None, k, "all equal")
    assert torch.equal(got[3], torch.arange(k, device="cuda", dtype=torch.int32).expand(1, M, k))


def test_alternatives_with_nan_rows_of_many_scores(tk):
    M, V, D = 300, 60_000, 24
    X, W, t = grid_rows((1, M, D), F16, 145), grid_rows((1, V, D), F16, 146), ids(1, M, V, 147)
    clean = [a.clone() for a in tk.tokens_logprobs(X, W, t, k=6, scale=0.25)]
    bad = [0, 131, 255, 256, 299]
    X[0, bad, 5] = float("nan")
    got = tk.tokens_logprobs(X, W, t, k=6, scale=0.25)
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[bad] = False
    for a, b in zip(clean, got):
        assert torch.equal(a[0, keep], b[0, keep])
    assert got[2][0, bad].isnan().all() and (got[3] < V).all() and (got[3] >= -1).all()


NARROW = [(1, 63, 65, 1, BF), (1, 64, 64, 16, F16), (2, 65, 129, 64, BF), (1, 129, 127, 65, F16),
          (3, 128, 1, 128, BF), (1, 1, 128, 128, F16), (1, 130, 600, 129, BF), (1, 2_000, 500, 136, F16),
          (2, 300, 300, 192, BF), (1, 900, 4_100, 256, BF), (1, 2_100, 2_100, 256, F16),
          (1, 6_000, 5_700, 256, BF), (1, 4_100, 8_300, 130, BF), (2, 9_000, 2_000, 224, F16),
          (3, 1_030, 900, 31, F16), (1, 20_000, 1_100, 48, BF)]


@pytest.mark.parametrize("B,M,V,D,dt", NARROW)
def test_gradients_of_short_rows(tk, B, M, V, D, dt):
    X, W, t = rows((B, M, D), dt, 151), rows((B, V, D), dt, 152), ids(B, M, V, 153)
    g, h = rows((B, M), F32, 154), rows((B, M), F32, 155, 0.3)
    bias = rows((B, V), F32, 156)
    bias[rows((B, V), F32, 157) > 0.9] = -INF
    scale = 1.7 / D ** 0.5
    g[:, ::5] = 0
    for b, e in ((None, None), (bias, None), (None, h), (bias, h)):
        check_grads(tk, X, W, t, g, e, scale, b, f"{B, M, V, D, dt} {b is not None} {e is not None}")


def test_gradients_of_short_rows_that_take_no_part(tk):
    """Idle positions with NaN, forbidden tokens with NaN, and the last of either idle."""
    for M, V, D in ((193, 257, 40), (700, 129, 200), (70, 1_000, 128)):
        X, W, t = rows((1, M, D), BF, 161), rows((1, V, D), BF, 162), ids(1, M, V, 163)
        for h in (None, rows((1, M), F32, 165, 0.1)):
            g = rows((1, M), F32, 164)
            idle = torch.arange(M, device="cuda") % 3 == (M - 1) % 3
            g[:, idle] = 0
            if h is not None:
                h[:, idle] = 0
            bias = torch.zeros((1, V), device="cuda")
            bias[:, (V - 1) % 5::5] = -INF
            for b in (None, bias):
                want = check_grads(tk, X, W, t, g, h, 0.2, b, f"{M, V, D} idle")
                _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.2, bias=b)
                X2, W2, lse2 = X.clone(), W.clone(), lse.clone()
                X2[:, idle] = float("nan")
                lse2[:, idle] = float("nan")
                if b is not None:
                    W2[:, (V - 1) % 5::5] = float("nan")
                got = tk.tokens_logprobs_grad(X2, W2, t, lse2, g, entropy=ent if h is not None else None,
                                              grad_entropy=h, scale=0.2, bias=b)
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_gradients_with_scale_zero_and_sharp_rows(tk):
    X, W, t = rows((1, 150, 64), F16, 171), rows((1, 300, 64), F16, 172), ids(1, 150, 300, 173)
    g = rows((1, 150), F32, 174)
    dX, dW = check_grads(tk, X, W, t, g, None, 0.0, None, "scale 0")
    assert not dX.any() and not dW.any()
    # one token has all the probability: p is 1 or 0
    check_grads(tk, X, W, t, g, rows((1, 150), F32, 175, 0.1), 30.0, None, "sharp")
    bias = torch.full((1, 300), LOWEST, device="cuda")
    bias[:, 7] = 0
    check_grads(tk, X, W, t, g, rows((1, 150), F32, 176, 0.1), 0.3, bias, "the lowest value")


@pytest.mark.parametrize("B,M,V,D", [(1, 6_000, 50_000, 264), (2, 3_000, 50_000, 260)])
def test_blocks_of_table_rows_of_long_rows(tk, B, M, V, D):
    X, W, t = rows((B, M, D), BF, 181), rows((B, V, D), BF, 182), ids(B, M, V, 183)
    check_grads(tk, X, W, t, rows((B, M), F32, 184), None, 0.1, None, f"{B, M, V, D}")


@pytest.mark.parametrize("M,V,D", [(5_000_000, 40, 264), (6_000_001, 70, 250)])
def test_gradients_of_millions_of_positions(tk, M, V, D):
    """Offsets past 2^31 bytes within a block of rows; the reference in parts."""
    X, W, t = rows((1, M, D), BF, 191), rows((1, V, D), BF, 192), ids(1, M, V, 193)
    g = rows((1, M), F32, 194)
    _, _, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.1)
    dX, dW = tk.tokens_logprobs_grad(X, W, t, lse, g, scale=0.1)
    total, err = 0, 0
    part = 500_000
    for m in range(0, M, part):
        s = slice(m, min(M, m + part))
        wX, wW, eX, eW = ref.grads(X[:, s], W, t[:, s], g[:, s], None, 0.1)
        bad = ((dX[:, s].double() - wX).abs() > eX)
        assert not bad.any(), (m, int(bad.sum()))
        total, err = total + wW, err + eW
    # (the parts' bounds together hold for their sum; a running sum of M terms in fp32
    # within the shares is what eW counts as X.shape[1] steps of a part: M / part times it)
    within(dW, total, err * (M / part), "dW")


def test_embed_grad_by_radix_in_instances(tk):
    for B, M, V, D in ((3, 5_000, 77, 16), (2, 8_193, 70_000, 8), (9, 8_192, 5, 33)):
        G, t = rows((B, M, D), BF, 201), ids(B, M, V, 202)
        want, bound = ref.embed_grad(G, t, V, 0.7)
        got = tk.tokens_embed_grad(G, t, V, 0.7)
        within(got, want, bound, f"{B, M, V, D}")
        assert torch.equal(got, tk.tokens_embed_grad(G, t, V, 0.7))


def test_two_streams_of_gradients(tk):
    a = (rows((1, 500, 128), BF, 211), rows((1, 5_000, 128), BF, 212), ids(1, 500, 5_000, 213))
    b = (rows((1, 400, 320), F16, 214), rows((1, 7_000, 320), F16, 215), ids(1, 400, 7_000, 216))

    def go(X, W, t):
        _, _, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.1)
        g = torch.ones(t.shape, device="cuda")
        dX, dW = tk.tokens_logprobs_grad(X, W, t, lse, g, scale=0.1)
        return dX, dW, tk.tokens_embed_grad(dX, t, W.shape[1])

    want = [go(*s) for s in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        for st, s in zip(streams, (a, b)):
            with torch.cuda.stream(st):
                got.append(go(*s))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        for x, y in zip(r, want[i % 2]):
            assert torch.equal(x, y)


@pytest.mark.parametrize("D", [64, 256, 300])
def test_gradients_captured_and_replayed(tk, D):
    """On both ways of dz, with eager calls between the replays."""
    M, V = 700, 900

    def fresh(seed):
        return rows((1, M, D), F16, seed), rows((1, V, D), F16, seed + 1), ids(1, M, V, seed + 2), \
            rows((1, M), F32, seed + 3)

    def go(X, W, t, g, ws):
        _, ent, lse, _, _ = tk.tokens_logprobs(X, W, t, scale=0.1, ws=ws)
        return tk.tokens_logprobs_grad(X, W, t, lse, g, entropy=ent, grad_entropy=g, scale=0.1, ws=ws)

    def make_ws():
        return torch.empty(max(tk.logprobs_workspace_bytes(1, M, V, D, 0, F16),
                               tk.logprobs_grad_workspace_bytes(1, M, V, D, F16)), dtype=torch.uint8,
                           device="cuda")

    s, ws = fresh(221), make_ws()
    go(*fresh(225), make_ws())
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        outs = go(*s, ws)
    for r in range(4):
        new = fresh(231 + 4 * r)
        for x, y in zip(s, new):
            x.copy_(y)
        gr.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, go(*new, make_ws())):
            assert torch.equal(x, y), r


@pytest.mark.parametrize("B,M,V,D", [(8, 1, 8_931, 586), (1, 12, 4_477, 704), (1, 64, 300, 64), (1, 65, 300, 64),
                                     (1, 3, 50, 1_000)])
@pytest.mark.parametrize("entropy", [False, True])
def test_fp16_gradients_of_few_positions(tk, B, M, V, D, entropy):
    """Rows made mostly by one token's dz: forms of a target's dz of any size next to 1 - p."""
    X, W, t = rows((B, M, D), F16, 241), rows((B, V, D), F16, 242), ids(B, M, V, 243, none=0.1)
    for lean in (0.0, 0.5, 3.0):  # p of the target from near 0 to near 1
        at = torch.where((t >= 0) & (t < V), t, 0).long().unsqueeze(-1).expand(-1, -1, D)
        Y = (X.float() + lean * torch.gather(W, 1, at).float()).half()
        g = rows((B, M), F32, 244) * torch.logspace(0, -4, M, device="cuda")
        h = rows((B, M), F32, 245, 0.2) if entropy else None
        check_grads(tk, Y, W, t, g, h, 2.0 / D ** 0.5, None, f"{B, M, V, D} {lean}")


@pytest.mark.parametrize("D", [1, 64, 200, 300])
@pytest.mark.parametrize("V", [1, 2, 33, 65])
def test_fp16_gradients_where_the_last_token_has_all_the_probability(tk, D, V):
    M = 5
    X, W = rows((1, M, D), F16, 251), rows((1, V, D), F16, 252, 0.1)
    X[0, :, 0], W[0, V - 1, 0] = 4.0, 4.0
    t = torch.full((1, M), V - 1, dtype=torch.int32, device="cuda")
    for h in (None, rows((1, M), F32, 254)):
        check_grads(tk, X, W, t, rows((1, M), F32, 253), h, 1.0, None, f"{V, D}")
        check_grads(tk, X, W, t - 1, rows((1, M), F32, 253), h, 1.0, None, f"{V, D} another")


def test_blocks_of_table_rows_of_many_results(tk):
    """Several blocks of table rows and so many results of dX that each block adds to them."""
    M, V, D = 9_000, 32_000, 2_304
    X, W, t = rows((1, M, D), BF, 261), rows((1, V, D), BF, 262), ids(1, M, V, 263)
    check_grads(tk, X, W, t, rows((1, M), F32, 264), None, 0.02, None, f"{M, V, D}")
