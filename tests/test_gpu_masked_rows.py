"""Tokens that a mask or a NaN leaves without an expert, through locmoe_route and the block's steps behind it: every index stays
one of an expert, and other tokens keep their results.

A score is 1 / sum exp(v - best): the argument's rounding is at most |v - best| f, 8 f here, the exponential's 2 f, the sum's
E f and the quotient's 2 f, f = 2^-24: (E + 12) f.
"""
import numpy as np
import pytest

from test_gpu_block import Setup
from paper_2401_13920_amd import workloads as wl

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2401_13920_amd import harness, locmoe as lm
    assert torch.cuda.is_available(), "these tests need the MI355X"
    lm.lib()
    return torch, lm, harness


def expected(G, relu):
    """eid and w (NaN where there is no choice or a NaN takes part) of values G, float32."""
    if relu:
        G = np.where(np.isnan(G), 0.0, np.maximum(G, 0.0)).astype(np.float32)
    eid = np.argmax(np.where(np.isnan(G), -np.inf, G), axis=1)
    G = G.astype(np.float64)
    with np.errstate(invalid="ignore"):
        return eid, 1.0 / np.exp(G - G[np.arange(len(G)), eid][:, None]).sum(axis=1)


def rows(rng, T, E):
    """Gating values in [-4, 4] among which some tokens have nothing, a NaN, a mask over all but one or over the first half."""
    g = rng.uniform(-4.0, 4.0, (T, E)).astype(np.float32)
    g[0] = -np.inf
    if T > 1:
        g[T - 1] = np.nan
    if T > 6:
        g[2] = -np.inf
        g[2, E - 1] = -3.0
        g[3, :E // 2] = -np.inf
        g[4, 0] = np.nan
        g[5, E // 2:] = np.nan
        g[T // 2] = np.where(np.arange(E) % 2, np.nan, -np.inf)
    return g


# one launch and two, one expert and several a lane, a work-group's tokens and more
@pytest.mark.parametrize("T,E,N", [(1, 1, 1), (1, 4, 2), (9, 5, 5), (192, 16, 4), (2049, 4, 2), (700, 64, 8), (4099, 96, 6),
                                   (300, 300, 3), (65, 1024, 16)])
@pytest.mark.parametrize("relu", [False, True])
def test_route(env, T, E, N, relu):
    torch, lm, _ = env
    print(f"[route masked] T={T} E={E} N={N} relu={relu}", flush=True)
    rng = np.random.default_rng(T + E)
    g = rows(rng, T, E)
    desc = lm.make_desc(T, 8 * E, E, N, 8, T, relu=relu)
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    home = torch.from_numpy(rng.integers(0, N, T).astype(np.int32)).cuda()
    e2n = torch.from_numpy((np.arange(E) % N).astype(np.int32)).cuda()
    n = lm.locmoe_workspace_bytes(desc)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    for eps in (None, np.full(E, -np.inf, np.float32)):
        for map_ in (e2n, None):        # (None: node e / (E / N))
            eid, w, cnt = torch.full((T,), 99, **i32), torch.full((T,), 7.0, **f32), torch.full((E,), 99, **i32)
            Psum, stats = torch.empty(E, **f32), torch.empty(8, **f32)
            e = None if eps is None else torch.from_numpy(eps).cuda()
            lm.locmoe_route(desc, torch.from_numpy(g).cuda(), e, home, map_, eid, w, cnt, Psum, stats, ws, n)
            want, score = expected(g if eps is None else g + eps, relu)
            assert np.array_equal(eid.cpu().numpy(), want)
            assert np.array_equal(cnt.cpu().numpy(), np.bincount(want, minlength=E))
            got = w.double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(score))
            live = ~np.isnan(score)
            assert (np.abs(got - score)[live] <= (E + 12) * F * score[live]).all()


def clean_and_nan(env, T, dtype):
    """A block whose gate has no ReLU, and the same with a NaN in a token of expert 0."""
    torch, lm, _ = env
    s = Setup(env, wl.small_config(T=T, d=192, E=6, N=3, h=104, dtype=dtype), T)
    s.desc.relu, s.desc.mu = 0, 0.0
    lm.forward_block(s.desc, s.xd, s.homed, None, *s.Wd, s.block, s.b, s.kb)
    m = int((s.b.eid == 0).nonzero()[0, 0])
    bad = s.xd.clone()
    bad[m, 77] = float("nan")
    return s, bad, m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [40, 700])
def test_block_with_a_nan_token(env, T, dtype):
    """The norm makes all of the token NaN, its gating values too: expert 0, as before, and no other token changes."""
    torch, lm, _ = env
    print(f"[block NaN] T={T} {dtype}", flush=True)
    s, bad, m = clean_and_nan(env, T, dtype)
    gb, others = lm.alloc_grad_buffers(s.desc), [k for k in range(T) if k != m]
    got = []
    for x in (s.xd, bad):
        lm.forward_block_train(s.desc, x, s.homed, None, *s.Wd, s.block, s.b, s.kb, gb)
        lm.backward_block(s.desc, s.dyd, x, s.homed, None, *s.Wt, s.block, s.b, s.kb, gb)
        got.append([t.clone() for t in (s.b.eid, s.b.slot, s.b.cnt, s.b.y[others], gb.dx[others], gb.dW_in[1:], gb.dW_out[1:])])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.isnan(s.b.w[m]) and torch.isnan(s.b.y[m]).all() and torch.isnan(gb.dx[m]).all()
    assert all(torch.isfinite(t).all() for t in got[0][3:])
    if T <= lm.LOCMOE_FEW_MAX_TOKENS:
        lm.decode_block(s.desc, bad, *s.Wd, s.block, s.b, s.kb)
        assert torch.equal(s.b.eid, got[0][0]) and torch.isnan(s.b.y[m]).all() and torch.isfinite(s.b.y[others]).all()


def test_block_without_experts(env):
    """Every expert masked: all tokens to expert 0 with a score of NaN; those past its capacity pass on the residual."""
    torch, lm, hz = env
    s = Setup(env, wl.small_config(T=50, d=192, E=6, N=3, h=104), 20)
    s.desc.relu = 0
    eps = torch.full((6,), -float("inf"), device="cuda")
    for run in (lambda: lm.forward_block(s.desc, s.xd, s.homed, None, *s.Wd, s.block, s.b, s.kb, eps=eps),
                lambda: lm.decode_block(s.desc, s.xd, *s.Wd, s.block, s.b, s.kb, eps=eps)):
        s.b.y.fill_(7.0)
        run()
        assert (s.b.eid == 0).all() and torch.isnan(s.b.w).all()
        assert (s.b.slot[:20] >= 0).all() and (s.b.slot[20:] == -1).all()
        assert torch.isnan(s.b.y[:20]).all() and torch.equal(s.b.y[20:], s.xd[20:])


def test_gradients_beside_masked_experts(env):
    """locmoe_route_bwd with experts masked by -inf and the locality loss on (0 ln 0 = 0): the formula, which central differences
    of the objective bear out.  With D = max |dw| + max |coef|: p is (E + 12) f off (above), <p, dp> (2 E + 14) f D, and three
    roundings follow: (4 E + 42) f D; and in coef 80 additions of fp32 behind P, mu / T of them each."""
    torch, lm, _ = env
    for T, E, N in ((37, 6, 3), (5000, 12, 4)):     # one launch and three
        print(f"[route_bwd masked] T={T} E={E}", flush=True)
        rng = np.random.default_rng(T)
        g, dw = rng.normal(size=(T, E)).astype(np.float32), rng.normal(size=T).astype(np.float32)
        eps = np.where(np.arange(E) % 3 == 1, -np.inf, 0.1 * rng.normal(size=E)).astype(np.float32)
        home, alpha, mu = rng.integers(0, N, T).astype(np.int32), 0.3, 0.2
        desc = lm.make_desc(T, 8 * E, E, N, 8, T, relu=False, alpha=alpha, mu=mu)
        i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
        eid, w, cnt, Psum, stats = torch.empty(T, **i32), torch.empty(T, **f32), torch.empty(E, **i32), torch.empty(E, **f32), torch.empty(8, **f32)
        n = lm.locmoe_workspace_bytes(desc)
        gd, epsd, homed, dwd = (torch.from_numpy(a).cuda() for a in (g, eps, home, dw))
        lm.locmoe_route(desc, gd, epsd, homed, None, eid, w, cnt, Psum, stats, torch.empty(n, dtype=torch.uint8, device="cuda"), n)
        coef, dg = torch.empty(E, **f32), torch.empty(T, E, **f32)
        lm.locmoe_route_bwd(desc, gd, epsd, homed, None, eid, cnt, Psum, dwd, coef, dg)
        assert torch.isfinite(stats).all() and torch.isfinite(coef).all() and (Psum[1::3] == 0).all()
        e, live = eid.cpu().numpy(), np.isfinite(eps)
        assert live[e].all()
        f = np.bincount(e, minlength=E) / T
        Dl = np.repeat(np.bincount(home, minlength=N), E // N) / (T * (E // N))

        def probs(G):
            z = np.exp(G - G.max(axis=1, keepdims=True))
            return z / z.sum(axis=1, keepdims=True)

        def objective(G):
            p = probs(G)
            P = p.mean(axis=0)
            return (dw * p[np.arange(T), e]).sum() + alpha * E * f @ P + mu * np.sum(P[live] * np.log(P[live] / Dl[live]))

        G = (g + eps).astype(np.float64)
        p = probs(G)
        c = alpha * E * f / T
        c[live] += mu * (np.log(p.mean(axis=0)[live] / Dl[live]) + 1) / T
        dp = c[None, :] + dw[:, None] * (np.arange(E)[None, :] == e[:, None])
        ref = p * (dp - (p * dp).sum(axis=1, keepdims=True))
        for m, i in ((0, 0), (T // 2, 2), (T - 1, E - 1)):
            step = np.zeros_like(G)
            step[m, i] = 1e-5
            assert abs((objective(G + step) - objective(G - step)) / 2e-5 - ref[m, i]) <= 1e-7
        got = dg.double().cpu().numpy()
        assert (got[:, ~live] == 0).all()
        D = np.abs(dw).max() + np.abs(c).max()
        assert (np.abs(got - ref) <= (4 * E + 42) * F * D + 80 * F * mu / T).all()


def few(env, T, d, E, C, relu, dtype="bf16"):
    """locmoe_layer_few's call with weights of ones: f(x, g) -> eid, w, slot, y."""
    torch, lm, _ = env
    desc = lm.make_desc(T, d, E, 1, 8, C, dtype, relu)
    W_in, W_out = (torch.ones(E, *s, dtype=torch.bfloat16, device="cuda") for s in ((8, d), (d, 8)))
    n = lm.locmoe_layer_few_workspace_bytes(desc)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")

    def call(x, g=None):
        i32 = dict(dtype=torch.int32, device="cuda")
        eid, slot, w, y = torch.full((T,), 99, **i32), torch.full((T,), 99, **i32), torch.full((T,), 7.0, device="cuda"), torch.full_like(x, 7.0)
        lm.locmoe_layer_few(desc, x, g, None, W_in, W_out, True, eid, w, slot, y, ws, n)
        return eid, w, slot, y
    return desc, call


@pytest.mark.parametrize("T,E", [(1, 1), (1, 4), (9, 5), (7, 12), (64, 16), (33, 96), (2, 257), (64, 1024)])
@pytest.mark.parametrize("relu", [False, True])
def test_few_tokens(env, T, E, relu):
    """The layer for a few tokens takes the experts that locmoe_route takes, NaN or not."""
    torch, lm, _ = env
    print(f"[few masked] T={T} E={E} relu={relu}", flush=True)
    rng = np.random.default_rng(T + E)
    C = max(1, T // 2)
    _, call = few(env, T, 8 * E, E, C, relu)
    x = torch.ones(T, 8 * E, dtype=torch.bfloat16, device="cuda")
    # NaN in each place of a row by itself too: the first of a lane's experts, a later one, the only one above the rest
    sets = [rows(rng, T, E)]
    for at in range(0, E, max(1, E // 5)):
        g = rng.uniform(-4.0, 4.0, (T, E)).astype(np.float32)
        g[::2, at] = np.nan
        sets.append(g)
    for g in sets:
        eid, w, slot, y = call(x, torch.from_numpy(g).cuda())
        want, score = expected(g, relu)
        assert np.array_equal(eid.cpu().numpy(), want)
        place = [m if (want[:m] == want[m]).sum() < C else -1 for m in range(T)]
        assert slot.tolist() == place
        got = w.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(score))
        live = ~np.isnan(score)
        assert (np.abs(got - score)[live] <= (E + 12) * F * score[live]).all()
        dead = torch.tensor([p >= 0 and not l for p, l in zip(place, live)], device="cuda")
        assert torch.isnan(y[dead]).all() and torch.isfinite(y[~dead]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("relu", [False, True])
def test_nan_in_x_of_a_few_tokens(env, relu, dtype):
    """Gating values formed by the layer: a NaN in x reaches its own block's value, so the token goes where locmoe_gate and
    locmoe_route send it, and no other token changes."""
    torch, lm, _ = env
    for T, d, E in ((1, 64, 8), (5, 96, 12), (17, 600, 50), (64, 1024, 64)):
        print(f"[few NaN in x] T={T} d={d} E={E} relu={relu} {dtype}", flush=True)
        gen = torch.Generator(device="cuda").manual_seed(T)
        desc, call = few(env, T, d, E, T, relu, dtype)
        x = torch.randn(T, d, generator=gen, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        clean = call(x)
        for m, at in ((0, 0), (T // 2, d // 2), (T - 1, d - 1)):
            bad = x.clone()
            bad[m, at] = float("nan")
            eid, w, slot, y = call(bad)
            g, rest = torch.empty(T, E, device="cuda"), [k for k in range(T) if k != m]
            lm.locmoe_gate(desc, bad, g)
            want, _ = expected(g.cpu().numpy(), relu)
            assert eid.tolist() == want.tolist() and slot.tolist() == list(range(T))
            assert bool(torch.isnan(w[m])) == (not relu) and torch.isnan(y[m]).all()
            assert torch.equal(w[rest], clean[1][rest]) and torch.isfinite(y[rest]).all()
