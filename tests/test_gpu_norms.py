"""The norms around the layer against their formulas in float64 (oracle/block_oracle.py).

Tolerances.  u is half a rounding step of the storage type (torch.finfo(t).eps / 2), f = 2^-24 that of fp32.  A mean of squares
is a sum of positive terms with at most CHAIN additions one after another, so it is CHAIN f off, relative to itself, r half
of that and three roundings more: R = CHAIN f covers r, and the products with r, gamma, w and scale (at most six roundings).
  xn             (u + 2 R) |ref|
  g              (2 R + n f) mean |xn| over the n features of the block
  y              u |y| + (2 R + f) (|branch| + |res|)
  dw             (2 R + n f) sum |terms| over the n features
  dgamma         (2 R + n f) sum |terms| over n tokens, n at most the number of tokens
  dout, dx       u |ref| and, for every term of the formula, (2 R + n f) of its magnitude with sums of magnitudes inside
"""
import numpy as np
import pytest

from oracle import block_oracle as blk

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
CHAIN = 8 * 4 + 10 + 16 + 6   # chunks of a lane, a chunk's tree, waves of a row, lanes of a wave
R = CHAIN * F
EPS, SCALE = 1e-5, 0.7


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2401_13920_amd import locmoe as lm
    assert torch.cuda.is_available(), "these tests need the MI355X"
    lm.lib()
    return torch, lm


# every width of a row's lanes and chunks a lane, and each form of the gate: blocks of a power of two of chunks, of whole
# chunks, of neither; one expert, as many experts as features
SHAPES = [(1, 8, 1, "bf16"), (1, 8, 8, "bf16"), (3, 24, 6, "f32"), (65, 48, 6, "bf16"), (70, 128, 8, "bf16"),
          (19, 232, 29, "bf16"), (7, 600, 50, "f32"), (7, 600, 50, "bf16"), (130, 1000, 125, "bf16"), (33, 1000, 8, "f32"),
          (33, 1600, 40, "bf16"), (1100, 1600, 40, "f32"), (257, 2048, 32, "bf16"), (5, 4096, 4, "bf16"), (9, 4096, 64, "f32"),
          (6, 4104, 27, "bf16"), (4, 1024, 1024, "bf16"), (4, 1024, 1, "f32"), (3, 10240, 64, "bf16"), (3, 16384, 64, "bf16"),
          (2, 8200, 41, "f32"), (2, 32768, 16, "bf16"), (2, 32760, 1, "bf16"), (2, 16384, 1024, "f32"), (2500, 128, 8, "f32")]


def case(torch, T, d, E, dtype, seed, drop, gamma):
    rng = np.random.default_rng(seed)
    st = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows = T + 5                       # the send buffer's rows; the last ones belong to no token
    dev = lambda a, t=st: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(t)  # noqa: E731
    p = dict(x=dev(rng.standard_normal((T, d)) * np.exp(rng.standard_normal((T, 1)))), out=dev(rng.standard_normal((rows, d))),
             dy=dev(rng.standard_normal((T, d))), dsend=dev(rng.standard_normal((rows, d))),
             dg=dev(rng.standard_normal((T, E)), torch.float32), w=dev(rng.uniform(0.1, 1, T), torch.float32),
             gi=dev(rng.uniform(0.5, 1.5, d), torch.float32) if gamma else None,
             go=dev(rng.uniform(-1.5, 1.5, d), torch.float32) if gamma else None)
    kept = {"none": np.ones(T, bool), "all": np.zeros(T, bool)}.get(drop, rng.random(T) < 0.7)
    slot = np.where(kept, rng.permutation(T), -1).astype(np.int32)
    unused = np.setdiff1d(np.arange(rows), slot[kept])
    for name in ("out", "dsend"):      # rows of no token are never read
        p[name][torch.from_numpy(unused).cuda()] = float("nan")
    p["slot"], p["kept"], p["unused"] = torch.from_numpy(slot).cuda(), kept, unused
    return p, st, rows


def host(t):
    return None if t is None else t.double().cpu().numpy()


def within(got, ref, bound, what):
    off = np.abs(host(got) - ref)
    assert (off <= bound + 1e-37).all(), (what, float((off - bound).max()), float((off / (np.abs(ref) + 1e-30)).max()))


@pytest.mark.parametrize("T,d,E,dtype", SHAPES)
@pytest.mark.parametrize("gamma", [True, False])
def test_norm_gate(env, T, d, E, dtype, gamma):
    torch, lm = env
    print(f"[norm_gate] T={T} d={d} E={E} {dtype} gamma={gamma}", flush=True)
    p, st, _ = case(torch, T, d, E, dtype, 1, "some", gamma)
    u = torch.finfo(st).eps / 2
    desc = lm.make_desc(T, d, E, 1, 8, 4, dtype)
    xn, rstd, g = torch.full_like(p["x"], 7.0), torch.full((T,), 7.0, device="cuda"), torch.full((T, E), 7.0, device="cuda")
    lm.locmoe_norm_gate(desc, p["x"], p["gi"], EPS, xn, rstd, g)
    ref, r, gr = blk.norm_gate(host(p["x"]), host(p["gi"]), EPS, E)
    within(rstd, r, R * r, "rstd")
    within(xn, ref, (u + 2 * R) * np.abs(ref), "xn")
    mean = np.abs(ref).reshape(T, E, -1).mean(2)
    within(g, gr, (2 * R + d // E * F) * mean, "g")
    # without g and rstd, in place, and with rstd alone: the same bits
    for rs in (None, torch.zeros_like(rstd)):
        y = p["x"].clone()
        lm.locmoe_norm_gate(desc, y, p["gi"], EPS, y, rs, None)
        assert torch.equal(y, xn) and (rs is None or torch.equal(rs, rstd))


@pytest.mark.parametrize("T,d,E,dtype", SHAPES)
@pytest.mark.parametrize("post,drop,gamma", [(True, "some", True), (False, "some", True), (True, "none", False), (True, "all", True)])
def test_combine_norm(env, T, d, E, dtype, post, drop, gamma):
    torch, lm = env
    print(f"[combine_norm] T={T} d={d} {dtype} post={post} drop={drop}", flush=True)
    p, st, rows = case(torch, T, d, E, dtype, 2, drop, gamma)
    u = torch.finfo(st).eps / 2
    desc = lm.make_desc(T, d, E, 1, 8, -(-rows // E), dtype)
    y, rstd = torch.full_like(p["x"], 7.0), torch.full((T,), 7.0, device="cuda")
    lm.locmoe_combine_norm(desc, p["out"], p["slot"], p["w"], p["x"], p["go"], post, EPS, SCALE, y, rstd)
    out = np.nan_to_num(host(p["out"]))
    ref, r = blk.combine_norm(out, host(p["slot"]).astype(int), host(p["w"]), host(p["x"]), host(p["go"]), post, EPS, SCALE)
    within(rstd, r, R * r, "rstd")
    res = host(p["x"])
    within(y, ref, u * np.abs(ref) + (2 * R + F) * (np.abs(ref - res) + np.abs(res)), "y")
    kept = torch.from_numpy(p["kept"]).cuda()
    assert torch.equal(y[~kept], p["x"][~kept])     # bit for bit
    z = p["x"].clone()
    lm.locmoe_combine_norm(desc, p["out"], p["slot"], p["w"], z, p["go"], post, EPS, SCALE, z, None)
    assert torch.equal(z, y)


@pytest.mark.parametrize("T,d,E,dtype", SHAPES)
@pytest.mark.parametrize("post,drop,gamma", [(True, "some", True), (False, "some", True), (True, "none", False), (True, "all", True)])
def test_combine_norm_bwd(env, T, d, E, dtype, post, drop, gamma):
    torch, lm = env
    print(f"[combine_norm_bwd] T={T} d={d} {dtype} post={post} drop={drop}", flush=True)
    p, st, rows = case(torch, T, d, E, dtype, 3, drop, gamma)
    u = torch.finfo(st).eps / 2
    desc = lm.make_desc(T, d, E, 1, 8, -(-rows // E), dtype)
    slot, out = host(p["slot"]).astype(int), np.nan_to_num(host(p["out"]))
    _, r = blk.combine_norm(out, slot, host(p["w"]), host(p["x"]), host(p["go"]), post, EPS, SCALE)
    rstd = torch.from_numpy(r.astype(np.float32)).cuda()
    r = host(rstd)
    dy = p["dy"].clone()
    dy[torch.from_numpy(~p["kept"]).cuda()] = float("nan")     # dropped tokens' rows are not read
    dout, dw, dg = torch.full_like(p["out"], 7.0), torch.full((T,), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda")
    n = lm.locmoe_norm_workspace_bytes(desc)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    call = lambda dgamma, w: lm.locmoe_combine_norm_bwd(desc, dy, p["out"], p["slot"], p["w"], p["go"], post, SCALE,  # noqa: E731
                                                        rstd if post else None, dout, dw, dgamma, w, n if w is not None else 0)
    call(dg, ws)
    ref, dwr, dgr = blk.combine_norm_backward(host(p["dy"]), out, slot, host(p["w"]), host(p["go"]), post, SCALE, r)
    assert (dout[torch.from_numpy(p["unused"]).cuda()] == 7.0).all()      # rows of no token stay as they are
    kept, at = p["kept"], slot[p["kept"]]
    go = np.ones(d) if p["go"] is None else host(p["go"])
    rk = r[kept][:, None] if post else 1.0
    nrm, uu = np.abs(out[at] * rk), np.abs(SCALE * go * host(p["dy"])[kept])
    wk = host(p["w"])[kept][:, None]
    sums = (uu * nrm).sum(1, keepdims=True)
    within(dw, dwr, np.zeros(T), "dw of dropped") if not kept.any() else None
    b = np.zeros(T)
    b[kept] = (2 * R + d * F) * sums[:, 0]
    within(dw, dwr, b, "dw")
    mag = rk * wk * (uu + (nrm * sums / d if post else 0.0))
    got = dout[torch.from_numpy(at).cuda()]
    within(got, ref[at], u * np.abs(ref[at]) + (2 * R + d * F) * mag, "dout")
    terms = (np.abs(SCALE * wk * host(p["dy"])[kept]) * nrm).sum(0)
    within(dg, dgr, (2 * R + T * F) * terms, "dgamma")
    first = [t.clone() for t in (dout, dw, dg)]
    call(dg, ws)
    assert all(torch.equal(a, c) for a, c in zip((dout, dw, dg), first))
    call(None, None)                    # without dgamma no workspace is asked for
    assert torch.equal(dout, first[0]) and torch.equal(dw, first[1])


@pytest.mark.parametrize("T,d,E,dtype", SHAPES)
@pytest.mark.parametrize("res,drop,gamma", [(True, "some", True), (False, "none", True), (True, "all", False)])
def test_dispatch_norm_bwd(env, T, d, E, dtype, res, drop, gamma):
    torch, lm = env
    print(f"[dispatch_norm_bwd] T={T} d={d} E={E} {dtype} res={res} drop={drop}", flush=True)
    p, st, rows = case(torch, T, d, E, dtype, 4, drop, gamma)
    u = torch.finfo(st).eps / 2
    desc = lm.make_desc(T, d, E, 1, 8, -(-rows // E), dtype)
    slot = host(p["slot"]).astype(int)
    _, r, _ = blk.norm_gate(host(p["x"]), None, EPS, E)
    rstd = torch.from_numpy(r.astype(np.float32)).cuda()
    r = host(rstd)
    dres = p["dy"] if res else None
    dx, dg = torch.full_like(p["x"], 7.0), torch.full((d,), 7.0, device="cuda")
    n = lm.locmoe_norm_workspace_bytes(desc)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    lm.locmoe_dispatch_norm_bwd(desc, p["dsend"], p["slot"], p["dg"], p["x"], p["gi"], rstd, dres, dx, dg, ws, n)
    dsend = np.nan_to_num(host(p["dsend"]))
    ref, dgr = blk.dispatch_norm_backward(dsend, slot, host(p["dg"]), host(p["x"]), host(p["gi"]), r, host(dres))
    gi = np.ones(d) if p["gi"] is None else np.abs(host(p["gi"]))
    dxn = np.repeat(np.abs(host(p["dg"])) * (E / d), d // E, axis=1)
    dxn[p["kept"]] += np.abs(dsend[slot[p["kept"]]])
    xh = np.abs(host(p["x"])) * r[:, None]
    sums = (dxn * gi * xh).sum(1, keepdims=True)
    mag = r[:, None] * (dxn * gi + xh * sums / d) + (np.abs(host(dres)) if res else 0.0)
    within(dx, ref, u * np.abs(ref) + (2 * R + d * F) * mag, "dx")
    within(dg, dgr, (2 * R + T * F) * (dxn * xh).sum(0), "dgamma")
    first = [dx.clone(), dg.clone()]
    if res:                             # in place over the residual's gradient
        z = dres.clone()
        lm.locmoe_dispatch_norm_bwd(desc, p["dsend"], p["slot"], p["dg"], p["x"], p["gi"], rstd, z, z, dg, ws, n)
        assert torch.equal(z, first[0]) and torch.equal(dg, first[1])
    z = p["x"].clone()                  # in place over x, without dgamma and workspace
    lm.locmoe_dispatch_norm_bwd(desc, p["dsend"], p["slot"], p["dg"], z, p["gi"], rstd, dres, z, None, None, 0)
    assert torch.equal(z, first[0])


def test_rows_of_zeros_infinities_and_nan(env):
    torch, lm = env
    T, d, E = 5, 256, 4
    desc = lm.make_desc(T, d, E, 1, 8, 4, "f32")
    x = torch.ones(T, d, device="cuda")
    x[0], x[1, 3], x[2, 3], x[3] = 0.0, float("inf"), float("nan"), 1e-30
    xn, rstd, g = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, E, device="cuda")
    lm.locmoe_norm_gate(desc, x, None, EPS, xn, rstd, g)
    assert (xn[0] == 0).all() and (g[0] == 0).all() and torch.isfinite(xn[3]).all()
    assert rstd[1] == 0 and torch.isnan(xn[1, 3]) and (xn[1, :3] == 0).all() and torch.isnan(xn[2]).all()
    assert torch.allclose(xn[4], torch.full((d,), (1.0 + EPS) ** -0.5, device="cuda"), rtol=1e-6)   # others untouched
    # an infinity in one token's output stays with that token
    slot, w, y = torch.tensor([1, 0, -1, 2, 3], dtype=torch.int32, device="cuda"), torch.ones(T, device="cuda"), torch.empty_like(x)
    out = torch.ones(E * 4, d, device="cuda")
    out[0, 7] = float("inf")
    res = torch.zeros_like(x)
    lm.locmoe_combine_norm(desc, out, slot, w, res, None, True, EPS, 1.0, y, None)
    assert torch.isnan(y[1, 7]) and (y[1, :7] == 0).all() and (y[2] == 0).all() and torch.isfinite(y[[0, 3, 4]]).all()


def test_offsets_past_32_bits(env):
    """Buffers of more than 2^32 bytes: rows on both sides of that boundary and the last one."""
    torch, lm = env
    T, d, E = 131072 + 300, 16384, 16
    sel = [0, 131071, 131072, 131200, T - 1]
    desc = lm.make_desc(T, d, E, 1, 8, -(-T // E), "bf16")
    gen = torch.Generator(device="cuda").manual_seed(5)
    big = lambda: torch.randn(T, d, dtype=torch.bfloat16, device="cuda", generator=gen)  # noqa: E731
    x, out, dy = big(), big(), big()
    gamma = torch.rand(d, device="cuda", generator=gen) + 0.5
    w, u = torch.rand(T, device="cuda", generator=gen), torch.finfo(torch.bfloat16).eps / 2
    slot = torch.arange(T, dtype=torch.int32, device="cuda").flip(0).contiguous()    # row T - 1 - m is token m's
    at = host(slot[sel]).astype(int)
    y, rstd, g = torch.full_like(x, 7.0), torch.empty(T, device="cuda"), torch.empty(T, E, device="cuda")
    lm.locmoe_norm_gate(desc, x, gamma, EPS, y, rstd, g)
    ref, r, gr = blk.norm_gate(host(x[sel]), host(gamma), EPS, E)
    within(y[sel], ref, (u + 2 * R) * np.abs(ref), "xn")
    within(g[sel], gr, (2 * R + d // E * F) * np.abs(ref).reshape(len(sel), E, -1).mean(2), "g")
    rstd2 = torch.empty(T, device="cuda")
    lm.locmoe_combine_norm(desc, out, slot, w, x, gamma, True, EPS, SCALE, y, rstd2)
    o, own = host(out[at]), np.arange(len(sel))
    ref, r2 = blk.combine_norm(o, own, host(w[sel]), host(x[sel]), host(gamma), True, EPS, SCALE)
    res = host(x[sel])
    within(y[sel], ref, u * np.abs(ref) + (2 * R + F) * (np.abs(ref - res) + np.abs(res)), "y")
    n = lm.locmoe_norm_workspace_bytes(desc)
    ws, dw, dgamma = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda"), torch.empty(d, device="cuda")
    lm.locmoe_combine_norm_bwd(desc, dy, out, slot, w, gamma, True, SCALE, rstd2, y, dw, dgamma, ws, n)     # y: dout
    r2 = host(rstd2[sel])
    ref, dwr, _ = blk.combine_norm_backward(host(dy[sel]), o, own, host(w[sel]), host(gamma), True, SCALE, r2)
    uu, nrm = np.abs(SCALE * host(gamma) * host(dy[sel])), np.abs(o) * r2[:, None]
    sums = (uu * nrm).sum(1, keepdims=True)
    within(dw[sel], dwr, (2 * R + d * F) * sums[:, 0], "dw")
    mag = r2[:, None] * host(w[sel])[:, None] * (uu + nrm * sums / d)
    within(y[at], ref, u * np.abs(ref) + (2 * R + d * F) * mag, "dout")
    dg = torch.randn(T, E, device="cuda", generator=gen)
    lm.locmoe_dispatch_norm_bwd(desc, out, slot, dg, x, gamma, rstd, dy, y, dgamma, ws, n)                  # y: dx
    r = host(rstd[sel])
    ref, _ = blk.dispatch_norm_backward(o, own, host(dg[sel]), res, host(gamma), r, host(dy[sel]))
    dxn = np.abs(o) + np.repeat(np.abs(host(dg[sel])) * (E / d), d // E, axis=1)
    xh = np.abs(res) * r[:, None]
    mag = r[:, None] * (dxn * host(gamma) + xh * (dxn * host(gamma) * xh).sum(1, keepdims=True) / d) + np.abs(host(dy[sel]))
    within(y[sel], ref, u * np.abs(ref) + (2 * R + d * F) * mag, "dx")
    want, size = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    for i in range(0, T, 8192):
        j = slice(i, min(T, i + 8192))
        t = (out[slot[j].long()].double() + dg[j].double().repeat_interleave(d // E, 1) * (E / d)) * x[j].double() * rstd[j, None].double()
        want += t.sum(0)
        size += t.abs().sum(0)
    within(dgamma, host(want), (2 * R + T * F) * host(size), "dgamma")
