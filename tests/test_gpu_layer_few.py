"""The layer for a few tokens against the oracle in float64.

Tolerances, element by element.  f = 2^-24, u half a step of bf16 (2^-8).  z is a sum of d exact products in fp32:
dz = d f sum |x W_in|.  |GeLU'| < 1.13.  bf16 storage: H = GeLU(z) by a polynomial (5e-5 relative or 7e-6 absolute) and
rounded, so dH = 1.13 dz + 5e-5 |H| + 7e-6 + u |H|;  fp32 storage: dH = 1.13 dz + 8 f |z| (erfc, two products, three parts).
y = w out: the error of out is sum |W_out| dH + h f sum |W_out H|, the score's is (E + 8) f w, then a rounding to storage.
"""
import numpy as np
import pytest

from oracle import block_oracle as blk
from oracle import locmoe_oracle as orc
from paper_2401_13920_amd import workloads as wl

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2401_13920_amd import locmoe as lm
    assert torch.cuda.is_available(), "these tests need the MI355X"
    lm.lib()
    return torch, lm


class Layer:
    def __init__(self, env, T, d, E, h, C, dtype="bf16", packed=False, relu=True, seed=0, experts=None):
        self.torch, self.lm = torch, lm = env
        self.T, self.d, self.E, self.h, self.C, self.dtype, self.relu = T, d, E, h, C, dtype, relu
        rng = np.random.default_rng(seed + 1000 * T + d)
        self.rng = rng
        self.x = wl.round_to_storage(rng.standard_normal((T, d)).astype(np.float32), dtype)
        if experts is not None:           # token m leans to expert experts[m % len]
            b = d // E
            for m in range(T):
                e = experts[m % len(experts)]
                self.x[m, e * b:(e + 1) * b] += 4.0
            self.x = wl.round_to_storage(self.x, dtype)
        bf = lambda a: wl.round_to_storage(a.astype(np.float32), "bf16")  # noqa: E731
        self.W = [(bf(rng.standard_normal((h, d)) * d ** -0.5), bf(rng.standard_normal((d, h)) * h ** -0.5)) for _ in range(E)]
        self.desc = lm.make_desc(T, d, E, 1, h, C, dtype, relu)
        st = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.xd = torch.from_numpy(self.x).cuda().to(st)
        W_in = torch.from_numpy(np.stack([w[0] for w in self.W])).cuda().to(torch.bfloat16)
        W_out = torch.from_numpy(np.stack([w[1] for w in self.W])).cuda().to(torch.bfloat16)
        if packed:
            Wi, Wo = torch.empty_like(W_in), torch.empty_like(W_out)
            lm.locmoe_pack_weights(self.desc, W_in, W_out, Wi, Wo)
            W_in, W_out, self.desc.w_packed = Wi, Wo, 1
        self.W_in, self.W_out = W_in, W_out
        i32 = dict(dtype=torch.int32, device="cuda")
        self.eid, self.slot, self.w = torch.full((T,), 99, **i32), torch.full((T,), 99, **i32), torch.full((T,), 7.0, device="cuda")
        self.y = torch.full((T, d), 7.0, device="cuda").to(st)
        self.n = lm.locmoe_layer_few_workspace_bytes(self.desc)
        self.ws = torch.full((self.n,), 255, dtype=torch.uint8, device="cuda")   # nothing in it has to be set

    def call(self, g=None, eps=None, weighted=True, stream=None):
        self.lm.locmoe_layer_few(self.desc, self.xd, g, eps, self.W_in, self.W_out, weighted, self.eid, self.w, self.slot,
                                 self.y, self.ws, self.n, stream)

    def check(self, g32, eps=None, weighted=True):
        eid, w, slot, out = blk.layer_few(self.x, g32, eps, self.relu, self.C, lambda e: self.W[e])
        host = lambda t: t.double().cpu().numpy()  # noqa: E731
        assert np.array_equal(host(self.eid), eid) and np.array_equal(host(self.slot), slot)
        assert (np.abs(host(self.w) - w) <= (self.E + 8) * F * w).all()
        u = (2.0 ** -8 if self.dtype == "bf16" else F)
        got = host(self.y)
        for m in range(self.T):
            if slot[m] < 0:
                assert (got[m] == (0.0 if weighted else 7.0)).all()
                continue
            Wi, Wo = (v.astype(np.float64) for v in self.W[eid[m]])
            x = self.x[m].astype(np.float64)
            z = Wi @ x
            H = orc.gelu(z)
            dH = 1.13 * self.d * F * (np.abs(Wi) @ np.abs(x))
            dH = dH + (5e-5 * np.abs(H) + 7e-6 + 2.0 ** -8 * np.abs(H) if self.dtype == "bf16" else 8 * F * np.abs(z))
            f = w[m] if weighted else 1.0
            ref = f * out[m]
            b = f * (np.abs(Wo) @ (dH + self.h * F * np.abs(H))) * (1 + 2.0 ** -7) + (self.E + 10) * F * np.abs(ref) + u * np.abs(ref)
            off = np.abs(got[m] - ref)
            assert (off <= b).all(), (m, float((off / b).max()))


# lengths around the MFMA's 16 columns and the wave's 64 lanes, inner sizes that end inside an MFMA step or a 16-row tile,
# more experts than tokens and than lanes, one expert
SHAPES = [(1, 8, 1, 8, 1), (1, 8, 8, 8, 1), (2, 24, 6, 40, 2), (3, 48, 3, 40, 1), (15, 128, 8, 256, 15), (16, 120, 15, 264, 3),
          (17, 136, 4, 72, 17), (33, 256, 128, 512, 33), (49, 600, 50, 96, 7), (64, 1024, 1, 520, 64), (64, 1024, 1024, 64, 64),
          (64, 80, 10, 3200, 2), (5, 1600, 40, 640, 5), (31, 2056, 257, 24, 31)]


@pytest.mark.parametrize("T,d,E,h,C", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer(env, T, d, E, h, C, dtype):
    torch, lm = env
    print(f"[few] T={T} d={d} E={E} h={h} C={C} {dtype}", flush=True)
    L = Layer(env, T, d, E, h, C, dtype)
    L.call()
    g32 = torch.empty(T, E, device="cuda")
    lm.locmoe_gate(L.desc, L.xd, g32)
    assert (L.x.reshape(T, E, -1).astype(np.float64).mean(2) - g32.double().cpu().numpy()).__abs__().max() < 1e-5
    L.check(g32.cpu().numpy())
    first = [t.clone() for t in (L.y, L.eid, L.w, L.slot)]
    L.ws.fill_(3)
    L.call()
    assert all(torch.equal(a, b) for a, b in zip(first, (L.y, L.eid, L.w, L.slot)))


@pytest.mark.parametrize("T,d,E,h,C", [(1, 256, 8, 512, 1), (16, 512, 16, 256, 2), (20, 256, 4, 768, 20), (64, 1024, 64, 256, 64)])
@pytest.mark.parametrize("experts", [None, [2], [1, 3, 1, 1]])
def test_packed_weights(env, T, d, E, h, C, experts):
    torch, lm = env
    print(f"[few packed] T={T} d={d} E={E} h={h} C={C} experts={experts}", flush=True)
    g32 = torch.empty(T, E, device="cuda")
    ref = None
    for packed in (False, True):
        L = Layer(env, T, d, E, h, C, packed=packed, experts=experts)
        lm.locmoe_gate(L.desc, L.xd, g32)
        L.call()
        L.check(g32.cpu().numpy())
        assert ref is None or torch.equal(L.y, ref)   # the same products in the same order
        ref = L.y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 7, 40])
def test_given_gating_values_bias_and_no_relu(env, T, dtype):
    torch, lm = env
    print(f"[few given] T={T} {dtype}", flush=True)
    for relu in (True, False):
        L = Layer(env, T, 96, 12, 56, max(1, T // 3), dtype, relu=relu)
        g = L.rng.standard_normal((T, 12)).astype(np.float32) - 1.0
        eps = L.rng.standard_normal(12).astype(np.float32)
        L.call(torch.from_numpy(g).cuda(), torch.from_numpy(eps).cuda(), weighted=False)
        L.check(g, eps, weighted=False)


def test_ties_go_to_the_lowest_expert(env):
    torch, lm = env
    for E in (8, 96, 512):
        L = Layer(env, 6, 1024 if E == 512 else 96 * 8, E, 16, 6)
        g = np.zeros((6, E), np.float32)
        g[0] = -3.0                    # nothing above zero: expert 0, score 1 / E
        g[1, [E - 1, 5]] = 2.0
        g[2, E // 2:] = 1.0
        g[3, [7, 3]] = 0.25
        g[4, E - 1] = 1e30
        L.call(torch.from_numpy(g).cuda())
        L.check(g)
        assert L.eid.tolist()[:5] == [0, 5, E // 2, 3, E - 1]


@pytest.mark.parametrize("E", [4, 12, 96, 512])
def test_masked_experts(env, E):
    """Experts of gating value minus infinity: never taken, nothing in the score; so are the type's lowest values."""
    torch, lm = env
    d = 1024 if E == 512 else 96 * 8
    for T in (1, 6, 64):
        for low in (-np.inf, float(np.finfo(np.float32).min)):
            print(f"[few masked] E={E} T={T} low={low}", flush=True)
            L = Layer(env, T, d, E, 16, T, relu=False)
            g = L.rng.standard_normal((T, E)).astype(np.float32)
            eps = np.zeros(E, np.float32)
            eps[::2] = low                       # the first expert of most lanes, and all of some
            g[:, E // 2:E - 1] = low
            with np.errstate(over="ignore"):
                L.call(torch.from_numpy(g).cuda(), torch.from_numpy(eps).cuda())
                L.check(g, eps)
            assert (L.eid % 2 == 1).all() and torch.isfinite(L.w).all()


@pytest.mark.parametrize("E", [1, 4, 96])
def test_token_without_experts(env, E):
    """Every expert masked: expert 0 and a score of NaN, which stay with that token."""
    torch, lm = env
    for T in (1, 5, 40):
        print(f"[few none] E={E} T={T}", flush=True)
        L = Layer(env, T, 96, E, 16, T, relu=False)
        g = L.rng.standard_normal((T, E)).astype(np.float32)
        L.call(torch.from_numpy(g).cuda())
        eid, y = L.eid.clone(), L.y.clone()
        g[T // 2] = -np.inf
        L.call(torch.from_numpy(g).cuda())
        others = [m for m in range(T) if m != T // 2]
        assert L.eid[T // 2] == 0 and torch.isnan(L.w[T // 2]) and torch.isnan(L.y[T // 2]).all()
        assert torch.equal(L.eid[others], eid[others]) and torch.isfinite(L.y[others]).all()
        if E == 1:     # (elsewhere another group's size may change how a GEMM is cut)
            assert torch.equal(L.y[others], y[others])


def test_all_tokens_alike(env):
    """The same token 64 times: one group of 64, of which the capacity keeps the first ones."""
    torch, lm = env
    for C in (1, 16, 17, 64):
        L = Layer(env, 64, 256, 8, 256, C, experts=[5])
        L.x[:] = L.x[0]
        L.xd[:] = L.xd[0].clone()
        g32 = torch.empty(64, 8, device="cuda")
        lm.locmoe_gate(L.desc, L.xd, g32)
        L.call()
        L.check(g32.cpu().numpy())
        assert all(torch.equal(L.y[0], L.y[m]) for m in range(C)) and (L.slot[:C] >= 0).all() and (L.slot[C:] == -1).all()


def test_y_over_x(env):
    torch, lm = env
    for dtype in ("bf16", "f32"):
        L = Layer(env, 9, 64, 4, 64, 2, dtype)
        L.call()
        want, L.y = L.y, L.xd
        L.call()
        assert torch.equal(L.y, want)


def test_many_tiles(env):
    """More tiles than waves: every wave takes several, each with all of K."""
    torch, lm = env
    for T, experts in ((12, list(range(12))), (60, [0, 0, 0, 0, 1, 2, 3])):
        L = Layer(env, T, 384, 12, 10920, T, experts=experts)
        g32 = torch.empty(T, 12, device="cuda")
        lm.locmoe_gate(L.desc, L.xd, g32)
        L.call()
        L.check(g32.cpu().numpy())


def test_infinities_stay_with_their_token(env):
    torch, lm = env
    for dtype in ("bf16", "f32"):
        L = Layer(env, 3, 64, 4, 32, 3, dtype)
        g = np.zeros((3, 4), np.float32)
        g[:, 1] = 1.0
        gd = torch.from_numpy(g).cuda()
        L.call(gd)
        want = L.y.clone()
        L.xd[1, 5] = float("inf")
        L.call(gd)
        assert torch.equal(L.y[[0, 2]], want[[0, 2]]) and not torch.isfinite(L.y[1]).all()
        L.xd[1, 5] = float("nan")
        L.call(gd)
        assert torch.equal(L.y[[0, 2]], want[[0, 2]]) and torch.isnan(L.y[1]).all()


# fewer tiles of 16 rows of weights than compute units: tiles of 8 and of 4 rows, with K in two and four parts side by side
@pytest.mark.parametrize("T", [1, 2, 4, 5, 8, 9])
@pytest.mark.parametrize("d,h", [(512, 768), (256, 64), (384, 200), (64, 1024)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_narrow_tiles(env, T, d, h, dtype):
    torch, lm = env
    print(f"[few narrow] T={T} d={d} h={h} {dtype}", flush=True)
    for experts in (None, [3], [0, 2, 1]):
        for packed in (False, True):
            if packed and (dtype == "f32" or d % 256 or h % 256):
                continue
            L = Layer(env, T, d, 4, h, max(1, T - 1), dtype, packed=packed, experts=experts)
            g32 = torch.empty(T, 4, device="cuda")
            lm.locmoe_gate(L.desc, L.xd, g32)
            L.call()
            L.check(g32.cpu().numpy())


# more than 100 MiB of row-major weights in a launch: rows of whole 128-byte lines go past the caches (2048: 32 of them, 6592: 103);
# 6600 values are no whole lines, and end inside a tile of rows.  Groups of one to four column tiles.
@pytest.mark.parametrize("T,h,dtype,experts", [(5, 6600, "bf16", [0, 1, 2, 3]), (13, 6592, "bf16", [0, 1, 2, 3]),
                                               (13, 6592, "f32", [3, 2, 1, 0, 0]), (26, 6592, "bf16", [0] * 20 + [1, 2, 3]),
                                               (40, 6592, "f32", [0] * 37 + [1, 2, 3]), (40, 6592, "bf16", [0] * 37 + [1, 2, 3])])
def test_many_weights_row_major(env, T, h, dtype, experts):
    torch, lm = env
    print(f"[few rows] T={T} h={h} {dtype}", flush=True)
    L = Layer(env, T, 2048, 4, h, T, dtype, experts=experts)
    g = np.full((T, 4), -1.0, np.float32)
    g[np.arange(T), [experts[m % len(experts)] for m in range(T)]] = 1.0
    L.call(torch.from_numpy(g).cuda())
    L.check(g)
    assert sorted(set(L.eid.tolist())) == [0, 1, 2, 3]
