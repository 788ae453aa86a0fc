"""More rows than a launch of the forward norms takes (2^32 threads): the whole input in one call against
parts of it, bit for bit, and rows on both sides of a launch's end against float64 (the bounds of tests/test_gpu_norms.py)."""
import numpy as np
import pytest

from oracle import block_oracle as blk
from test_gpu_norms import EPS, F, R, SCALE, env, host, within  # noqa: F401

pytestmark = pytest.mark.gpu


# 16 lanes and one chunk a row (2^27 rows a launch): past 2^32 threads; a wave and two chunks, four and one gating value (2^25 rows)
@pytest.mark.parametrize("T,d,E", [(2 ** 28 + 37, 8, 1), (2 ** 25 + 5, 520, 5)])
def test_rows_of_more_than_one_launch(env, T, d, E):
    torch, lm = env
    print(f"[norms long] T={T} d={d} E={E}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    out = torch.empty(1000, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    gamma = torch.rand(d, device="cuda", generator=gen) + 0.5
    w = torch.rand(T, device="cuda", generator=gen)
    slot = torch.arange(T, dtype=torch.int32, device="cuda") % 1003 - 3          # (three of 1 003 tokens dropped)
    xn, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    f32 = dict(dtype=torch.float32, device="cuda")
    rstd, g, rstd2 = torch.full((T,), 7.0, **f32), torch.full((T, E), 7.0, **f32), torch.full((T,), 7.0, **f32)

    def both(a, z, xn, rstd, g, y, rstd2):
        desc = lm.make_desc(z - a, d, E, 1, 8, -(-1000 // E))
        lm.locmoe_norm_gate(desc, x[a:z], gamma, EPS, xn, rstd, g)
        lm.locmoe_combine_norm(desc, out, slot[a:z], w[a:z], x[a:z], gamma, True, EPS, SCALE, y, rstd2)

    both(0, T, xn, rstd, g, y, rstd2)
    cut = (10 ** 8 + 4) // 16 * 16 if d == 8 else 10 ** 7 // 16 * 16      # (rows that begin at 16 bytes in every buffer)
    for a in range(0, T, cut):
        z = min(T, a + cut)
        part = [torch.empty_like(t[a:z]) for t in (xn, rstd, g, y, rstd2)]
        both(a, z, *part)
        assert all(torch.equal(t[a:z], p) for t, p in zip((xn, rstd, g, y, rstd2), part)), a
    sel = sorted({0, 5, cut, T - 1, *(k + o for k in (2 ** 25, 2 ** 27, 2 ** 28) if k < T for o in (-1, 0, 1))})
    u = torch.finfo(torch.bfloat16).eps / 2
    ref, r, gr = blk.norm_gate(host(x[sel]), host(gamma), EPS, E)
    within(xn[sel], ref, (u + 2 * R) * np.abs(ref), "xn")
    within(rstd[sel], r, R * r, "rstd")
    within(g[sel], gr, (2 * R + d // E * F) * np.abs(ref).reshape(len(sel), E, -1).mean(2), "g")
    ref, r = blk.combine_norm(host(out), host(slot[sel]).astype(int), host(w[sel]), host(x[sel]), host(gamma), True, EPS, SCALE)
    res = host(x[sel])
    within(y[sel], ref, u * np.abs(ref) + (2 * R + F) * (np.abs(ref - res) + np.abs(res)), "y")
    within(rstd2[sel], r, R * r, "rstd2")
