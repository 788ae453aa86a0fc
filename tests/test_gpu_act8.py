"""Hidden activations kept in 8 bits.

Which values are kept: against z in float64.  f = 2^-24; z is a sum of d exact products in fp32, dz = d f sum |x W_in| off.  The
unit is max |z| / 127 in bf16, so at most 2^-8 of itself and the error of z / 127 off; a value read back is at most half a
unit and dz from z.
What the backward makes of them: with units that are powers of two a value q unit is a bf16 number, and the data gradients are
bit for bit those of locmoe_expert_ffn_dgrad with these numbers as Z.
"""
import numpy as np
import pytest

from oracle import block_oracle as blk
from oracle import locmoe_oracle as orc
from test_gpu_any_shape import KERNEL_SHAPES, rows_with_nan_tail, segments, storage

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2401_13920_amd import locmoe as lm
    assert torch.cuda.is_available(), "these tests need the MI355X"
    lm.lib()
    return torch, lm


def sizes(rows, E, h, torch):
    """Guarded outputs: rows behind the last segment's end hold a pattern that has to stay."""
    K = sum(rows)
    H = torch.full((K + 8, h), 3.0, dtype=torch.bfloat16, device="cuda")
    Zq = torch.full((K + 8, h), 55, dtype=torch.int8, device="cuda")
    Zs = torch.full((K + 8, -(-h // 16)), 3.0, dtype=torch.bfloat16, device="cuda")
    return K, H, Zq, Zs


def weights(torch, lm, desc, W_in, W_out, packed):
    if not packed:
        return W_in, W_out
    Wi, Wo = torch.empty_like(W_in), torch.empty_like(W_out)
    desc.w_packed = 0
    lm.locmoe_pack_weights(desc, W_in, W_out, Wi, Wo)
    desc.w_packed = 1
    return Wi, Wo


# (packed, E, d, h, T, C, rows, dtype): tails of rows and of 16-column blocks on both kinds of storage; the stream kernel of few
# rows; then every shape that the FFN's other kernels are tested with
SMALL = [(False, 4, 8, 8, 60, 40, [0, 1, 33, 16], "bf16"), (False, 4, 120, 264, 60, 40, [17, 0, 1, 32], "f32"),
         (False, 6, 264, 1000, 600, 100, [0, 1, 31, 32, 33, 97], "bf16"), (False, 6, 264, 520, 600, 100, [97, 0, 1, 31, 64, 33], "f32"),
         (True, 64, 1024, 4096, 192, 6, [0, 6, 1, 3] * 16, "bf16"), (True, 64, 1024, 4096, 700, 20, [17, 20, 0, 1] * 16, "bf16")]
SHAPES = SMALL + [(p, E, d, h, T, C, rows, "bf16") for p, _, _, E, d, h, T, C, rows in KERNEL_SHAPES if E > 4]


@pytest.mark.parametrize("packed,E,d,h,T,C,rows,dtype", SHAPES)
def test_forward(env, packed, E, d, h, T, C, rows, dtype):
    torch, lm = env
    print(f"[save8] packed={packed} E={E} d={d} h={h} T={T} C={C} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(d + h)
    off, seg, be = segments(torch, rows)
    K, H, Zq, Zs = sizes(rows, E, h, torch)
    d = d if d % E == 0 else d * E
    send = rows_with_nan_tail(torch, K, 8, d, storage(torch, dtype), gen)
    W_in = torch.randn(E, h, d, generator=gen, device="cuda").mul_(d ** -0.5).to(torch.bfloat16)
    W_out = torch.zeros(E, d, h, dtype=torch.bfloat16, device="cuda")
    desc = lm.make_desc(T, d, E, 1, h, C, dtype)
    Wi, _ = weights(torch, lm, desc, W_in, W_out, packed)
    lm.locmoe_expert_ffn_in_save8(desc, send, seg, be, Wi, H, Zq, Zs)
    plain = torch.empty_like(H)
    lm.locmoe_expert_ffn_in(desc, send, seg, be, Wi, plain)
    torch.cuda.synchronize()
    assert torch.equal(H[:K], plain[:K])
    assert (H[K:] == 3.0).all() and (Zq[K:] == 55).all() and (Zs[K:] == 3.0).all()
    pad = -h % 16
    for r in range(E):
        a, z = off[r], off[r + 1]
        if a == z or (r > 8 and E > 16 and r % 11):    # (all segments of a few experts, some of many)
            continue
        x = send[a:z].to(torch.bfloat16).double()       # (the FFN's operands are bf16)
        W = W_in[E - 1 - r].double()
        zr = x @ W.T
        dz = torch.nn.functional.pad(d * F * (x.abs() @ W.abs().T), (0, pad)).view(z - a, -1, 16)
        blocks = torch.nn.functional.pad(zr, (0, pad)).view(z - a, -1, 16)
        unit, q = Zs[a:z].double(), torch.nn.functional.pad(Zq[a:z].double(), (0, pad)).view(z - a, -1, 16)
        most, err = blocks.abs().amax(2), dz.amax(2)
        assert ((unit - most / 127).abs() <= 2.0 ** -8 * unit + err / 127 + 2 * F * unit).all()
        assert q.abs().max() <= 127 and (q.abs().amax(2)[unit > 0] >= 126).all()
        assert ((q * unit[:, :, None] - blocks).abs() <= unit[:, :, None] * (0.5 + 130 * F) + dz).all()


@pytest.mark.parametrize("packed,E,d,h,T,C,rows,dtype", SHAPES)
def test_backward(env, packed, E, d, h, T, C, rows, dtype):
    torch, lm = env
    print(f"[dgrad8] packed={packed} E={E} d={d} h={h} T={T} C={C} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(d + h)
    off, seg, be = segments(torch, rows)
    K, H, Zq, Zs = sizes(rows, E, h, torch)
    d = d if d % E == 0 else d * E
    st = storage(torch, dtype)
    dout = rows_with_nan_tail(torch, K, 8, d, st, gen)
    Zq[:K] = torch.randint(-127, 128, (K, h), generator=gen, device="cuda").to(torch.int8)
    Zs[:K] = torch.exp2(torch.randint(-9, -4, (K, Zs.shape[1]), generator=gen, device="cuda").float()).to(torch.bfloat16)
    value = Zq.double() * Zs.double().repeat_interleave(16, 1)[:, :h]
    Z = value.to(torch.bfloat16)
    assert torch.equal(Z.double(), value)               # 7 bits and a power of two
    W_out_t = torch.randn(E, h, d, generator=gen, device="cuda").mul_(d ** -0.5).to(torch.bfloat16)
    W_in_t = torch.randn(E, d, h, generator=gen, device="cuda").mul_(h ** -0.5).to(torch.bfloat16)
    desc = lm.make_desc(T, d, E, 1, h, C, dtype)
    Wo, Wi = weights(torch, lm, desc, W_out_t, W_in_t, packed)   # (W_out_t has the shape of W_in)
    ws = torch.zeros(lm.LOCMOE_FFN_WS_BYTES, dtype=torch.uint8, device="cuda")
    got = None
    for queues in (False, True):
        dZ, dsend = torch.full_like(H, 3.0), torch.full_like(dout, 3.0)
        if queues:
            lm.locmoe_expert_ffn_dgrad8_ws(desc, dout, Zq, Zs, seg, be, Wo, Wi, dZ, H, dsend, ws, lm.LOCMOE_FFN_WS_BYTES)
        else:
            lm.locmoe_expert_ffn_dgrad8(desc, dout, Zq, Zs, seg, be, Wo, Wi, dZ, H, dsend)
        torch.cuda.synchronize()
        assert (H[K:] == 3.0).all() and (dZ[K:] == 3.0).all() and (dsend[K:] == 3.0).all()
        assert got is None or (torch.equal(dZ, got[0]) and torch.equal(dsend, got[1]))
        got = dZ, dsend
    dZ_ref, dsend_ref = torch.full_like(H, 3.0), torch.full_like(dout, 3.0)
    lm.locmoe_expert_ffn_dgrad(desc, dout, Z, seg, be, Wo, Wi, dZ_ref, dsend_ref)
    assert torch.equal(got[0], dZ_ref) and torch.equal(got[1], dsend_ref)
    ref = value[:K] * torch.special.ndtr(value[:K])
    assert ((H[:K].double() - ref).abs() <= 2.0 ** -8 * ref.abs() * (1 + 2.0 ** -7) + 5e-5 * ref.abs() + 7e-6).all()


def test_zeros_infinities_and_nan(env):
    torch, lm = env
    E, d, h, K = 2, 16, 40, 6
    off, seg, be = segments(torch, [3, 3])
    W_in = torch.zeros(E, h, d, dtype=torch.bfloat16, device="cuda")
    W_in[:, :, 0] = torch.arange(h, device="cuda").to(torch.bfloat16) - 5.0   # z = x[0] (column - 5)
    send = torch.zeros(K, d, dtype=torch.bfloat16, device="cuda")
    send[:, 0] = torch.tensor([0.0, 1.0, float("inf"), float("nan"), 2.0 ** -126, 1e30], device="cuda").to(torch.bfloat16)
    desc = lm.make_desc(6, d, E, 1, h, 3)
    H, Zq, Zs = (torch.empty(K, n, dtype=t, device="cuda") for n, t in ((h, torch.bfloat16), (h, torch.int8), (3, torch.bfloat16)))
    lm.locmoe_expert_ffn_in_save8(desc, send, seg, be, W_in, H, Zq, Zs)
    back = Zq.float() * Zs.float().repeat_interleave(16, 1)[:, :h]
    z = torch.arange(h, device="cuda").float() - 5.0
    assert (back[0] == 0).all() and (Zs[0] == 0).all() and (Zq[0] == 0).all()
    assert ((back[1] - z).abs() <= 0.5 * Zs[1].float().repeat_interleave(16)[:h] * (1 + 1e-5)).all()
    assert torch.isnan(back[2]).all() and torch.isnan(back[3]).all()
    assert (back[4] == 0).all()                       # below 127 x 2^-126
    assert ((back[5] / 1e30 - z).abs() <= 0.02 * z.abs().max()).all()
    # ... and the backward of them is zero-filled, finite, or NaN in the rows concerned alone
    W_t = torch.ones(E, h, d, dtype=torch.bfloat16, device="cuda")
    dout, dZ, dsend = torch.ones_like(send), torch.empty_like(H), torch.empty_like(send)
    lm.locmoe_expert_ffn_dgrad8(desc, dout, Zq, Zs, seg, be, W_t, W_t.transpose(1, 2).contiguous(), dZ, H, dsend)
    assert torch.isfinite(dZ[[0, 1, 4, 5]]).all() and torch.isnan(dZ[[2, 3]]).all()
    assert torch.isfinite(dsend[[0, 1, 4, 5]]).all() and torch.isnan(dsend[[2, 3]]).all()
    assert (dZ[0] == 0.5 * d).all() and (H[0] == 0).all()                        # GeLU'(0) = 1/2


def test_oracle_blocks_are_the_kernels(env):
    """A row whose products are exact: q and the unit equal the oracle's."""
    torch, lm = env
    E, d, h = 1, 8, 56
    rng = np.random.default_rng(0)
    W = np.zeros((E, h, d), np.float32)
    W[0, :, 0] = rng.integers(-120, 121, h)
    x = np.zeros((5, d), np.float32)
    x[:, 0] = [1, 3, -0.125, 96, 2.0 ** 40]
    desc = lm.make_desc(5, d, E, 1, h, 5)
    off, seg, be = segments(torch, [5])
    dev = lambda a: torch.from_numpy(a).cuda().to(torch.bfloat16)  # noqa: E731
    H, Zq, Zs = (torch.empty(5, n, dtype=t, device="cuda") for n, t in ((h, torch.bfloat16), (h, torch.int8), (4, torch.bfloat16)))
    lm.locmoe_expert_ffn_in_save8(desc, dev(x), seg, be, dev(W), H, Zq, Zs)
    q, unit = blk.to8(x.astype(np.float64) @ W[0].T)
    assert np.array_equal(Zs.double().cpu().numpy(), unit) and np.array_equal(Zq.cpu().numpy(), q)
    assert np.allclose(H.double().cpu().numpy(), orc.gelu(x.astype(np.float64) @ W[0].T), rtol=2.0 ** -7, atol=1e-5)
