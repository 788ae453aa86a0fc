"""H that the 8-bit data gradients form again, for pre-activations of every size.

GeLU of a bf16 output: 5e-5 relative or 7e-6 absolute by the polynomial, and half a step of bf16 (tests/test_gpu_act8.py has the
same bound on values of ordinary size).
"""
import pytest

from test_gpu_act8 import sizes, weights
from test_gpu_any_shape import segments

pytestmark = pytest.mark.gpu


# the tiles of ffn_any, row-major and packed, the stream of few rows, the 256-column tiles
@pytest.mark.parametrize("packed,E,d,h,T,C,rows", [(False, 4, 64, 1040, 60, 40, [17, 0, 1, 32]), (True, 4, 256, 1024, 60, 40, [17, 0, 1, 32]),
                                                   (True, 64, 1024, 4096, 192, 6, [0, 6, 1, 3] * 16),
                                                   (True, 8, 1024, 4096, 2048, 300, [256, 0, 300, 17] * 2)])
def test_h_of_far_values(packed, E, d, h, T, C, rows):
    import torch
    from paper_2401_13920_amd import locmoe as lm
    print(f"[dgrad8 far] packed={packed} E={E} d={d} h={h} T={T} C={C}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(d + h)
    _, seg, be = segments(torch, rows)
    K, H, Zq, Zs = sizes(rows, E, h, torch)
    Zq[:K] = torch.randint(-127, 128, (K, h), generator=gen, device="cuda").to(torch.int8)
    Zs[:K] = torch.exp2(torch.randint(-12, 118, (K, Zs.shape[1]), generator=gen, device="cuda").float()).to(torch.bfloat16)
    Zs[0, 1] = float("nan")
    z = Zq[:K].double() * Zs[:K].double().repeat_interleave(16, 1)[:, :h]
    desc = lm.make_desc(T, d, E, 1, h, C)
    W = torch.zeros(E, h, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(E, d, h, dtype=torch.bfloat16, device="cuda")
    Wo, Wi = weights(torch, lm, desc, *W, packed)
    dout = torch.zeros(K + 8, d, dtype=torch.bfloat16, device="cuda")
    lm.locmoe_expert_ffn_dgrad8(desc, dout, Zq, Zs, seg, be, Wo, Wi, torch.empty_like(H), H, torch.empty_like(dout))
    assert torch.isnan(H[0, 16:32]).all()
    ref = z * torch.special.ndtr(z)
    ok = (H[:K].double() - ref).abs() <= 2.0 ** -8 * ref.abs() * (1 + 2.0 ** -7) + 5e-5 * ref.abs() + 7e-6
    assert (ok | torch.isnan(z)).all()
