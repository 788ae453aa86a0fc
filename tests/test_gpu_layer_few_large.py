"""The layer for a few tokens on weights that are loaded past the caches (more than 100 MiB in a launch), packed and in rows; with
starts of K that differ from tile to tile; and weights that lie more than 2^32 bytes from the first.

Every sum is exact: x in {0 .. 3}, W_in in {0, 1}, W_out in {-1, 0, 1}, so z is a whole number, far above 8, where GeLU(z) is z in
fp32; H = z in bf16 is rounded as the oracle rounds it, and the sums of W_out H stay below 2^24.  A product that is left out, taken twice or
from another place changes a whole number.  What is left: the score, (E + 8) f off as in tests/test_gpu_layer_few.py, its product
and the rounding to storage: (E + 10) f + u relative.
"""
import pytest

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2401_13920_amd import locmoe as lm
    assert torch.cuda.is_available(), "these tests need the MI355X"
    lm.lib()
    return torch, lm


def start_offsets(torch, T, E, groups, N, K, packed, bf16):
    """(past the caches, starts differ) of a GEMM, by the rules of csrc/few.hip."""
    cus, groups_most = torch.cuda.get_device_properties(0).multi_processor_count, min(T, E)
    assert groups_most * N >= 16 * cus                    # (tiles of 16 rows)
    past = groups_most * N * K * 2 > 100 << 20 and (packed or K % 64 == 0)
    waves = 8 * min(2 * cus, groups_most * -(-N // 16))
    steps = -(-K // 32)
    cost = [-(-(groups * -(-N // 16) << i) // waves) * (((steps - 1) >> i) + 5) for i in range(4)]
    parts = 1 << cost.index(min(cost))
    lines = past and not packed
    units = steps // 2 if lines else steps
    turns = units // parts // ((8 if bf16 else 4) // (2 if lines else 1))
    return past, turns >= (16 if packed else 8) and past


# (experts, their tokens, d, h, starts of K that differ in the two GEMMs: packed / in rows)
ONE_EACH, UNEVEN = [1] * 16, [33, 17] + [1] * 14
CASES = [(4, [1, 1, 1, 1], 4096, 4096, (0, 0), (0, 0)),
         (4, [7, 0, 1, 5], 4352, 4608, (0, 0), (0, 0)),
         (4, [33, 5, 1, 1], 4096, 4096, (0, 0), (0, 0)),
         (16, ONE_EACH, 4096, 4096, (1, 1), (1, 1)),
         (16, UNEVEN, 4096, 4096, (1, 1), (1, 1)),
         (64, [1] + [0] * 32 + [1] + [0] * 29 + [1], 4096, 16384, (0, 1), (0, 1))]
FORMS = [("bf16", True), ("bf16", False), ("f32", False)]


@pytest.mark.parametrize("E,sizes,d,h,packed_starts,row_starts", CASES)
@pytest.mark.parametrize("dtype,packed", FORMS)
@pytest.mark.parametrize("weighted,most", [(True, 64), (False, 3)])
def test_exact_sums(env, E, sizes, d, h, packed_starts, row_starts, dtype, packed, weighted, most):
    torch, lm = env
    T, bf16 = sum(sizes), dtype == "bf16"
    print(f"[few large] T={T} d={d} E={E} h={h} {dtype} packed={packed} weighted={weighted}", flush=True)
    groups = sum(n > 0 for n in sizes)
    got = [start_offsets(torch, T, E, groups, N, K, packed, bf16) for N, K in ((h, d), (d, h))]
    assert all(past for past, _ in got)
    if bf16:        # (fp32 storage takes half as many steps at a time: more turns)
        assert tuple(int(differ) for _, differ in got) == (packed_starts if packed else row_starts)
    gen = torch.Generator(device="cuda").manual_seed(d + h + T)
    owner = torch.tensor([e for e in range(E) for _ in range(sizes[e])], device="cuda")
    owner = owner[torch.randperm(T, generator=gen, device="cuda")]
    st = torch.bfloat16 if bf16 else torch.float32
    x = torch.randint(0, 4, (T, d), generator=gen, device="cuda").to(st)
    W_in, W_out = (torch.zeros(E, *s, dtype=torch.bfloat16, device="cuda") for s in ((h, d), (d, h)))
    for e in range(E):
        if sizes[e]:
            W_in[e] = (torch.rand(h, d, generator=gen, device="cuda") < 128.0 / d).to(torch.bfloat16)
            W_out[e] = torch.randint(-1, 2, (d, h), generator=gen, device="cuda").to(torch.bfloat16)
    desc = lm.make_desc(T, d, E, 1, h, most, dtype, relu=False)
    Wi, Wo = W_in, W_out
    if packed:
        Wi, Wo = torch.empty_like(W_in), torch.empty_like(W_out)
        lm.locmoe_pack_weights(desc, W_in, W_out, Wi, Wo)
        desc.w_packed = 1
    g = torch.rand(T, E, generator=gen, device="cuda")
    g[torch.arange(T, device="cuda"), owner] += 1.0
    i32 = dict(dtype=torch.int32, device="cuda")
    eid, slot, w, y = torch.full((T,), 99, **i32), torch.full((T,), 99, **i32), torch.full((T,), 7.0, device="cuda"), torch.full((T, d), 7.0, dtype=st, device="cuda")
    n = lm.locmoe_layer_few_workspace_bytes(desc)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    lm.locmoe_layer_few(desc, x, g, None, Wi, Wo, weighted, eid, w, slot, y, ws, n)
    assert torch.equal(eid.long(), owner)
    own = owner.tolist()
    kept = [m for m in range(T) if own[:m].count(own[m]) < most]
    assert slot.tolist() == [m if m in set(kept) else -1 for m in range(T)]
    score = torch.softmax(g.double(), 1)[torch.arange(T, device="cuda"), owner]
    assert ((w.double() - score).abs() <= (E + 8) * F * score).all()
    rest = [m for m in range(T) if m not in set(kept)]
    assert (y[rest] == (0.0 if weighted else 7.0)).all()
    u = torch.finfo(st).eps / 2
    for e in sorted(set(own)):
        at = torch.tensor([m for m in kept if own[m] == e], device="cuda")
        z = x[at].double() @ W_in[e].double().T
        assert z.min() >= 16 and z.max() < 512
        out = (z.to(torch.bfloat16).double() if bf16 else z) @ W_out[e].double().T
        ref = out * (score[at, None] if weighted else 1.0)
        b = (u + ((E + 10) * F if weighted else 0.0)) * ref.abs()
        off = (y[at].double() - ref).abs()
        assert (off <= b * (1 + 2.0 ** -7)).all(), (e, float((off - b).max()))
