"""Refusals of the block's entry points (norms, the layer for a few tokens, activations in 8 bits) without a GPU: every
argument error is caught before a launch, so the addresses below are never touched."""
import pytest

from paper_2401_13920_amd import locmoe as lm

P = 0x1000
OK, NULL, SHAPE, ARG, WS = 0, lm.LOCMOE_ERR_NULL, lm.LOCMOE_ERR_SHAPE, lm.LOCMOE_ERR_ARG, lm.LOCMOE_ERR_WORKSPACE
NAN, INF = float("nan"), float("inf")


def desc(**kw):
    return lm.make_desc(**{**dict(T=16, d=64, E=8, N=2, h=32, Cap=4), **kw})


def status(fn, *a):
    try:
        fn(*a)
    except lm.LocMoEError as e:
        return e.status
    return OK


def refused(fn, good, places, dsc=None):
    """Every argument in `places` (index -> (bad value, status)) is refused by itself."""
    for i, (bad, want) in places.items():
        a = list(good)
        a[i] = bad
        assert status(fn, dsc or desc(), *a, 0) == want, (fn.__name__, i, bad)


def test_norm_gate():
    good = [P, P, 1e-5, P, P, P]
    refused(lm.locmoe_norm_gate, good, {0: (None, NULL), 3: (None, NULL)})
    for eps in (0.0, -1e-5, NAN, INF):
        refused(lm.locmoe_norm_gate, good, {2: (eps, ARG)})
    for bad in (dict(d=60), dict(T=0), dict(E=0)):
        refused(lm.locmoe_norm_gate, good, {0: (P, SHAPE)}, desc(**bad))
    refused(lm.locmoe_norm_gate, good, {0: (P, ARG)}, desc(Cap=0))


def test_combine_norm():
    good = [P, P, P, P, P, True, 1e-5, 1.0, P, P]
    refused(lm.locmoe_combine_norm, good, {i: (None, NULL) for i in (0, 1, 2, 3, 8)})
    refused(lm.locmoe_combine_norm, good, {5: (2, ARG), 6: (0.0, ARG), 7: (INF, ARG)})
    refused(lm.locmoe_combine_norm, good, {6: (NAN, ARG), 7: (NAN, ARG)})
    refused(lm.locmoe_combine_norm, good, {0: (P, SHAPE)}, desc(h=12))


def test_combine_norm_bwd():
    n = lm.locmoe_norm_workspace_bytes(desc())
    good = [P, P, P, P, P, True, 1.0, P, P, P, P, P, n]
    refused(lm.locmoe_combine_norm_bwd, good, {i: (None, NULL) for i in (0, 1, 2, 3, 7, 8, 9)})
    refused(lm.locmoe_combine_norm_bwd, good, {5: (-1, ARG), 6: (NAN, ARG), 11: (None, WS), 12: (n - 1, WS)})
    refused(lm.locmoe_combine_norm_bwd, good, {0: (P, SHAPE)}, desc(d=68))


def test_dispatch_norm_bwd():
    n = lm.locmoe_norm_workspace_bytes(desc())
    good = [P, P, P, P, P, P, P, P, P, P, n]
    refused(lm.locmoe_dispatch_norm_bwd, good, {i: (None, NULL) for i in (0, 1, 2, 3, 5, 7)})
    refused(lm.locmoe_dispatch_norm_bwd, good, {9: (None, WS), 10: (n - 1, WS)})
    refused(lm.locmoe_dispatch_norm_bwd, good, {0: (P, SHAPE)}, desc(N=9))


def test_rows_of_at_most_64_kib():
    assert lm.locmoe_norm_workspace_bytes(desc(d=32768)) > 0
    assert lm.locmoe_norm_workspace_bytes(desc(d=16384, dtype="f32")) > 0
    for long in (desc(d=32768 + 64), desc(d=16384 + 64, dtype="f32")):
        assert lm.locmoe_norm_workspace_bytes(long) == 0
        assert status(lm.locmoe_norm_gate, long, P, P, 1e-5, P, P, P, 0) == SHAPE
        assert status(lm.locmoe_combine_norm, long, P, P, P, P, P, True, 1e-5, 1.0, P, P, 0) == SHAPE
        assert status(lm.locmoe_combine_norm_bwd, long, P, P, P, P, P, True, 1.0, P, P, P, P, P, 1 << 40, 0) == SHAPE
        assert status(lm.locmoe_dispatch_norm_bwd, long, P, P, P, P, P, P, P, P, P, P, 1 << 40, 0) == SHAPE


def test_layer_few():
    n = lm.locmoe_layer_few_workspace_bytes(desc())
    assert n >= 16 * 32 * 2
    assert lm.locmoe_layer_few_workspace_bytes(desc(dtype="f32")) >= 3 * 16 * 32 * 2
    good = [P, P, P, P, P, True, P, P, P, P, P, n]
    refused(lm.locmoe_layer_few, good, {i: (None, NULL) for i in (0, 3, 4, 6, 7, 8, 9)})
    refused(lm.locmoe_layer_few, good, {5: (2, ARG), 10: (None, WS), 11: (n - 1, WS)})
    for T, want in ((64, True), (65, False)):
        assert (lm.locmoe_layer_few_workspace_bytes(desc(T=T)) > 0) == want
    refused(lm.locmoe_layer_few, good, {0: (P, SHAPE)}, desc(T=65))
    refused(lm.locmoe_layer_few, good, {0: (P, SHAPE)}, desc(d=60))
    refused(lm.locmoe_layer_few, good, {0: (P, ARG)}, desc(w_packed=True))                          # no such layout
    refused(lm.locmoe_layer_few, good, {0: (P, ARG)}, desc(d=256, h=256, dtype="f32", w_packed=True))


@pytest.mark.parametrize("name,nargs", [("locmoe_expert_ffn_in_save8", 7), ("locmoe_expert_ffn_dgrad8", 10)])
def test_activations_in_8_bits(name, nargs):
    plain, ws = getattr(lm, name), getattr(lm, name + "_ws")
    good = [P] * nargs
    refused(plain, good, {i: (None, NULL) for i in range(nargs)})
    good += [P, lm.LOCMOE_FFN_WS_BYTES]
    refused(ws, good, {i: (None, NULL) for i in range(nargs)})
    refused(ws, good, {nargs: (None, WS), nargs + 1: (lm.LOCMOE_FFN_WS_BYTES - 1, WS)})
    refused(ws, good, {nargs: (P + 2, WS)})
    refused(ws, good, {0: (P, SHAPE)}, desc(h=12))
    refused(ws, good, {0: (P, ARG)}, desc(w_packed=True))


def test_decode_block_takes_few_tokens():
    n = lm.locmoe_norm_workspace_bytes(desc(T=65))
    kb = lm.BlockBuffers(xn=P, rstd_in=P, rstd_out=P, dgamma_in=P, dgamma_out=P, ws=P, ws_bytes=n)  # (as allocated for 65 tokens)
    assert status(lm.decode_block, desc(T=65), P, P, P, lm.Block(), None, kb) == SHAPE
