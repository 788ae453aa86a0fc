"""The operators that put the layer into a transformer block, as cases to be timed: what is listed, more of the same ranges
(`draw`), the inputs of a case (`prepare`), one pass (`run`: in plain torch operations, or with `own` through the entry points of
`paper_2401_13920_amd.locmoe`), the same in 64 bits (`exact`) and what a pass cannot do without (`work`).

Kinds of pass:
  "few"        the whole layer for a handful of tokens, as decoding calls it
  "act8"       the expert FFN of a training step that keeps its hidden activations in 8 bits: forward and backward
  "norms"      the block's norms, forward: ahead of the layer with its gate, and behind it with score, scale and residual
  "norms_bwd"  the same, backward
"""
import math

import torch

own = False

# A case: kind; T tokens, width d, E experts, inner width h, capacity C in rows; storage dtype; `packed`: weights in the packed
# layout; `spread` of the tokens over the experts: "even", "zipf" or "hot" (70 % on four); `given`: the gating values come from
# the block's norm instead of being formed by the layer; `post`: a norm behind the layer too, else a scale per channel.
_DEFAULTS = dict(dtype="bf16", packed=False, spread="even", given=False, post=True, h=8)


def _case(name, kind, T, d, E, C, **more):
    return dict(_DEFAULTS, name=name, kind=kind, T=T, d=d, E=E, C=C, **more)


def listed():
    return [
        # one token of the small model's layer: the smallest call of a decoder, latency only
        _case("few_one_token", "few", 1, 1024, 16, 1, h=4096, packed=True),
        # a unit-sized model in fp32 storage, one batch of its decoder
        _case("few_f32", "few", 16, 128, 8, 16, h=256, dtype="f32"),
        # an odd number of sequences of a model whose width divides by nothing, weights row-major, gating values given
        _case("few_odd", "few", 5, 1600, 40, 5, h=6400, given=True),
        # 64 sequences of the headline layer
        _case("few_large", "few", 64, 4096, 64, 64, h=16384, packed=True, spread="zipf"),
        # a small layer of an odd expert count, row-major weights, uneven segments
        _case("act8_small", "act8", 1000, 384, 12, 167, h=1536, spread="zipf"),
        # a training step of the small model's layer
        _case("act8_mid", "act8", 8192, 1024, 16, 640, h=4096, packed=True),
        # a training step of the capacity ablation's layer
        _case("act8_large", "act8", 32768, 2048, 32, 1280, h=8192, packed=True, spread="zipf"),
        # the norms around a decoder's layer
        _case("norms_small", "norms", 64, 1024, 16, 64),
        # blocks of twelve features, which no vector of 16 bytes fits, fp32 storage, a scale per channel behind the layer
        _case("norms_odd_f32", "norms", 4999, 600, 50, 100, dtype="f32", spread="zipf", post=False),
        # the norms around the headline layer
        _case("norms_large", "norms", 65536, 4096, 64, 1280, spread="zipf"),
        # backward of the norms in fp32 storage, an odd token count
        _case("norms_bwd_odd_f32", "norms_bwd", 5003, 1600, 40, 157, dtype="f32", post=False),
        # backward of the norms around the headline layer
        _case("norms_bwd_large", "norms_bwd", 65536, 4096, 64, 1280, spread="zipf"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Layers between the smallest and the headline one; token counts that divide by nothing in particular."""
    kind = rng.choice(["few", "few", "act8", "act8", "norms", "norms_bwd"])
    while True:
        d = rng.choice([128, 256, 384, 512, 600, 640, 1000, 1024, 1280, 1600, 2048, 2560, 4096])
        E = rng.choice([4, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 50, 64, 80, 96, 128])
        h = rng.choice([2 * d, 4 * d, (8 * d // 3 + 7) // 8 * 8])
        c = dict(_DEFAULTS, kind=kind, d=d, E=E, spread=rng.choice(["even", "zipf", "hot"]), given=False, post=True)
        if d % E:
            continue
        if kind == "few":
            T = _log_int(rng, 1, 64)
            c.update(T=T, h=h, C=max(1, rng.choice([T, T, (T + 3) // 4])), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     given=rng.random() < 0.4)
            if E * d * h > 64 * 4096 * 16384:
                continue
        elif kind == "act8":
            T = _log_int(rng, 128, 32768)
            c.update(T=T, h=h, C=max(1, math.ceil(rng.choice([0.5, 1.0, 1.25, 2.0]) * T / E)))
            if min(T, E * c["C"]) * d * h > 4e11 or E * d * h > 32 * 2048 * 8192:
                continue
        else:
            T = _log_int(rng, 1, 65536)
            c.update(T=T, C=max(1, math.ceil(rng.choice([0.5, 1.0, 1.25]) * T / E)), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     post=rng.random() < 0.6)
            if T * d * (4 if c["dtype"] == "f32" else 2) > 65536 * 4096 * 2:
                continue
        if kind in ("few", "act8"):
            c["packed"] = c["dtype"] == "bf16" and d % 256 == 0 and h % 256 == 0 and rng.random() < 0.7
        return c


# ---- inputs ------------------------------------------------------------------------------------------------
EPS = 1e-5     # of the norms
SCALE = 0.7    # of the residual branch


def _storage(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _shares(case):
    """The experts' shares of the tokens."""
    E = case["E"]
    if case["spread"] == "even":
        p = [1.0] * E
    elif case["spread"] == "zipf":
        p = [(i + 1) ** -1.2 for i in range(E)]
    else:
        hot = {k * max(1, E // 4) % E for k in range(min(4, E))}
        p = [0.7 / len(hot) * (i in hot) + 0.3 / E for i in range(E)]
    return [v / sum(p) for v in p]


class _Inputs:
    """Seeded random tensors on the GPU."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed))

    def normal(self, *shape, std=1.0, dtype=torch.float32):
        return (std * torch.randn(*shape, generator=self.gen, device="cuda")).to(dtype)

    def weights(self, E, rows, cols):
        w = torch.empty(E, rows, cols, dtype=torch.bfloat16, device="cuda")
        for e in range(E):
            w[e].normal_(0.0, cols ** -0.5, generator=self.gen)
        return w

    def experts(self, case):
        p = torch.tensor(_shares(case), device="cuda")
        return torch.multinomial(p, case["T"], replacement=True, generator=self.gen)


def _packed(W):
    """The packed layout of W [E, N, K]: blocks of 256 rows x 32 columns, the four 16-byte chunks of a row permuted."""
    E, N, K = W.shape
    blocks = W.view(E, N // 256, 256, K // 32, 4, 8).permute(0, 1, 3, 2, 4, 5).contiguous()
    row = torch.arange(256, device=W.device)[:, None]
    chunk = (torch.arange(4, device=W.device)[None, :] ^ (row // 2 % 4)).view(1, 1, 1, 256, 4, 1)
    out = torch.empty_like(blocks)
    for e in range(E):
        out[e] = torch.gather(blocks[e], 3, chunk[0].expand_as(blocks[e]))
    return out.view(E, N, K)


def _slots(eid, E, C):
    """First-come slots under the capacity, experts in order: slot [T] (-1: dropped) and seg_off [E+1]."""
    T = eid.numel()
    cnt = torch.bincount(eid, minlength=E)
    order = torch.argsort(eid, stable=True)
    first = torch.cumsum(cnt, 0) - cnt
    pos = torch.empty_like(eid)
    pos[order] = torch.arange(T, device=eid.device) - first[eid[order]]
    kept = cnt.clamp(max=C)
    off = torch.zeros(E + 1, dtype=torch.int64, device=eid.device)
    off[1:] = torch.cumsum(kept, 0)
    return torch.where(pos < C, off[eid] + pos, -1).to(torch.int32), off.to(torch.int32)


class State:
    """What a program holds between passes: tokens, weights, routing and buffers."""


def prepare(case, seed):
    s, r = State(), _Inputs(seed)
    s.case = case
    T, d, E, h, C = (case[k] for k in ("T", "d", "E", "h", "C"))
    st = _storage(case)
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
    eid = r.experts(case)
    rows = E * C
    if case["kind"] == "few":
        # tokens near the direction of an expert, as a trained gate sees them
        blk = d // E
        s.x = (r.normal(T, d) + (torch.arange(d, device="cuda")[None, :] // blk == eid[:, None]) * (6.0 * blk ** -0.5)).to(st)
        s.g = s.x.float().view(T, E, blk).mean(2) if case["given"] else None
        s.W_in, s.W_out = r.weights(E, h, d), r.weights(E, d, h)
        if case["packed"]:
            s.Wp_in, s.Wp_out = _packed(s.W_in), _packed(s.W_out)
        s.eid, s.w, s.slot, s.y = torch.empty(T, **i32), torch.empty(T, **f32), torch.empty(T, **i32), torch.empty(T, d, dtype=st, device="cuda")
    else:
        s.slot, s.seg = _slots(eid, E, C)
        s.order = torch.arange(E, **i32)
        live = (torch.arange(rows, device="cuda") < s.seg[E])[:, None]
        w = torch.rand(T, generator=r.gen, device="cuda") * 0.9 + 0.1
    if case["kind"] == "act8":
        s.send = r.normal(rows, d, dtype=st) * live
        s.dout = r.normal(rows, d, std=d ** -0.5, dtype=st) * live
        s.W_in, s.W_out = r.weights(E, h, d), r.weights(E, d, h)
        s.Wt_in, s.Wt_out = s.W_in.transpose(1, 2).contiguous(), s.W_out.transpose(1, 2).contiguous()
        if case["packed"]:
            s.Wp_in, s.Wp_out, s.Wpt_in, s.Wpt_out = (_packed(W) for W in (s.W_in, s.W_out, s.Wt_in, s.Wt_out))
        bf = dict(dtype=torch.bfloat16, device="cuda")
        s.H, s.dZ = torch.empty(rows, h, **bf), torch.empty(rows, h, **bf)
        s.Zq, s.Zs = torch.empty(rows, h, dtype=torch.int8, device="cuda"), torch.empty(rows, -(-h // 16), **bf)
        s.out, s.dsend = torch.zeros(rows, d, **bf), torch.zeros(rows, d, **bf)
        s.dW_in, s.dW_out = torch.empty(E, h, d, **bf), torch.empty(E, d, h, **bf)
        s.ffn_ws = torch.zeros(128, dtype=torch.uint8, device="cuda")
    elif case["kind"] != "few":
        # a residual stream whose channels have scales of their own, as they grow in training
        s.x = r.normal(T, d).mul_(torch.exp(r.normal(d, std=0.5))).to(st)
        s.out = (r.normal(rows, d, std=0.3) * live).to(st)
        s.gamma_in, s.gamma_out, s.w = 1.0 + r.normal(d, std=0.1), 1.0 + r.normal(d, std=0.1), w
        s.xn, s.y, s.g = torch.empty_like(s.x), torch.empty_like(s.x), torch.empty(T, E, **f32)
        s.rstd_in, s.rstd_out = torch.empty(T, **f32), torch.empty(T, **f32)
        if case["kind"] == "norms_bwd":
            s.dy = r.normal(T, d, std=d ** -0.5).to(st)
            s.dsend = (r.normal(rows, d, std=d ** -0.5) * live).to(st)
            s.dg = r.normal(T, E, std=0.01)
            # (rounded from 64 bits, as the forward leaves them)
            s.rstd_in = (s.x.double().square().mean(1) + EPS).rsqrt().float()
            at = s.out[s.slot.clamp(min=0).long()].double()
            s.rstd_out = torch.where(s.slot >= 0, (at.square().mean(1) + EPS).rsqrt(), 0.0).float()
            s.dout, s.dx, s.dw = torch.zeros(rows, d, dtype=st, device="cuda"), torch.empty_like(s.x), torch.empty(T, **f32)
            s.dgamma_in, s.dgamma_out = torch.empty(d, **f32), torch.empty(d, **f32)
    if own:
        from paper_2401_13920_amd import locmoe as lm
        s.lm = lm
        s.desc = lm.make_desc(T, d, E, 1, h, C, case["dtype"], w_packed=case["packed"])
        s.ws_bytes = {"few": lm.locmoe_layer_few_workspace_bytes, "act8": lambda _: 0}.get(
            case["kind"], lm.locmoe_norm_workspace_bytes)(s.desc)
        s.ws = torch.empty(max(1, s.ws_bytes), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------
def run(s):
    return globals()[("_own_" if own else "_plain_") + s.case["kind"]](s)


def _own_few(s):
    lm, packed = s.lm, s.case["packed"]
    lm.locmoe_layer_few(s.desc, s.x, s.g, None, s.Wp_in if packed else s.W_in, s.Wp_out if packed else s.W_out, True, s.eid, s.w,
                        s.slot, s.y, s.ws, s.ws_bytes)
    return {"y": s.y, "eid": s.eid, "w": s.w, "slot": s.slot}


def _own_act8(s):
    lm, d = s.lm, s.desc
    Wi, Wo, Wti, Wto = (s.Wp_in, s.Wp_out, s.Wpt_in, s.Wpt_out) if s.case["packed"] else (s.W_in, s.W_out, s.Wt_in, s.Wt_out)
    lm.locmoe_expert_ffn_in_save8_ws(d, s.send, s.seg, s.order, Wi, s.H, s.Zq, s.Zs, s.ffn_ws, 128)
    lm.locmoe_expert_ffn_out_ws(d, s.H, s.seg, s.order, Wo, s.out, s.ffn_ws, 128)
    lm.locmoe_expert_ffn_dgrad8_ws(d, s.dout, s.Zq, s.Zs, s.seg, s.order, Wto, Wti, s.dZ, s.H, s.dsend, s.ffn_ws, 128)
    lm.locmoe_expert_ffn_wgrad(d, s.send, s.H, s.dout, s.dZ, s.seg, s.order, s.dW_in, s.dW_out)
    return {"out": s.out, "dsend": s.dsend, "dW_in": s.dW_in, "dW_out": s.dW_out}


def _own_norms(s):
    lm, d = s.lm, s.desc
    lm.locmoe_norm_gate(d, s.x, s.gamma_in, EPS, s.xn, s.rstd_in, s.g)
    lm.locmoe_combine_norm(d, s.out, s.slot, s.w, s.x, s.gamma_out, s.case["post"], EPS, SCALE, s.y, s.rstd_out)
    return {"xn": s.xn, "rstd_in": s.rstd_in, "g": s.g, "y": s.y, "rstd_out": s.rstd_out}


def _own_norms_bwd(s):
    lm, d = s.lm, s.desc
    lm.locmoe_combine_norm_bwd(d, s.dy, s.out, s.slot, s.w, s.gamma_out, s.case["post"], SCALE, s.rstd_out, s.dout, s.dw,
                               s.dgamma_out, s.ws, s.ws_bytes)
    lm.locmoe_dispatch_norm_bwd(d, s.dsend, s.slot, s.dg, s.x, s.gamma_in, s.rstd_in, s.dy, s.dx, s.dgamma_in, s.ws, s.ws_bytes)
    return {"dout": s.dout, "dw": s.dw, "dgamma_out": s.dgamma_out, "dx": s.dx, "dgamma_in": s.dgamma_in}


def _gelu(z):
    return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))


def _gelu_grad(z):
    return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2.0 * math.pi) ** -0.5


def _plain_few(s):
    T, E, C, d = s.case["T"], s.case["E"], s.case["C"], s.case["d"]
    x = s.x.float()
    g = torch.relu(x.view(T, E, d // E).mean(2) if s.g is None else s.g)
    eid = torch.argmax((g == g.amax(1, keepdim=True)).to(torch.int8), 1)  # ties: the lowest index
    w = 1.0 / torch.exp(g - g.amax(1, keepdim=True)).sum(1)
    before = torch.tril(eid[:, None] == eid[None, :], -1).sum(1)
    kept = before < C
    H = _gelu(torch.matmul(s.W_in[eid].float(), x[:, :, None]))
    out = torch.matmul(s.W_out[eid].float(), H)[:, :, 0]
    slot = torch.where(kept, torch.arange(T, device=x.device), -1)
    return {"y": ((w * kept)[:, None] * out).to(s.x.dtype), "eid": eid.to(torch.int32), "w": w, "slot": slot.to(torch.int32)}


def _plain_act8(s):
    E, C, d, h = (s.case[k] for k in ("E", "C", "d", "h"))
    # the segments side by side, every one padded to the capacity
    at = s.seg[:-1, None].long() + torch.arange(C, device="cuda")[None, :]
    live = at < s.seg[1:, None]
    at = torch.where(live, at, E * C)  # (a row of zeros behind the last)
    rows = lambda t: torch.cat([t, t.new_zeros(1, d)])[at].float()  # noqa: E731
    x, dout = rows(s.send), rows(s.dout)
    z = torch.bmm(x, s.Wt_in.float())
    out = torch.bmm(_gelu(z), s.Wt_out.float())
    pad = -h % 16
    blocks = torch.nn.functional.pad(z, (0, pad)).view(E, C, -1, 16)
    unit = (blocks.abs().amax(3, keepdim=True) / 127.0).to(torch.bfloat16).float()
    z8 = (torch.round(blocks / torch.where(unit > 0, unit, 1.0)) * unit).view(E, C, -1)[:, :, :h]
    dZ = torch.bmm(dout, s.W_out.float()) * _gelu_grad(z8)
    dsend = torch.bmm(dZ, s.W_in.float())
    dW_in = torch.bmm(dZ.transpose(1, 2).contiguous(), x)
    dW_out = torch.bmm(dout.transpose(1, 2).contiguous(), _gelu(z8))

    def back(t):
        flat = torch.zeros(E * C + 1, d, device="cuda")
        flat[at.view(-1)] = t.reshape(-1, d)
        return flat[:-1].to(torch.bfloat16)
    return {"out": back(out), "dsend": back(dsend), "dW_in": dW_in.to(torch.bfloat16), "dW_out": dW_out.to(torch.bfloat16)}


def _plain_norms(s):
    T, E, d = s.case["T"], s.case["E"], s.case["d"]
    x = s.x.float()
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    xn = x * rstd[:, None] * s.gamma_in
    o = s.out[s.slot.clamp(min=0).long()].float()
    kept = s.slot >= 0
    r2 = 1.0 / torch.sqrt((o * o).mean(1) + EPS) if s.case["post"] else torch.ones(T, device="cuda")
    y = x + (SCALE * s.w * r2 * kept)[:, None] * s.gamma_out * o
    return {"xn": xn.to(s.x.dtype), "rstd_in": rstd, "g": xn.view(T, E, d // E).mean(2), "y": y.to(s.x.dtype),
            "rstd_out": torch.where(kept, r2, 0.0)}


def _plain_norms_bwd(s):
    E, d, post = s.case["E"], s.case["d"], s.case["post"]
    kept = s.slot >= 0
    at = s.slot.clamp(min=0).long()
    dy, x = s.dy.float(), s.x.float()
    n = s.out[at].float() * (s.rstd_out * kept if post else kept)[:, None]
    u = SCALE * s.gamma_out * dy
    dw = (u * n).sum(1)
    dgamma_out = SCALE * (s.w[:, None] * dy * n).sum(0)
    dn = s.w[:, None] * (s.rstd_out[:, None] * (u - n * (dw / d)[:, None]) if post else u)
    dout = torch.zeros(s.out.shape[0] + 1, d, device="cuda")
    dout[torch.where(kept, at, s.out.shape[0])] = dn
    dxn = s.dsend[at].float() * kept[:, None] + (s.dg * (E / d)).repeat_interleave(d // E, 1)
    xh = x * s.rstd_in[:, None]
    dh = dxn * s.gamma_in
    dx = dy + s.rstd_in[:, None] * (dh - xh * (dh * xh).mean(1, keepdim=True))
    return {"dout": dout[:-1].to(s.x.dtype), "dw": dw, "dgamma_out": dgamma_out, "dx": dx.to(s.x.dtype),
            "dgamma_in": (dxn * xh).sum(0)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, prepare(case, seed))


def _phi(z):
    return torch.special.ndtr(z)


def _exact_few(case, s):
    T, d, E, C = (case[k] for k in ("T", "d", "E", "C"))
    y, eids, ws, slots = torch.zeros(T, d, dtype=torch.float64, device="cuda"), [], [], []
    for m in range(T):
        x = s.x[m].double()
        G = (x.reshape(E, -1).sum(1) * (E / d) if s.g is None else s.g[m].double()).clamp(min=0.0)
        e = min(i for i, v in enumerate(G.tolist()) if v == float(G.max()))
        p = float(torch.softmax(G, 0)[e])
        keep = eids.count(e) < C
        if keep:
            z = s.W_in[e].double() @ x
            y[m] = p * (s.W_out[e].double() @ (z * _phi(z)))
        eids.append(e), ws.append(p), slots.append(m if keep else -1)
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"y": y, "eid": torch.tensor(eids, **i32), "w": torch.tensor(ws, dtype=torch.float64, device="cuda"),
            "slot": torch.tensor(slots, **i32)}


def _exact_act8(case, s):
    E, h = case["E"], case["h"]
    out, dsend = torch.zeros_like(s.send, dtype=torch.float64), torch.zeros_like(s.send, dtype=torch.float64)
    dW_in, dW_out = (torch.zeros_like(W, dtype=torch.float64) for W in (s.W_in, s.W_out))
    seg = s.seg.tolist()
    for e in range(E):
        a, b = seg[e], seg[e + 1]
        if a == b:
            continue
        x, dout, Wi, Wo = (t.double() for t in (s.send[a:b], s.dout[a:b], s.W_in[e], s.W_out[e]))
        z = x @ Wi.T
        out[a:b] = (z * _phi(z)) @ Wo.T
        for c in range(0, h, 16):
            part = z[:, c:c + 16]
            unit = (part.abs().max(1).values / 127).to(torch.bfloat16).double()[:, None]
            z[:, c:c + 16] = torch.where(unit > 0, (part / unit).round() * unit, 0.0)
        P = _phi(z)
        dZ = (dout @ Wo) * (P + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        dsend[a:b] = dZ @ Wi
        dW_in[e], dW_out[e] = dZ.T @ x, dout.T @ (z * P)
    return {"out": out, "dsend": dsend, "dW_in": dW_in, "dW_out": dW_out}


def _exact_norms(case, s):
    T, d, E = (case[k] for k in ("T", "d", "E"))
    xn, y = torch.empty(T, d, dtype=torch.float64, device="cuda"), s.x.double()
    kept = (s.slot >= 0).nonzero()[:, 0]
    rstd, r2 = (s.x.double().pow(2).sum(1) / d + EPS).pow(-0.5), torch.zeros(T, dtype=torch.float64, device="cuda")
    torch.mul(s.x.double() * s.gamma_in.double(), rstd[:, None], out=xn)
    o = s.out.double()[s.slot[kept].long()]
    r2[kept] = (o.pow(2).sum(1) / d + EPS).pow(-0.5) if case["post"] else 1.0
    y[kept] += o * s.gamma_out.double() * (r2[kept] * s.w[kept].double() * SCALE)[:, None]
    return {"xn": xn, "rstd_in": rstd, "g": xn.reshape(T * E, -1).sum(1).view(T, E) * (E / d), "y": y, "rstd_out": r2}


def _exact_norms_bwd(case, s):
    """The chain rule, a step at a time, over the kept tokens alone."""
    T, d, E = (case[k] for k in ("T", "d", "E"))
    kept = (s.slot >= 0).nonzero()[:, 0]
    rows = s.slot[kept].long()
    dy, o, w, gamma = s.dy.double(), s.out.double()[rows], s.w.double()[kept], s.gamma_out.double()
    branch = SCALE * dy[kept]                      # with respect to w gamma n
    r = s.rstd_out.double()[kept][:, None] if case["post"] else 1.0
    dn = branch * gamma * w[:, None]
    dout, dw = torch.zeros(s.out.shape, dtype=torch.float64, device="cuda"), torch.zeros(T, dtype=torch.float64, device="cuda")
    dw[kept] = torch.sum(branch * gamma * (o * r), 1)
    dout[rows] = r * dn - (r ** 3 / d) * torch.sum(dn * o, 1, keepdim=True) * o if case["post"] else dn
    dgamma_out = torch.sum(branch * w[:, None] * (o * r), 0)
    dxn = (s.dg.double() * E / d)[:, :, None].expand(T, E, d // E).reshape(T, d).clone()
    dxn[kept] += s.dsend.double()[rows]
    x, r = s.x.double(), s.rstd_in.double()[:, None]
    dgamma_in = torch.sum(dxn * x * r, 0)
    dxn *= s.gamma_in.double()
    dx = dy + r * dxn - x * (r ** 3 * torch.sum(dxn * x, 1, keepdim=True) / d)
    return {"dout": dout, "dw": dw, "dgamma_out": dgamma_out, "dx": dx, "dgamma_in": dgamma_in}


# ---- what a pass cannot do without -----------------------------------------------------------------------------
def work(case):
    T, d, E, h, C = (case[k] for k in ("T", "d", "E", "h", "C"))
    b = 2 if case["dtype"] == "bf16" else 4
    p = _shares(case)
    K = sum(min(T * v, C) for v in p)  # rows that reach the experts
    x = T * d * b
    if case["kind"] == "few":
        used = sum(1.0 - (1.0 - v) ** T for v in p)  # experts whose weights are read
        return {"bytes": 2 * x + used * 4.0 * d * h + 12 * T, "flops": 4.0 * K * d * h}
    if case["kind"] == "act8":
        # send and dout read, out and dsend written; both weights for the forward and transposed for the backward; both
        # gradients; 9 bits for each hidden value, written and read again
        return {"bytes": 4 * K * d * b + 6 * 2.0 * E * d * h + 2 * 9 / 8 * K * h, "flops": 12.0 * K * d * h}
    if case["kind"] == "norms":
        # x for the norm ahead of the layer, and again as the residual behind it: the layer's own work lies in between
        return {"bytes": 4 * x + K * d * b + 4 * T * E + 20 * T, "flops": 6.0 * T * d + 6.0 * K * d}
    # dy of the kept tokens for the layer's output, dy again as the residual's gradient; x and dsend; dx and dout
    return {"bytes": 3 * x + 4 * K * d * b + 4 * T * E + 20 * T + 16 * d, "flops": 12.0 * T * d + 12.0 * K * d}
