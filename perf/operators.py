"""The operators of a mixture-of-experts feed-forward block in microscaled FP4, as measurable cases.

Eight kinds, in the order in which a block meets them:

  route          scores of a token's experts, selection (bias for balance, groups, top-k), weights, and the plan that sorts
                 the chosen (token, expert) pairs into slots, expert by expert
  route_grads    gradient of the router's logits from that of the weights
  experts        product of the slots' rows with their experts' MXFP4 weights, the rows quantized to MXFP4 on the way
                 (gather: the rows are the tokens', else the slots'); forward and input gradient are the same call
  experts_wgrad  the experts' weight gradients, both operands quantized along the slots of each expert
  combine        a token's weighted sum over its experts' rows
  combine_grads  gradients of those rows and of the weights
  activation     gated activation that leaves an 8-bit checkpoint of its inputs, and the gradient taken from the checkpoint
  checkpoint     a tensor saved in 8 bits and restored

`run` computes them by elementary torch operations, or, where `own` is true, by the framework's calls.

Sizes: the hidden size and the token counts of the benchmark's configurations, 8 to 256 experts, ragged and odd ones between.  Tokens
choose their experts with a mild imbalance, as a router with a balancing bias leaves it.
"""
import math

import torch

own = False

BLOCK = 32                                       # elements under one scale


def listed():
    return [
        # one token of a served model passes the router: latency is all it costs
        dict(name="route_token", kind="route", T=1, E=64, k=4, scores="softmax", groups=1, top_groups=1, bias=False, renorm=True, padded=False),
        # a packed batch of 16384 tokens, some of them padding, through a router with many experts in groups
        dict(name="route_batch", kind="route", T=16384, E=256, k=8, scores="sigmoid", groups=8, top_groups=4, bias=True, renorm=True,
             padded=True),
        # the router's backward pass, probabilities over all experts not renormalised (every logit has a gradient)
        dict(name="route_grads", kind="route_grads", T=16384, E=64, k=4, scores="softmax", renorm=False, dtype="f32"),
        # one token through its four experts' stacked gate and up projections
        dict(name="experts_token", kind="experts", T=1, E=64, k=4, N=2048, K=4096, gather=True, out="bf16"),
        # the down projections of a decode step of 24 sequences
        dict(name="experts_decode", kind="experts", T=24, E=64, k=4, N=4096, K=1024, gather=False, out="bf16"),
        # a prompt of 1000 tokens: some sixty rows an expert
        dict(name="experts_prompt", kind="experts", T=1000, E=64, k=4, N=2048, K=4096, gather=True, out="bf16"),
        # training, gate and up projections of 16384 tokens
        dict(name="experts_step", kind="experts", T=16384, E=64, k=4, N=2048, K=4096, gather=True, out="bf16"),
        # training, weight gradient of the same projections over half the batch
        dict(name="experts_wgrad", kind="experts_wgrad", T=8192, E=64, k=4, N=2048, K=4096, gather=True, out="bf16"),
        # the experts' rows back to the tokens, and the gradients of that
        dict(name="combine_step", kind="combine", T=16384, k=4, D=4096, E=64, dtype="bf16"),
        dict(name="combine_grads", kind="combine_grads", T=8192, k=4, D=4096, E=64, dtype="bf16"),
        # training, gated activation of 16384 tokens' four experts, forward and backward
        dict(name="activation_step", kind="activation", S=65536, F=1024),
        # a small activation of odd length kept for the backward pass
        dict(name="checkpoint_odd", kind="checkpoint", M=1111, N=2080, dtype="bf16"),
    ]


def _log_uniform(rng, lo, hi, multiple=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(max(multiple * round(v / multiple), multiple * math.ceil(lo / multiple)), hi // multiple * multiple)


def draw(rng):
    kind = rng.choice(["route", "route_grads", "experts", "experts", "experts", "experts_wgrad", "experts_wgrad", "combine",
                       "combine_grads", "activation", "checkpoint"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    E, k = rng.choice([8, 16, 32, 60, 64, 96, 128, 160, 256]), rng.randint(1, 8)
    T = _log_uniform(rng, 1, 16384)
    if kind == "route":
        groups, top_groups = rng.choice([(1, 1), (1, 1), (4, 2), (4, 3)])
        k = min(k, E // groups * top_groups)
        return dict(kind=kind, T=T, E=E, k=k, scores=rng.choice(["softmax", "sigmoid"]), groups=groups, top_groups=top_groups,
                    bias=rng.random() < 0.5, renorm=rng.random() < 0.7, padded=rng.random() < 0.4)
    if kind == "route_grads":
        return dict(kind=kind, T=_log_uniform(rng, 16, 16384), E=E, k=k, scores=rng.choice(["softmax", "sigmoid"]),
                    renorm=rng.random() < 0.5, dtype=dtype)
    if kind in ("experts", "experts_wgrad"):
        multiple = 32 if kind == "experts" else 8
        N, K = _log_uniform(rng, 64, 4096, 8), _log_uniform(rng, 256, 8192, multiple)
        T = _log_uniform(rng, 1 if kind == "experts" else 32, 16384)
        while E * N * K > 64 * 2048 * 4096:
            E //= 2
        # rows: the product's work, and what the padding to the fullest expert costs the plain form
        while T * k * N * K > 65536 * 2048 * 4096 or T * k * max(N, K) > 65536 * 4096:
            T //= 2
        return dict(kind=kind, T=T, E=E, k=min(k, E), N=N, K=K, gather=rng.random() < 0.5,
                    out="bf16" if kind == "experts" else dtype)
    if kind in ("combine", "combine_grads"):
        D = _log_uniform(rng, 64, 8192, rng.choice([1, 8, 8]))
        T = _log_uniform(rng, 8, 16384)
        while T * k * D > 65536 * 4096 // (2 if dtype == "f32" else 1):
            T //= 2
        return dict(kind=kind, T=T, k=k, D=D, E=E, dtype=dtype)
    if kind == "activation":
        F, S = _log_uniform(rng, 64, 8192, 32), _log_uniform(rng, 16, 65536)
        while S * F > 65536 * 1024:
            S //= 2
        return dict(kind=kind, S=S, F=F)
    M, N = _log_uniform(rng, 32, 16384), _log_uniform(rng, 128, 8192, 32)
    return dict(kind=kind, M=M, N=N, dtype=dtype)


_TYPES = dict(bf16=torch.bfloat16, f32=torch.float32)


# ---- inputs ---------------------------------------------------------------------------------------------------------

class _Draws:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1))

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)

    def logits(self, T, E):
        """Spread over the experts as of a trained router, with an imbalance between the experts."""
        return 1.5 * self.normal(T, E) + 0.15 * self.normal(1, E)

    def activation(self, M, N):
        """Unit scale, one channel in a thousand twenty times larger."""
        return self.normal(M, N) * torch.where(self.uniform(1, N) < 0.001, 20.0, 1.0)

    def gradient(self, M, N):
        """Rows of very different scale."""
        return 1e-3 * self.normal(M, N) * torch.exp(self.normal(M, 1))

    def plan(self, T, E, k):
        idx = torch.topk(self.logits(T, E), k, dim=1).indices
        return _plan(idx, E)


def prepare(case, seed):
    d = _Draws(seed)
    kind = case["kind"]
    s = dict(case=case)
    if kind == "route":
        T, E = case["T"], case["E"]
        s["logits"] = d.logits(T, E)
        if T >= 64:                              # an expert out of service, and one token with a single expert left
            s["logits"][:, E - 1] = -math.inf
            s["logits"][T // 2, 1:] = torch.finfo(torch.float32).min
        s["bias"] = 0.05 * d.normal(E) if case["bias"] else None
        s["valid"] = (d.uniform(T) > 0.03).to(torch.uint8) if case["padded"] else None
    elif kind == "route_grads":
        T, E, k = case["T"], case["E"], case["k"]
        s["logits"] = d.logits(T, E).to(_TYPES[case["dtype"]])
        s["idx"] = torch.topk(s["logits"].float(), k, dim=1).indices.to(torch.int32)
        s["idx"][T // 3] = -1                    # a padding token
        s["dw"] = d.normal(T, k)
    elif kind in ("experts", "experts_wgrad"):
        T, E, k, N, K = (case[x] for x in ("T", "E", "k", "N", "K"))
        s["plan"] = d.plan(T, E, k)
        s["most"] = int((s["plan"][0][1:] - s["plan"][0][:-1]).max())
        s["x"] = d.activation(T if case["gather"] else T * k, K).to(torch.bfloat16)
        if kind == "experts":                    # weights quantized when the model was loaded
            s["codes"], s["scales"] = _mx_encode(0.02 * d.normal(E * N, K))
        else:
            s["g"] = d.gradient(T * k, N).to(torch.bfloat16)
    elif kind in ("combine", "combine_grads"):
        T, k, D, E = (case[x] for x in ("T", "k", "D", "E"))
        s["plan"] = d.plan(T, max(E, k), k)
        s["rows"] = d.normal(T * k, D).to(_TYPES[case["dtype"]])
        s["weights"] = torch.softmax(d.normal(T, k), dim=1)
        s["dy"] = d.gradient(T, D).to(torch.bfloat16) if kind == "combine_grads" else None
    elif kind == "activation":
        S, F = case["S"], case["F"]
        s["gu"] = (1.5 * d.activation(S, 2 * F)).to(torch.bfloat16)
        s["dact"] = d.gradient(S, F).to(torch.bfloat16)
    else:
        s["a"] = d.activation(case["M"], case["N"]).to(_TYPES[case["dtype"]])
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _grid():
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float32, device="cuda")


def _mx_scaled(x):
    """x [..., n] as blocks over their MXFP4 scales, and the scales' exponents: 2^(floor(log2 of the largest) - 2)."""
    b = x.unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(amax).exponent - 3).clamp(-127, 127)
    e = torch.where(amax > 0, e, -127)
    return torch.ldexp(b, -e), e


def _mx_codes(y):
    """E2M1 codes, nearest, ties to the even code, larger ones saturated."""
    a = y.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return c | (torch.signbit(y).to(torch.uint8) << 3)


def _mx_encode(x):
    y, e = _mx_scaled(x)
    c = _mx_codes(y).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), (e.squeeze(-1) + 127).to(torch.uint8)


def _mx_values(codes, scales):
    v = _grid()[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, BLOCK)) * torch.exp2(scales.float() - 127).unsqueeze(-1)).flatten(-2)


def _mx_round(x):
    y, e = _mx_scaled(x)
    return torch.ldexp(_grid()[_mx_codes(y).int()], e).flatten(-2)


def _mx8_round(x):
    """E4M3 under the smallest power of two that covers the block."""
    b = x.unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, (e - torch.where(m <= 0.875, 9, 8)).clamp(-127, 127), -127)
    return torch.ldexp(torch.ldexp(b, -e).to(torch.float8_e4m3fn).float(), e).flatten(-2)


def _plan(idx, E):
    """offsets [E + 1], token of each slot, slot of each choice: slots ordered by expert, then by choice; -1 where there is none."""
    T, k = idx.shape
    ids = torch.where(idx < 0, E, idx).flatten().long()
    ordered, order = torch.sort(ids, stable=True)
    offsets = torch.searchsorted(ordered, torch.arange(E + 1, device=idx.device)).to(torch.int32)
    used = ordered < E
    token = torch.where(used, order // k, -1).to(torch.int32)
    slot = torch.empty_like(order).scatter_(0, order, torch.where(used, torch.arange(T * k, device=idx.device), -1))
    return offsets, token, slot.view(T, k).to(torch.int32)


def _plain_route(s):
    c, x = s["case"], s["logits"].float()
    T, E, k, G = x.shape[0], c["E"], c["k"], c["groups"]
    alive = x > -math.inf
    if s["valid"] is not None:
        alive = alive & (s["valid"] != 0)[:, None]
    sigmoid = c["scores"] == "sigmoid"
    scores = 1 / (1 + torch.exp(-x)) if sigmoid else x
    key = scores if s["bias"] is None else scores + s["bias"]
    key = torch.where(alive, key, -math.inf)
    if c["top_groups"] < G:
        best = torch.topk(key.view(T, G, E // G), min(2, E // G), dim=2).values
        second = best[..., -1] if sigmoid and E // G > 1 else torch.full_like(best[..., 0], -math.inf)
        score = best[..., 0] + torch.where(second > -math.inf, second, 0.0)
        chosen = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=x.device).scatter_(1, chosen, True)
        key = torch.where(keep.repeat_interleave(E // G, 1), key, -math.inf)
    values, idx = torch.sort(key, dim=1, descending=True, stable=True)
    got, idx = values[:, :k] > -math.inf, idx[:, :k]
    picked = torch.where(got, scores.gather(1, idx), 0.0 if sigmoid else -math.inf)
    if sigmoid:
        total = picked.sum(1, keepdim=True)
        w = torch.where(total > 0, picked / total, 0.0) if c["renorm"] else picked
    else:
        over = picked if c["renorm"] else torch.where(alive, x, -math.inf)
        top = over.amax(1, keepdim=True)
        e = torch.exp(over - top).sum(1, keepdim=True)
        w = torch.where(got, torch.exp(picked - top) / e, 0.0)
    idx = torch.where(got, idx, -1).to(torch.int32)
    return (idx, w) + _plan(idx, E)


def _plain_route_grads(s):
    c, x, idx, dw = s["case"], s["logits"].float(), s["idx"].long(), s["dw"]
    got = idx >= 0
    at = idx.clamp(min=0)
    dw = torch.where(got, dw, 0.0)
    if c["scores"] == "sigmoid":
        p = torch.where(got, 1 / (1 + torch.exp(-x.gather(1, at))), 0.0)
        dp = dw
        if c["renorm"]:
            total = p.sum(1, keepdim=True)
            dp = torch.where(total > 0, (dw - (dw * p).sum(1, keepdim=True) / total) / total, 0.0)
        dx = torch.zeros_like(x).scatter_add_(1, at, dp * p * (1 - p))
    elif c["renorm"]:
        p = torch.where(got, torch.softmax(torch.where(got, x.gather(1, at), -math.inf), 1), 0.0)
        dx = torch.zeros_like(x).scatter_add_(1, at, p * (dw - (dw * p).sum(1, keepdim=True)))
    else:
        e = torch.exp(x - x.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
        dx = p * (torch.zeros_like(x).scatter_add_(1, at, dw) - (dw * p.gather(1, at)).sum(1, keepdim=True))
    return dx.to(s["logits"].dtype)


def _by_expert(s):
    """For each expert its slots, as many places as the fullest has, and which of the places are taken."""
    offsets = s["plan"][0].long()
    at = offsets[:-1, None] + torch.arange(s["most"], device="cuda")
    return at.clamp(max=s["plan"][1].numel() - 1), at < offsets[1:, None]


def _plain_experts(s):
    c, (offsets, token, _) = s["case"], s["plan"]
    E, N, K, S = c["E"], c["N"], c["K"], token.numel()
    x = _mx_round(s["x"].float())
    if c["gather"]:
        x = x[token.long()]
    codes, scales = s["codes"].view(E, N, -1), s["scales"].view(E, N, -1)
    expert = torch.searchsorted(offsets[1:], torch.arange(S, device="cuda", dtype=torch.int32), right=True)
    if S < E:                                    # few rows: only their experts' weights
        out = (_mx_values(codes[expert], scales[expert]) @ x[:, :, None]).squeeze(2)
    else:
        at, taken = _by_expert(s)
        out = torch.bmm(x[at] * taken[..., None], _mx_values(codes, scales).transpose(1, 2))
        out = out[expert, torch.arange(S, device="cuda") - offsets.long()[expert]]
    return out.to(_TYPES[c["out"]])


def _plain_experts_wgrad(s):
    c = s["case"]
    at, taken = _by_expert(s)
    pad = (0, 0, 0, -s["most"] % BLOCK)
    g = s["g"].float()[at] * taken[..., None]
    x = (s["x"][s["plan"][1].long()] if c["gather"] else s["x"]).float()[at] * taken[..., None]
    g = _mx_round(torch.nn.functional.pad(g, pad).transpose(1, 2).contiguous())
    x = _mx_round(torch.nn.functional.pad(x, pad).transpose(1, 2).contiguous())
    return torch.bmm(g, x.transpose(1, 2)).flatten(0, 1).to(_TYPES[c["out"]])


def _plain_combine(s):
    rows = s["rows"].float()[s["plan"][2].long()]
    return (rows * s["weights"][..., None]).sum(1).to(torch.bfloat16)


def _plain_combine_grads(s):
    slot, dy = s["plan"][2].long(), s["dy"].float()
    drows = torch.empty_like(s["rows"])
    drows[slot] = (dy[:, None, :] * s["weights"][..., None]).to(drows.dtype)
    return drows, (s["rows"].float()[slot] * dy[:, None, :]).sum(2)


def _plain_activation(s):
    g, u = s["gu"].float().chunk(2, 1)
    act = (g / (1 + torch.exp(-g)) * u).to(torch.bfloat16)
    g, u = _mx8_round(s["gu"].float()).chunk(2, 1)              # what the backward pass has
    d, p = s["dact"].float(), 1 / (1 + torch.exp(-g))
    again = (g * p * u).to(torch.bfloat16)
    return act, torch.cat((d * u * p * (1 + g * (1 - p)), d * g * p), 1).to(torch.bfloat16), again


def _plain_checkpoint(s):
    return _mx8_round(s["a"].float()).to(s["a"].dtype)


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _empty(rows, cols, dtype):
    return torch.empty((rows, cols), dtype=dtype, device="cuda")


def _own_plan(metis, s, E):
    offsets, token, slot = s["plan"]
    return metis.ExpertPlan(slot.shape[0], E, slot.shape[1], buffers=(offsets, token, slot))


def _own_route(metis, s):
    c = s["case"]
    idx, w = metis.route(s["logits"], c["k"], bias=s["bias"], valid=s["valid"], scores=c["scores"], groups=c["groups"],
                         top_groups=c["top_groups"], renorm=c["renorm"])
    plan = metis.dispatch(idx, c["E"])
    return idx, w, plan.offsets, plan.token, plan.slot


def _own_route_grads(metis, s):
    c = s["case"]
    return metis.route_grads(s["logits"], s["idx"], s["dw"], scores=c["scores"], renorm=c["renorm"])


def _own_experts(metis, s):
    c = s["case"]
    W = metis.MxTensor(c["E"] * c["N"], c["K"], buffers=(s["codes"], s["scales"]))
    out = _empty(c["T"] * c["k"], c["N"], _TYPES[c["out"]])
    return metis.experts_product(s["x"], W, _own_plan(metis, s, c["E"]), out, gather=c["gather"])


def _own_experts_wgrad(metis, s):
    c = s["case"]
    dW = _empty(c["E"] * c["N"], c["K"], _TYPES[c["out"]])
    return metis.experts_wgrad(s["g"], s["x"], _own_plan(metis, s, c["E"]), dW, gather=c["gather"])


def _own_combine(metis, s):
    c = s["case"]
    return metis.combine(s["rows"], _own_plan(metis, s, max(c["E"], c["k"])), _empty(c["T"], c["D"], torch.bfloat16), s["weights"])


def _own_combine_grads(metis, s):
    c = s["case"]
    return metis.combine_grads(s["dy"], s["rows"], _own_plan(metis, s, max(c["E"], c["k"])), s["weights"])


def _own_activation(metis, s):
    S, F = s["case"]["S"], s["case"]["F"]
    act, again, dgu = _empty(S, F, torch.bfloat16), _empty(S, F, torch.bfloat16), _empty(S, 2 * F, torch.bfloat16)
    saved = metis.Mx8Tensor(S, 2 * F)
    metis.swiglu(s["gu"], act, saved)
    metis.swiglu_grads(saved, s["dact"], dgu, again)
    return act, dgu, again


def _own_checkpoint(metis, s):
    a = s["a"]
    saved = metis.quantize_mx8(a, metis.Mx8Tensor(*a.shape))
    return metis.dequantize_mx8(saved, torch.empty_like(a))


_PLAIN = dict(route=_plain_route, route_grads=_plain_route_grads, experts=_plain_experts, experts_wgrad=_plain_experts_wgrad,
              combine=_plain_combine, combine_grads=_plain_combine_grads, activation=_plain_activation, checkpoint=_plain_checkpoint)
_OWN = dict(route=_own_route, route_grads=_own_route_grads, experts=_own_experts, experts_wgrad=_own_experts_wgrad,
            combine=_own_combine, combine_grads=_own_combine_grads, activation=_own_activation, checkpoint=_own_checkpoint)


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2509_00404_amd import metis
        return _OWN[kind](metis, state)
    return _PLAIN[kind](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    kind, k = case["kind"], case.get("k", 1)
    size = 4.0 if case.get("dtype", case.get("out")) == "f32" else 2.0
    if kind == "route":                          # logits in; choices, weights, the plan out
        T, E = case["T"], case["E"]
        return dict(bytes=4.0 * T * E + 16.0 * T * k + 4.0 * E, flops=0.0)
    if kind == "route_grads":
        T, E = case["T"], case["E"]
        return dict(bytes=2 * size * T * E + 8.0 * T * k, flops=0.0)
    if kind == "activation":                     # the checkpoint is written by one call and read by the other
        n = case["S"] * case["F"]
        return dict(bytes=n * (4.0 + 2.0 + 2 * 2.0625 + 2.0 + 4.0 + 2.0), flops=0.0)
    if kind == "checkpoint":
        return dict(bytes=case["M"] * case["N"] * (2 * size + 2 * 1.03125), flops=0.0)
    T, S = case["T"], case["T"] * k
    if kind == "combine":
        return dict(bytes=size * S * case["D"] + 2.0 * T * case["D"] + 8.0 * S, flops=2.0 * S * case["D"])
    if kind == "combine_grads":
        return dict(bytes=2 * size * S * case["D"] + 2.0 * T * case["D"] + 12.0 * S, flops=3.0 * S * case["D"])
    E, N, K = case["E"], case["N"], case["K"]
    rows = T if case["gather"] else S
    if kind == "experts":
        return dict(bytes=2.0 * rows * K + 0.53125 * min(E, S) * N * K + size * S * N + 4.0 * S, flops=2.0 * S * N * K)
    return dict(bytes=2.0 * rows * K + 2.0 * S * N + size * E * N * K + 4.0 * S, flops=2.0 * S * N * K)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _fp4_64(x):
    """Nearest E2M1 multiple of the block's scale: the step is a half below 2, 1 below 4, 2 above, at most 6."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(torch.where(amax > 0, amax, 1.0))) - 2)
    y = b / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (torch.clamp(torch.round(y / step) * step, -6, 6) * scale).flatten(-2)


def _fp8_64(x):
    """Three bits behind the leading one, none finer than 2^-9, under the smallest power of two that keeps the block within 448."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    amax = b.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / 448)))
    y = b / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(y / step) * step * scale).flatten(-2)


def exact(case, seed):
    kind = case["kind"]
    if kind in ("experts", "experts_wgrad") and 2.0 * case["T"] * case["k"] * case["N"] * case["K"] > 1e13:
        return None
    s = prepare(case, seed)
    if kind == "route":
        x = s["logits"].double()
        live = torch.isfinite(x)
        if s["valid"] is not None:
            live &= s["valid"].bool()[:, None]
        p = torch.sigmoid(x) if case["scores"] == "sigmoid" else x
        rank = (p + s["bias"].double() if s["bias"] is not None else p).masked_fill(~live, -math.inf)
        T, E, G = case["T"], case["E"], case["groups"]
        if case["top_groups"] < G:
            high = rank.view(T, G, -1).sort(2, descending=True).values
            high = high[..., 0] + (high[..., 1].clamp(min=-1e300).where(high[..., 1] > -math.inf, torch.zeros_like(high[..., 1]))
                                   if case["scores"] == "sigmoid" and E // G > 1 else 0)
            line = high.sort(dim=1, descending=True, stable=True).indices[:, case["top_groups"]:]
            out = torch.zeros((T, G), dtype=torch.bool, device="cuda").scatter_(1, line, True)
            rank = rank.masked_fill(out.repeat_interleave(E // G, 1), -math.inf)
        best = rank.sort(dim=1, descending=True, stable=True)
        order, none = best.indices[:, :case["k"]], best.values[:, :case["k"]] == -math.inf
        if case["scores"] == "softmax":
            over = x.masked_fill(~live, -math.inf)
            if case["renorm"]:
                over = torch.full_like(x, -math.inf).scatter(1, order, x.gather(1, order).masked_fill(none, -math.inf))
            w = torch.softmax(over, 1).gather(1, order).masked_fill(none, 0)
        else:
            w = p.gather(1, order).masked_fill(none, 0)
            if case["renorm"]:
                w = (w / w.sum(1, keepdim=True)).nan_to_num(0.0)
        return None, w, None, None, None
    if kind == "route_grads":
        x = s["logits"].double().requires_grad_(True)
        got = s["idx"] >= 0
        p = torch.sigmoid(x) if case["scores"] == "sigmoid" else torch.softmax(x, 1)
        w = p.gather(1, s["idx"].long().clamp(min=0)) * got
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
        return torch.autograd.grad((w * s["dw"].double()).sum(), x)[0]
    if kind == "checkpoint":
        return _fp8_64(s["a"])
    if kind == "activation":
        g, u = s["gu"].double().chunk(2, 1)
        act = torch.nn.functional.silu(g) * u
        z = _fp8_64(s["gu"]).requires_grad_(True)
        again = torch.nn.functional.silu(z[:, :case["F"]]) * z[:, case["F"]:]
        return act, torch.autograd.grad(again, z, s["dact"].double())[0], again.detach()
    offsets, token, slot = (t.long() for t in s["plan"])
    if kind == "combine":
        return torch.einsum("tkd,tk->td", s["rows"].double()[slot], s["weights"].double())
    if kind == "combine_grads":
        T, k = slot.shape
        place = torch.empty(T * k, dtype=torch.long, device="cuda")
        place[slot.flatten()] = torch.arange(T * k, device="cuda")          # the choice that a slot serves
        drows = s["dy"].double()[place // k] * s["weights"].double().flatten()[place, None]
        return drows, torch.einsum("tkd,td->tk", s["rows"].double()[slot], s["dy"].double())
    ends = offsets.tolist()
    E, N = case["E"], case["N"]
    x = s["x"][token] if case["gather"] else s["x"]
    out = []
    if kind == "experts":
        x = _fp4_64(x)
        for e in range(E):                       # the weights as the codes stand for them
            if ends[e] < ends[e + 1]:
                codes, scales = s["codes"][e * N:(e + 1) * N].long(), s["scales"][e * N:(e + 1) * N]
                w = torch.stack((codes % 16, codes // 16), 2).flatten(1)
                w = torch.where(w < 8, 1.0, -1.0).double() * torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], device="cuda").double()[w % 8] / 2
                w = w * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)
                out.append(x[ends[e]:ends[e + 1]] @ w.t())
        return torch.cat(out)
    for e in range(E):
        g, h = s["g"][ends[e]:ends[e + 1]], x[ends[e]:ends[e + 1]]
        more = -g.shape[0] % BLOCK
        g, h = (torch.cat((t.double(), t.new_zeros((more, t.shape[1])).double())) for t in (g, h))
        if g.shape[0] == 0:
            out.append(torch.zeros((N, case["K"]), dtype=torch.float64, device="cuda"))
        else:
            out.append(_fp4_64(g.t().contiguous()) @ _fp4_64(h.t().contiguous()).t())
    return torch.cat(out)
