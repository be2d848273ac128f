"""Operators at the end of a pipeline and beside its projections, as measurable calls: the product in 8-bit integers with a scale
for each token and each output channel, the log-probabilities of given logits (with entropy and the likeliest alternatives), and the
log-probabilities of given tokens behind the final norm and the vocabulary projection, whose weights are bf16 or 8-bit integers.

Every case is one call that a serving engine makes.  Where `own` is false, `run` computes it in elementary torch operations;
where it is true, through `paper_2506_10470_amd.tdp`.  Widths are those of the model shapes in the repository's benchmark and tests.

Quantisation, of a row of activations or a column of weights v: with a = max |v| the scale is a / 127 and a code
rint(v * (127 / a)), each of the three operations rounded in fp32 (a vector of zeros has scale 0 and codes 0).  Codes are whole
numbers: everything that is computed from them is a sum of products of integers, times two scales.
"""
import hashlib
import math

import torch

own = False

EPS = 1e-5


def listed():
    return [
        # -- products in 8-bit integers: x bf16 or fp32, quantised in the call; weights hold codes and scales
        # the smallest call: the output projection of a toy stage for one request
        {"name": "linear_m1_256", "kind": "linear", "m": 1, "k": 256, "n": 256, "gated": False, "residual": True, "bias": False, "f32": False},
        # q, k and v side by side for a decode batch, with the biases that some models have
        {"name": "linear_m48_5120_qkv", "kind": "linear", "m": 48, "k": 5120, "n": 7168, "gated": False, "residual": False, "bias": True, "f32": False},
        # widths that are no multiple of any tile, activations and results in fp32
        {"name": "linear_m333_odd_f32", "kind": "linear", "m": 333, "k": 1000, "n": 2044, "gated": False, "residual": False, "bias": True, "f32": True},
        # the gated half of the MLP for the benchmark's decode batch
        {"name": "linear_m512_8192_gated", "kind": "linear", "m": 512, "k": 8192, "n": 57344, "gated": True, "residual": False, "bias": False, "f32": False},
        # the down projection of a batch of packed prompts, on top of the residual stream
        {"name": "linear_m8191_28672_down", "kind": "linear", "m": 8191, "k": 28672, "n": 8192, "gated": False, "residual": True, "bias": False, "f32": False},
        # -- log-probabilities of given logits
        # one request of a toy vocabulary, the five likeliest tokens beside the chosen one
        {"name": "rows_m1_1000_top5", "kind": "rows", "m": 1, "n": 1000, "top": 5, "bf16": False, "masked": False},
        # a decode batch as an API answers it, a quarter of the requests held to a grammar that allows few tokens
        {"name": "rows_m512_32000_top20", "kind": "rows", "m": 512, "n": 32000, "top": 20, "bf16": False, "masked": True},
        # an odd vocabulary, whose rows begin at no multiple of 16 bytes
        {"name": "rows_m257_32003_top1", "kind": "rows", "m": 257, "n": 32003, "top": 1, "bf16": False, "masked": False},
        # every position of packed prompts over a large vocabulary, logits in bf16, no alternatives
        {"name": "rows_m4000_128256_bf16", "kind": "rows", "m": 4000, "n": 128256, "top": 0, "bf16": True, "masked": False},
        # -- log-probabilities of given tokens from hidden states: final norm, vocabulary projection, statistics of every row
        # a few requests: the vocabulary projection is read for three rows
        {"name": "head_m3_5120", "kind": "head", "m": 3, "d": 5120, "n": 32000, "int8": False},
        # the benchmark's decode batch, the projection in 8 bits
        {"name": "head_m512_8192_int8", "kind": "head", "m": 512, "d": 8192, "n": 32000, "int8": True},
        # a batch of prompts is scored: every position's next token
        {"name": "head_m4099_4096", "kind": "head", "m": 4099, "d": 4096, "n": 32000, "int8": False},
    ]


def draw(rng):
    def spread(lo, hi, step=1):  # uniform in the logarithm, a multiple of step
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) / step)) * step
        return min(hi, max(lo, v))

    kind = rng.choice(["linear", "linear", "rows", "rows", "head"])
    if kind == "linear":
        k, n, gated = spread(64, 28672, 8), spread(64, 57344, 8), rng.random() < 0.3
        most = int(min(8191, 3.8e12 / (2.0 * k * n)))
        return {"kind": kind, "m": spread(1, max(1, most)), "k": k, "n": n, "gated": gated, "residual": not gated and rng.random() < 0.4,
                "bias": not gated and rng.random() < 0.3, "f32": rng.random() < 0.25}
    if kind == "rows":
        n, bf16, top = spread(500, 152000), rng.random() < 0.3, rng.choice([0, 1, 5, 20, 32])
        return {"kind": kind, "m": spread(1, int(min(4000, (2.5e8 if top == 0 else 6e7) / n))), "n": n, "top": top, "bf16": bf16,
                "masked": rng.random() < 0.3}
    d, n = spread(64, 8192, 64), spread(1000, 128256, 4)
    return {"kind": kind, "m": spread(1, int(min(4099, 1.07e12 / (2.0 * d * n), 1.3e8 / n))), "d": d, "n": n, "int8": rng.random() < 0.5}


# ---- inputs -----------------------------------------------------------------------------------------------------

def generator(seed, what):
    digest = hashlib.blake2b(repr((int(seed), what)).encode(), digest_size=7).digest()
    return torch.Generator(device="cuda").manual_seed(int.from_bytes(digest, "big"))


def normal(seed, what, shape, std=1.0):
    return torch.randn(shape, generator=generator(seed, what), device="cuda").mul_(std)


def whole(seed, what, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=generator(seed, what), device="cuda", dtype=torch.int32)


def quantised(v, dim):
    """(codes in fp32, scales) of the vectors of v along dim, as the module's comment says; v fp32."""
    a = v.abs().amax(dim, keepdim=True)
    bound = torch.full_like(a, 127.0)
    inverse = torch.where(a > 0, torch.div(bound, a), torch.zeros_like(a))
    return (v * inverse).round_(), torch.div(a, bound).squeeze(dim)


class State:
    """What an engine holds before the call."""


class Handle:
    """An object of the library, given back when nothing refers to it any more."""

    def __init__(self, handle, destroy):
        self.handle, self.destroy = handle, destroy

    def __del__(self):
        self.destroy(self.handle)


def activations(seed, m, k):
    """Rows of a decoder's hidden states: normal, with one channel in a hundred ten times as large and rows of different size."""
    x = normal(seed, "x", (m, k))
    x[:, whole(seed, "large", 0, k, (max(1, k // 100),)).long()] *= 10.0
    return x * torch.exp(normal(seed, "rows", (m, 1), 0.5))


def prepare(case, seed):
    S = State()
    S.kind, S.m, S.n = case["kind"], case["m"], case["n"]
    if S.kind == "rows":
        S.top = case["top"]
        S.logits = normal(seed, "logits", (S.m, S.n), 2.5)
        S.logits[:, whole(seed, "likely", 0, S.n, (8,)).long()] += 8.0
        if case["masked"]:  # every fourth row may answer with at most 24 tokens
            allowed = whole(seed, "allowed", 0, S.n, ((S.m + 3) // 4, 24)).long()
            keep = torch.zeros(allowed.shape[0], S.n, dtype=torch.bool, device="cuda").scatter_(1, allowed, True)
            S.logits[::4].masked_fill_(~keep, -math.inf)
        S.targets = whole(seed, "targets", 0, S.n, (S.m,))
        if S.m > 1:
            S.targets[-1] = -1  # nothing follows the last position
        if case["bf16"]:
            S.logits = S.logits.to(torch.bfloat16)
    elif S.kind == "linear":
        S.k, S.gated, S.f32 = case["k"], case["gated"], case["f32"]
        S.x = activations(seed, S.m, S.k).to(torch.float32 if S.f32 else torch.bfloat16)
        codes, S.w_scales = quantised(normal(seed, "weights", (S.k, S.n), 0.02), 0)
        S.codes = codes.to(torch.int8)
        S.cols = S.n // 2 if S.gated else S.n
        S.bias = normal(seed, "bias", (S.n,), 0.5) if case["bias"] else None
        S.residual = normal(seed, "residual", (S.m, S.n)).to(S.x.dtype) if case["residual"] else None
    else:
        S.d, S.int8 = case["d"], case["int8"]
        S.x = activations(seed, S.m, S.d).to(torch.bfloat16)
        S.gain = normal(seed, "gain", (S.d,), 0.02) + 1.0
        S.weights = normal(seed, "head", (S.d, S.n), 0.02).to(torch.bfloat16)
        S.targets = whole(seed, "targets", 0, S.n, (S.m,))
        if S.m > 1:
            S.targets[-1] = -1
        if S.int8:
            codes, S.w_scales = quantised(S.weights.float(), 0)
            S.codes = codes.to(torch.int8)
    if own:
        prepare_own(S)
    return S


def prepare_own(S):
    from paper_2506_10470_amd import tdp
    S.tdp = tdp
    if S.kind == "linear":
        S.owner = Handle(tdp.tdp_linear_i8_create(tdp.LinearI8Config(S.k, S.n, int(S.gated), S.m)), tdp.tdp_linear_i8_destroy)
        tdp.tdp_linear_i8_set_codes(S.owner.handle, S.codes, S.w_scales, tdp.DEVICE, S.k, S.n)
        if S.bias is not None:
            tdp.tdp_linear_i8_set_bias(S.owner.handle, S.bias, tdp.F32, tdp.DEVICE, S.n)
        S.out = torch.empty((S.m, S.cols), dtype=S.x.dtype, device="cuda")
        return
    S.logprob = torch.empty(S.m, device="cuda")
    S.entropy = torch.empty(S.m, device="cuda")
    if S.kind == "rows":
        S.index = torch.empty((S.m, S.top), dtype=torch.int32, device="cuda") if S.top else None
        S.top_logprob = torch.empty((S.m, S.top), device="cuda") if S.top else None
        return
    S.owner = Handle(tdp.tdp_ends_create(tdp.EndsConfig(S.n, S.d, EPS, S.m)), tdp.tdp_ends_destroy)
    tdp.tdp_ends_set_weight(S.owner.handle, tdp.E_FINAL_NORM, S.gain, tdp.F32, tdp.DEVICE, S.d, 1)
    tdp.tdp_ends_set_weight(S.owner.handle, tdp.E_LM_HEAD_I8 if S.int8 else tdp.E_LM_HEAD, S.weights, tdp.BF16, tdp.DEVICE, S.d, S.n)


# ---- the calls --------------------------------------------------------------------------------------------------

def run(S):
    if own:
        return run_own(S)
    return {"linear": plain_linear, "rows": plain_rows, "head": plain_head}[S.kind](S)


def run_own(S):
    tdp = S.tdp
    if S.kind == "linear":
        kind = tdp.F32 if S.f32 else tdp.BF16
        tdp.tdp_linear_i8_run(S.owner.handle, S.x, kind, S.k, S.m, S.residual, S.n, S.out, kind, S.cols)
        return S.out
    if S.kind == "rows":
        tdp.tdp_logprob_rows(S.logits, tdp.F32 if S.logits.dtype == torch.float32 else tdp.BF16, S.m, S.n, S.n, S.targets, S.top, S.logprob,
                             S.entropy, S.index, S.top_logprob)
        return answer(S.logprob, S.entropy, S.index, S.top_logprob)
    tdp.tdp_lm_head_logprobs(S.owner.handle, S.x, S.m, None, S.m, S.targets, 0, None, S.logprob, S.entropy, None, None)
    return answer(S.logprob, S.entropy)


def answer(logprob, entropy, index=None, top_logprob=None):
    return {"logprob": logprob, "entropy": entropy, **({"top_index": index, "top_logprob": top_logprob} if index is not None else {})}


def plain_linear(S):
    codes, scales = quantised(S.x.float(), 1)
    y = (codes @ S.codes.float()) * scales[:, None] * S.w_scales
    if S.bias is not None:
        y = y + S.bias
    if S.residual is not None:
        y = y + S.residual.float()
    if S.gated:
        gate, up = y[:, :S.cols], y[:, S.cols:]
        y = gate / (1 + torch.exp(-gate)) * up
    return y.to(S.x.dtype)


def statistics(z, targets):
    """(largest logit, log of the sum of exp(z - largest), log-probability of the targets, entropy), of every row; -1 is no token."""
    top = z.amax(1, keepdim=True)
    shifted = z - top
    e = torch.exp(shifted)
    total = e.sum(1)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * shifted, 0.0).sum(1) / total
    of_target = shifted.gather(1, targets.clamp(min=0).long()[:, None])[:, 0] - log_total
    return top[:, 0], log_total, torch.where(targets >= 0, of_target, -math.inf), entropy


def plain_rows(S):
    z = S.logits.float()
    largest, log_total, logprob, entropy = statistics(z, S.targets)
    if not S.top:
        return answer(logprob, entropy)
    # one whole number orders the tokens: the logit's bits made monotone, then the lower index
    bits = (z + 0.0).view(torch.int32)
    order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() * (1 << 32) + torch.arange(S.n - 1, -1, -1, device="cuda")
    index = order.topk(S.top, 1).indices
    return answer(logprob, entropy, index.int(), z.gather(1, index) - largest[:, None] - log_total[:, None])


def plain_head(S):
    x = S.x.float()
    r = torch.rsqrt((x * x).mean(1) + EPS)
    if S.int8:
        # the factor of the norm is common to a row: it changes its scale and no code
        codes, scales = quantised(x * S.gain, 1)
        z = (codes @ S.codes.float()) * (scales * r)[:, None] * S.w_scales
    else:
        # the norm hands its rows to the projection in bf16, like the norm of any layer
        z = (x * r[:, None] * S.gain).to(torch.bfloat16).float() @ S.weights.float()
    _, _, logprob, entropy = statistics(z, S.targets)
    return answer(logprob, entropy)


# ---- what a pass has to do, and its result in 64 bits -----------------------------------------------------------

def work(case):
    m, n = case["m"], case["n"]
    if case["kind"] == "linear":
        size, k, cols = 4 if case["f32"] else 2, case["k"], n // 2 if case["gated"] else n
        return {"bytes": m * k * size + k * n + 4 * n * (2 if case["bias"] else 1) + m * cols * size * (2 if case["residual"] else 1),
                "flops": 2.0 * m * k * n}
    if case["kind"] == "rows":
        return {"bytes": m * n * (2 if case["bf16"] else 4) + m * (12 + 8 * case["top"]), "flops": 6.0 * m * n}
    d = case["d"]
    return {"bytes": m * d * 2 + d * n * (1 if case["int8"] else 2) + 4 * d + (4 * n if case["int8"] else 0) + 12 * m,
            "flops": 2.0 * m * d * n + 6.0 * m * n}


def exact(case, seed):
    S = prepare({**case}, seed)
    if S.kind == "linear":
        codes, scales = codes_of(S.x)
        y = torch.mm(codes, S.codes.double()) * (scales.unsqueeze(1) * S.w_scales.double().unsqueeze(0))
        if S.bias is not None:
            y += S.bias.double()
        if S.residual is not None:
            y += S.residual.double()
        if S.gated:
            y = torch.sigmoid(y[:, :S.cols]).mul_(y[:, :S.cols]).mul_(y[:, S.cols:])
        return y
    if S.kind == "rows":
        z, top = S.logits.double(), S.top
    else:
        x, top = S.x.double(), 0
        r = x.square().mean(1, keepdim=True).add(EPS).rsqrt()
        if S.int8:
            codes, scales = codes_of(S.x.float() * S.gain)
            z = torch.mm(codes, S.codes.double()) * (scales.unsqueeze(1) * r * S.w_scales.double())
        else:
            z = torch.mm((x * r * S.gain.double()).to(torch.bfloat16).double(), S.weights.double())
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    entropy = -torch.xlogy(p, p).sum(1)
    chosen = z[torch.arange(S.m, device="cuda"), S.targets.long() % S.n] - lse
    chosen[S.targets < 0] = -math.inf
    return {"logprob": chosen, "entropy": entropy,
            **({"top_index": None, "top_logprob": z.sort(1, descending=True).values[:, :top] - lse[:, None]} if top else {})}


def codes_of(v):
    """The codes of rows, whole numbers by the rule in fp32, in 64 bits; the scales are exact."""
    v = v.float()
    largest = v.abs().max(1).values
    factor = torch.ones_like(largest).mul_(127).div_(largest.clamp(min=torch.finfo(torch.float32).tiny))
    return torch.round(v * factor[:, None]).double(), largest.double() / 127
