"""The learner's operators beside the rollout, case by case: what is computed, in plain form and through the library.

A learner that consumes rollouts scores them (the log-probability of every taken token, with the entropy of its
distribution and the most probable alternatives), forms the objective and its gradient per token, carries that
gradient back to the logits, and updates the weights that the next snapshot is made of.

  token_logprobs            logits [R][V], tokens [R] -> log-probability, entropy, row statistics, top alternatives
  token_logprobs_backward   the gradient of log-probabilities and entropies with respect to the logits
  grpo_gradient             the clipped objective per sequence and its gradient with respect to logp_new
  adamw                     one AdamW step over many tensors, first and second moments in 32 or in 8 bits

`own` False: elementary torch operations; True: the calls of paper_2602_02192_b200.binding.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 256                     # elements that share the two scales of 8-bit moments
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 3e-5, 0.1


# ---- cases ------------------------------------------------------------------------------------
def _logits_case(name, op, R, V, dtype, temperature=1.0, top_k=0, pad=0, drop=0.0, empty=0, entropy=True, offset=0):
    return {"name": name, "op": op, "R": R, "V": V, "dtype": dtype, "temperature": temperature, "top_k": top_k,
            "pad": pad, "drop": drop, "empty": empty, "entropy": entropy, "offset": offset}


def _grpo_case(name, n, T, mask, kl):
    return {"name": name, "op": "grpo_gradient", "n": n, "T": T, "mask": mask, "kl": kl}


def _adamw_case(name, bits, grad, copy, sizes, plain=0):
    return {"name": name, "op": "adamw", "bits": bits, "grad": grad, "copy": copy,
            "sizes": " ".join(str(s) for s in sizes), "undecayed": plain}


# matrices of one decoder layer at the 8B shape (d 4096, 32 / 8 heads of 128, F 12288), then its two gains
LAYER_8B = [4096 * 4096, 1024 * 4096, 1024 * 4096, 4096 * 4096, 12288 * 4096, 12288 * 4096, 4096 * 12288, 4096, 4096]
# the whole two-layer shape (d 256, 4 / 2 heads of 64, F 688, vocab 4096)
TINY = [4096 * 256, 4096 * 256] + 2 * [256 * 256, 128 * 256, 128 * 256, 256 * 256, 688 * 256, 688 * 256, 256 * 688] + 5 * [256]


def listed():
    return [
        # one token of one served sequence, with the alternatives that a client asks for: latency
        _logits_case("logprobs_one_token", "token_logprobs", 1, 151936, "bf16", top_k=20),
        # one decode step of 32 prompts x 8 samples on the engine's fp32 logits
        _logits_case("logprobs_decode_step", "token_logprobs", 256, 151936, "fp32", top_k=5),
        # a learner's scoring chunk; a tenth of the rows is prompt or padding (no token)
        _logits_case("logprobs_chunk", "token_logprobs", 2048, 151936, "bf16", top_k=0, drop=0.1),
        # an odd vocabulary in padded rows, ids that a grammar or the padding masks, rows with nothing left
        _logits_case("logprobs_odd_masked", "token_logprobs", 777, 50263, "fp16", temperature=0.7, top_k=8, pad=41, drop=0.2,
                empty=3, offset=1),
        # the same chunk's gradient, with an entropy bonus
        _logits_case("backward_chunk", "token_logprobs_backward", 2048, 151936, "bf16", drop=0.1),
        # a small model's batch in fp32, log-probabilities alone
        _logits_case("backward_small", "token_logprobs_backward", 512, 4096, "fp32", temperature=0.9, drop=0.3, entropy=False),
        # 16 short responses: latency
        _grpo_case("grpo_short", 16, 32, mask=False, kl=True),
        # 32 prompts x 8 samples x 2048 tokens, responses that end at different lengths
        _grpo_case("grpo_batch", 256, 2048, mask=True, kl=True),
        # every tensor of the two-layer shape, 32-bit moments: many small tensors, latency
        _adamw_case("adamw32_small_model", 32, "fp32", False, TINY, plain=5),
        # one layer of the 8B shape: fp32 weights, bf16 gradients, and the bf16 copy that the next snapshot is made of
        _adamw_case("adamw32_layer", 32, "bf16", True, LAYER_8B, plain=2),
        # the same with 8-bit moments
        _adamw_case("adamw8_layer", 8, "bf16", True, LAYER_8B, plain=2),
        # odd sizes, single elements among them, 8-bit moments
        _adamw_case("adamw8_odd", 8, "fp32", False, [1000003, 257, 1, 77777, 255, 256, 500009, 3, 12345], plain=3),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["token_logprobs", "token_logprobs", "token_logprobs_backward", "grpo_gradient", "adamw", "adamw"])
    if op in ("token_logprobs", "token_logprobs_backward"):
        V = _spread(rng, 64, 160000)
        R = _spread(rng, 1, min(4096, 2048 * 151936 // V // 2))
        c = _logits_case("", op, R, V, rng.choice(list(DTYPES)), temperature=rng.choice([1.0, 0.6, 0.85, 1.3]),
                    pad=rng.choice([0, 0, 1, 8, 37]), drop=rng.choice([0.0, 0.1, 0.5]),
                    empty=rng.choice([0, 0, 1, 2]), offset=rng.choice([0, 0, 1, 3]))
        if op == "token_logprobs":
            c["top_k"] = rng.choice([0, 0, 1, 5, 20, 32])
        else:
            c["entropy"] = rng.random() < 0.5
    elif op == "grpo_gradient":
        n = _spread(rng, 1, 512)
        c = _grpo_case("", n, _spread(rng, 1, min(8192, 524288 // n)), mask=rng.random() < 0.7, kl=rng.random() < 0.5)
    else:
        total, sizes = _spread(rng, 64, 100_000_000), []
        count = _spread(rng, 1, 24)
        for _ in range(count):
            sizes.append(_spread(rng, 1, max(1, total // count)))
        c = _adamw_case("", rng.choice([32, 8]), rng.choice(list(DTYPES)), rng.random() < 0.5, sizes, plain=rng.randint(0, count))
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 11)
    return g


def _normal(g, *shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda").mul_(std)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _prepare_logits(case, seed):
    """Logits with a handful of likely ids a row, in rows of `pad` further ids that are never read; the last ids of
    the vocabulary are masked (-inf in even rows, the type's lowest value in odd ones) where the rows are padded."""
    g, R, V, dtype = _gen(seed), case["R"], case["V"], DTYPES[case["dtype"]]
    ld = V + case["pad"]
    store = torch.empty(R * ld + case["offset"], dtype=dtype, device="cuda")
    z = store[case["offset"]:].view(R, ld)
    z.normal_(0.0, 2.0, generator=g)
    masked = min(V // 4, case["pad"])
    likely = torch.randint(0, V - masked, (R, 8), generator=g, device="cuda")
    z.scatter_add_(1, likely, (_uniform(g, R, 8) * 14).to(dtype))
    logits = z[:, :V]
    if masked:
        logits[0::2, V - masked:] = -math.inf
        logits[1::2, V - masked:] = torch.finfo(dtype).min
    if case["empty"]:
        logits[torch.randint(0, R, (case["empty"],), generator=g, device="cuda")] = -math.inf
    tokens = torch.randint(0, V - masked, (R,), generator=g, device="cuda", dtype=torch.int32)
    tokens = torch.where(_uniform(g, R) < 0.7, likely[:, 0].to(torch.int32), tokens)        # most are likely ones
    tokens[_uniform(g, R) < case["drop"]] = -1
    s = {"case": case, "logits": logits, "tokens": tokens, "temperature": case["temperature"]}
    if case["op"] == "token_logprobs_backward":      # what the forward call left
        out = _token_logprobs(logits, tokens, case["temperature"], 0)
        s["entropy"], s["stats"] = out["entropy"], out["stats"]
        s["grad_logprobs"] = _normal(g, R, std=1.0 / R)
        s["grad_entropy"] = _normal(g, R, std=0.01 / R) if case["entropy"] else None
    return s


def _prepare_grpo(case, seed):
    g, n, T = _gen(seed), case["n"], case["T"]
    logp = -4.0 * _uniform(g, n, T) ** 4
    s = {"case": case, "new": logp + _normal(g, n, T, std=0.15), "old": logp,
         "sampler": logp + _normal(g, n, T, std=0.05),
         "ref": logp + _normal(g, n, T, std=0.3) if case["kl"] else None,
         "adv": _normal(g, n), "grad_out": _uniform(g, n) / n, "mask": None}
    if case["mask"]:
        ends = torch.randint(0, T + 1, (n, 1), generator=g, device="cuda")       # some responses are empty
        s["mask"] = (torch.arange(T, device="cuda")[None, :] < ends).to(torch.uint8)
    return s


def _prepare_adamw(case, seed):
    """Tensors in one flat buffer of each kind, every one starting on a multiple of BLOCK."""
    g, sizes = _gen(seed), [int(x) for x in case["sizes"].split()]
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    kept = torch.zeros(at, dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        kept[a:a + n] = True
    decayed = starts[len(sizes) - case["undecayed"]] if case["undecayed"] else at
    s = {"case": case, "sizes": sizes, "starts": starts, "decayed": decayed, "step": 7, "seed": 1000 + int(seed),
         "p": _normal(g, at, std=0.02) * kept,
         "g": (_normal(g, at, std=1e-3) * kept).to(DTYPES[case["grad"]]),
         "grad_scale": torch.full((1,), 0.83, device="cuda"),
         "copy": torch.zeros(at, dtype=torch.bfloat16, device="cuda") if case["copy"] else None}
    if case["bits"] == 32:
        s["m"] = _normal(g, at, std=3e-4) * kept
        s["v"] = (_normal(g, at, std=1e-3) ** 2 + 1e-12) * kept
    else:
        s["m"] = (_normal(g, at, std=40.0).clamp_(-127, 127) * kept).round_().to(torch.int8)
        s["v"] = ((1 + 254 * _uniform(g, at)) * kept).to(torch.uint8)
        s["scales"] = torch.stack([1e-3 * (0.5 + _uniform(g, at // BLOCK)), 4e-6 * (0.5 + _uniform(g, at // BLOCK))])
        s["values"] = (torch.zeros(at, device="cuda"), torch.zeros(at, device="cuda"))
    # the plan a program keeps: pieces of the buffers, one of each kind for every tensor
    cut = lambda x, unit=1: [x[a // unit:a // unit + -(-n // unit)] for a, n in zip(starts, sizes)]  # noqa: E731
    s["pieces"] = {"params": cut(s["p"]), "grads": cut(s["g"]), "exp_avg": cut(s["m"]), "exp_avg_sq": cut(s["v"]),
                   "copies": cut(s["copy"]) if case["copy"] else None,
                   "weight_decay": [DECAY if a < decayed else 0.0 for a in starts]}
    if case["bits"] == 8:
        s["pieces"]["avg_scales"] = cut(s["scales"][0], BLOCK)
        s["pieces"]["sq_scales"] = cut(s["scales"][1], BLOCK)
        s["values_cut"] = (cut(s["values"][0]), cut(s["values"][1]))
    if own:          # the handle that holds the pieces' addresses, made once like the buffers
        from paper_2602_02192_b200 import binding
        s["plan"] = binding.AdamWTensors(**s["pieces"])
    return s


def prepare(case, seed):
    if case["op"] == "grpo_gradient":
        return _prepare_grpo(case, seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, seed)
    return _prepare_logits(case, seed)


# ---- plain forms ------------------------------------------------------------------------------
def _token_logprobs(logits, tokens, temperature, top_k):
    z = logits.float()
    zmax = z.amax(dim=1)
    base = torch.where(torch.isneginf(zmax), torch.zeros_like(zmax), zmax)
    s = (z - base[:, None]) / temperature
    e = torch.exp(s)
    total = e.sum(dim=1)
    logsum = torch.log(total)
    empty = total == 0
    weighted = torch.where(e > 0, e * s, torch.zeros_like(s)).sum(dim=1)
    entropy = torch.where(empty, torch.zeros_like(total), logsum - weighted / total)
    at = tokens.clamp(min=0).long()
    taken = torch.gather(s, 1, at[:, None])[:, 0] - logsum
    taken = torch.where(empty, torch.full_like(taken, -math.inf), taken)
    out = {"logprobs": torch.where(tokens < 0, torch.zeros_like(taken), taken), "entropy": entropy,
           "stats": torch.stack([zmax, logsum], dim=1)}
    if top_k:
        # largest logits first, equal ones by id: one whole number per entry that orders both
        bits = (z + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -2147483648 - bits - 1, bits) * (1 << 31) + (2147483647 - torch.arange(z.shape[1], device=z.device))
        k = min(top_k, z.shape[1])
        best = torch.topk(key, k, dim=1).values
        ids = 2147483647 - (best & 2147483647)
        lp = torch.gather(s, 1, ids) - logsum[:, None]
        none = torch.isneginf(torch.gather(z, 1, ids))
        ids, lp = torch.where(none, -torch.ones_like(ids), ids), torch.where(none, torch.full_like(lp, -math.inf), lp)
        fill = top_k - k
        out["top_ids"] = torch.nn.functional.pad(ids, (0, fill), value=-1).to(torch.int32)
        out["top_logprobs"] = torch.nn.functional.pad(lp, (0, fill), value=-math.inf)
    return out


def _token_logprobs_backward(logits, tokens, entropy, stats, grad_logprobs, grad_entropy, temperature):
    z = logits.float()
    zmax, logsum = stats[:, 0], stats[:, 1]
    empty = torch.isneginf(zmax)
    lp = (z - torch.where(empty, torch.zeros_like(zmax), zmax)[:, None]) / temperature
    lp -= torch.where(empty, torch.zeros_like(zmax), logsum)[:, None]
    p = torch.exp(lp)
    a = torch.where(tokens < 0, torch.zeros_like(grad_logprobs), grad_logprobs)
    d = -a[:, None] * p
    if grad_entropy is not None:
        d -= grad_entropy[:, None] * torch.where(p > 0, p * (lp + entropy[:, None]), torch.zeros_like(p))
    d.scatter_add_(1, tokens.clamp(min=0).long()[:, None], a[:, None])
    d = d / temperature
    return torch.where(empty[:, None], torch.zeros_like(d), d).to(logits.dtype)


def _grpo_gradient(s, eps_clip, C, beta):
    new, old, sampler = s["new"], s["old"], s["sampler"]
    m = torch.ones_like(new) if s["mask"] is None else (s["mask"] != 0).float()
    a = s["adv"][:, None]
    x = new.double() - old.double()                 # next to the clipping borders in 64 bits
    rho = torch.exp(new - old)
    w = torch.exp(old - sampler).clamp(max=C)
    term = torch.minimum(rho * a, rho.clamp(1 - eps_clip, 1 + eps_clip) * a)
    eps = float(np.float32(eps_clip))
    dead = torch.where(a > 0, x > math.log1p(eps), x < math.log1p(-eps))
    slope = torch.where(dead, torch.zeros_like(rho), rho * a)
    if s["ref"] is not None:
        d = s["ref"] - new
        term = term - beta * (torch.expm1(d) - d)
        slope = slope + beta * torch.expm1(d)
    count = m.sum(dim=1)
    share = torch.where(count > 0, 1.0 / count.clamp(min=1), torch.zeros_like(count))
    zero = torch.zeros_like(rho)
    return {"objective": torch.where(m > 0, w * term, zero).sum(dim=1) * share,
            "grad": torch.where(m > 0, w * slope, zero) * (s["grad_out"] * share)[:, None]}


def _halves(first, second, tensor, step, seed):
    """Philox4x32-10 words of counter (octet low, octet high, tensor, step) as eight 16-bit numbers per octet."""
    low = 0xFFFFFFFF
    c = [first, second, tensor, torch.full_like(first, step)]
    k0, k1 = seed & low, (seed >> 32) & low

    def product(const, x):
        part = const * (x & 0xFFFF)
        top = const * (x >> 16) + (part >> 16)
        return top >> 16, ((top & 0xFFFF) << 16) | (part & 0xFFFF)

    for _ in range(10):
        h0, l0 = product(0xD2511F53, c[0])
        h1, l1 = product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    w = torch.stack(c, dim=1)
    return torch.stack([w & 0xFFFF, w >> 16], dim=2).reshape(-1)


def _adamw(s):
    case, step = s["case"], s["step"]
    bits8 = case["bits"] == 8
    f = (lambda x: x) if bits8 else (lambda x: float(np.float32(x)))     # 8 bits: 64-bit moments, next to code borders
    m, v, grad = s["m"], s["v"], s["g"].float()
    scale = s["grad_scale"]
    if bits8:
        m_scale, v_scale = s["scales"]
        m, v = _codes_to_avg(m, m_scale.double()), _codes_to_sq(v, v_scale.double())
        grad, scale = grad.double(), scale.double()
    grad = grad * scale
    m = m * f(BETA1) + grad * f(1 - BETA1)
    v = v * f(BETA2) + (grad * f(1 - BETA2)) * grad
    update = m / (torch.sqrt(v) * f(1 / math.sqrt(1 - BETA2 ** step)) + f(EPS))
    p, cut = s["p"], s["decayed"]
    new = p.to(update.dtype)
    new = torch.cat([new[:cut] * f(1 - LR * DECAY), new[cut:]]) - update * f(LR / (1 - BETA1 ** step))
    p.copy_(new)
    out = {"params": p}
    if s["copy"] is not None:
        s["copy"].copy_(p)
        out["copy"] = s["copy"]
    if not bits8:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {**out, "exp_avg": s["m"], "exp_avg_sq": s["v"]}
    # first moment: |code| = nearest to 127 sqrt(|m| / M), M the block's largest as fp32
    mb, vb = m.view(-1, BLOCK), v.view(-1, BLOCK)
    top, inv = _block_scale(mb.abs().amax(dim=1))
    m_scale.copy_(top)
    code = torch.round(torch.sqrt(mb.abs() * inv) * 127.0)
    s["m"].copy_((code * torch.sign(mb)).view(-1))
    # second moment: code c stands for V (c / 255)^4, V the block's largest as fp32; one of the two codes around v, the
    # upper with the probability that keeps the mean, and never 0 for a v above 0
    top, inv = _block_scale(vb.amax(dim=1))
    v_scale.copy_(top)
    ratio = vb * inv
    low = torch.floor(torch.sqrt(torch.sqrt(ratio)) * 255.0).clamp(max=254.0)
    under, over = (low / 255) ** 4, ((low + 1) / 255) ** 4
    # random numbers: octets of a tensor count from its own start
    octets = torch.tensor([-(-n // BLOCK) for n in s["sizes"]], device=m.device) * (BLOCK // 8)
    total = mb.shape[0] * (BLOCK // 8)
    tensor = torch.repeat_interleave(torch.arange(len(s["sizes"]), device=m.device), octets, output_size=total)
    first = torch.arange(total, device=m.device) - (torch.cumsum(octets, 0) - octets)[tensor]
    u = _halves(first & 0xFFFFFFFF, first >> 32, tensor, step, s["seed"]).double().mul_(2.0 ** -16).view(-1, BLOCK)
    code = low + (u * (over - under) < ratio - under).double()
    code = torch.where(ratio > 0, code.clamp(min=1.0), torch.zeros_like(code))
    s["v"].copy_(code.view(-1))
    s["values"][0].copy_(_codes_to_avg(s["m"], m_scale.double()))
    s["values"][1].copy_(_codes_to_sq(s["v"], v_scale.double()))
    return {**out, "exp_avg": s["values"][0], "exp_avg_sq": s["values"][1]}


def _block_scale(largest):
    """The scale that is kept for a block, fp32, and one over it; a largest value under the normal numbers counts as 0."""
    top = largest.float()
    top = torch.where(top < 2.0 ** -126, torch.zeros_like(top), top)
    return top, torch.where(top > 0, 1.0 / top.double(), torch.zeros_like(largest))[:, None]


def _codes_to_avg(code, scale):
    q = code.view(-1, BLOCK).to(scale.dtype) / 127
    return (q * q.abs() * scale[:, None]).view(-1)


def _codes_to_sq(code, scale):
    q = code.view(-1, BLOCK).to(scale.dtype) / 255
    return (q ** 4 * scale[:, None]).view(-1)


# ---- one pass ---------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        from paper_2602_02192_b200 import binding as B
        if case["op"] == "token_logprobs":
            lp, entropy, stats, ids, top = B.echo_token_logprobs(state["logits"], state["tokens"], state["temperature"],
                                                                 case["top_k"])
            out = {"logprobs": lp, "entropy": entropy, "stats": stats}
            return {**out, "top_ids": ids, "top_logprobs": top} if case["top_k"] else out
        if case["op"] == "token_logprobs_backward":
            return B.echo_token_logprobs_backward(state["logits"], state["tokens"], state["entropy"], state["stats"],
                                                  state["grad_logprobs"], state["grad_entropy"], state["temperature"])
        if case["op"] == "grpo_gradient":
            value, grad = B.echo_grpo_gradient(state["new"], state["old"], state["sampler"], state["ref"], state["adv"],
                                               state["mask"], state["grad_out"], 0.2, 2.0, 0.04)
            return {"objective": value, "grad": grad}
        B.echo_adamw_step(state["plan"], state["step"], LR, BETA1, BETA2, EPS, grad_scale=state["grad_scale"],
                          seed=state["seed"])
        out = {"params": state["p"]}
        if state["copy"] is not None:
            out["copy"] = state["copy"]
        if case["bits"] == 32:
            return {**out, "exp_avg": state["m"], "exp_avg_sq": state["v"]}
        B.echo_adamw_unpack(state["plan"], *state["values_cut"])
        return {**out, "exp_avg": state["values"][0], "exp_avg_sq": state["values"][1]}
    if case["op"] == "token_logprobs":
        return _token_logprobs(state["logits"], state["tokens"], state["temperature"], case["top_k"])
    if case["op"] == "token_logprobs_backward":
        return _token_logprobs_backward(state["logits"], state["tokens"], state["entropy"], state["stats"],
                                        state["grad_logprobs"], state["grad_entropy"], state["temperature"])
    if case["op"] == "grpo_gradient":
        return _grpo_gradient(state, 0.2, 2.0, 0.04)
    return _adamw(state)


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    if case["op"] == "grpo_gradient":
        n = case["n"] * case["T"]
        arrays = 5 + (1 if case["kl"] else 0)            # three or four inputs, the gradient, and one byte of mask
        return {"bytes": n * (4 * (arrays - 1) + (1 if case["mask"] else 0)) + 12 * case["n"], "flops": 12 * n}
    if case["op"] == "adamw":
        n = sum(int(x) for x in case["sizes"].split())
        width = 4 if case["grad"] == "fp32" else 2
        moments = 16 if case["bits"] == 32 else 4 + 8    # 8 bits: codes in and out, and the values they stand for
        return {"bytes": n * (8 + width + moments + (2 if case["copy"] else 0)), "flops": 14 * n}
    R, V = case["R"], case["V"]
    width = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "token_logprobs":
        return {"bytes": R * V * width + R * (20 + 8 * case["top_k"]), "flops": 5 * R * V}
    read = 1.0 if case["entropy"] else 1.0 - case["drop"]      # a row without a gradient is written, not read
    return {"bytes": int((1 + read) * R * V * width) + R * 24, "flops": 6 * R * V}


# ---- the definitions in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "adamw":
        return _exact_adamw(case, seed)
    s = prepare(case, seed)
    if case["op"] == "grpo_gradient":
        return _exact_grpo(s)
    R, V, temp = case["R"], case["V"], float(np.float32(case["temperature"]))
    backward = case["op"] == "token_logprobs_backward"
    got = []
    rows = max(1, (1 << 26) // V)
    for a in range(0, R, rows):
        b = min(R, a + rows)
        z, y = s["logits"][a:b].to(torch.float64) / temp, s["tokens"][a:b].long()
        none = torch.isneginf(z).all(dim=1)
        z = z.masked_fill(none[:, None], 0.0)
        logp = z - torch.logsumexp(z, dim=1, keepdim=True)
        p = logp.exp()
        entropy = -(torch.special.xlogy(p, p).sum(dim=1)).masked_fill(none, 0.0)
        hot = y >= 0
        if backward:
            ga = s["grad_logprobs"][a:b].to(torch.float64) * hot
            dz = -ga[:, None] * p
            at = torch.nonzero(hot)[:, 0]
            dz[at, y[at]] += ga[at]
            if case["entropy"]:
                ge = s["grad_entropy"][a:b].to(torch.float64)
                dz -= ge[:, None] * (torch.special.xlogy(p, p) + p * entropy[:, None])
            got.append((dz / temp).masked_fill(none[:, None], 0.0).to(torch.float32 if R * V > 1 << 28 else torch.float64))
            continue
        lp = logp.gather(1, y.clamp(min=0)[:, None])[:, 0].masked_fill(none, -math.inf).masked_fill(~hot, 0.0)
        zmax = s["logits"][a:b].to(torch.float64).amax(dim=1)
        logsum = (torch.logsumexp(z, dim=1) - zmax / temp).masked_fill(none, -math.inf)
        top = None
        if case["top_k"]:
            k = min(case["top_k"], V)
            top = logp.masked_fill(none[:, None], -math.inf).sort(dim=1, descending=True).values[:, :k]
            top = torch.nn.functional.pad(top, (0, case["top_k"] - k), value=-math.inf)
        got.append((lp, entropy, torch.stack([zmax, logsum], dim=1), top))
    if backward:
        return torch.cat(got)
    lp, entropy, stats, top = ([x for x in column] for column in zip(*got))
    out = {"logprobs": torch.cat(lp), "entropy": torch.cat(entropy), "stats": torch.cat(stats)}
    return {**out, "top_ids": None, "top_logprobs": torch.cat(top)} if case["top_k"] else out


def _exact_grpo(s):
    host = {k: s[k].double().cpu().numpy() for k in ("new", "old", "sampler", "adv", "grad_out")}
    shape = host["new"].shape
    keep = np.ones(shape) if s["mask"] is None else (s["mask"].cpu().numpy() != 0).astype(np.float64)
    adv = np.broadcast_to(host["adv"][:, None], shape)
    ratio, eps, beta, cap = np.exp(host["new"] - host["old"]), float(np.float32(0.2)), float(np.float32(0.04)), 2.0
    weight = np.minimum(np.exp(host["old"] - host["sampler"]), cap)
    inside = (ratio >= 1 - eps) & (ratio <= 1 + eps)
    value = np.minimum(ratio * adv, np.clip(ratio, 1 - eps, 1 + eps) * adv)
    active = inside | (ratio * adv < np.clip(ratio, 1 - eps, 1 + eps) * adv)
    slope = np.where(active, ratio * adv, 0.0)
    if s["ref"] is not None:
        gap = s["ref"].double().cpu().numpy() - host["new"]
        value = value - beta * (np.expm1(gap) - gap)
        slope = slope + beta * np.expm1(gap)
    number = np.maximum(keep.sum(axis=1), 1.0)
    return {"objective": (keep * weight * value).sum(axis=1) / number,
            "grad": keep * weight * slope * (host["grad_out"] / number)[:, None]}


def _exact_adamw(case, seed):
    sizes = [int(x) for x in case["sizes"].split()]
    if case["bits"] == 8 and sum(sizes) > 30_000_000:
        return None                                      # the random numbers alone take too long
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    t = s["step"]
    grad = s["g"].double() * s["grad_scale"].double()
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        c, e = s["m"].double() / 127, s["v"].double() / 255
        wide = s["scales"].double().repeat_interleave(BLOCK, dim=1)
        m, v = wide[0] * c * c.abs(), wide[1] * e ** 4
    m, v = BETA1 * m + (1 - BETA1) * grad, BETA2 * v + (1 - BETA2) * grad ** 2
    p = s["p"].double()
    decay = torch.ones_like(p)
    decay[:s["decayed"]] = 1 - LR * DECAY
    p = p * decay - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"params": p}
    if case["copy"]:
        out["copy"] = p
    if case["bits"] == 32:
        return {**out, "exp_avg": m, "exp_avg_sq": v}
    m, v = m.cpu().numpy().reshape(-1, BLOCK), v.cpu().numpy().reshape(-1, BLOCK)
    top = np.abs(m).max(axis=1, keepdims=True).astype(np.float32).astype(np.float64)
    c = np.rint(127 * np.sqrt(np.abs(m) / np.where(top > 0, top, 1))) * np.sign(m)
    m = top * (c / 127) * np.abs(c / 127)
    top = v.max(axis=1, keepdims=True).astype(np.float32).astype(np.float64)
    c = np.minimum(np.floor(255 * (v / np.where(top > 0, top, 1)) ** 0.25), 254)
    under, over = top * (c / 255) ** 4, top * ((c + 1) / 255) ** 4
    u = np.concatenate([_exact_halves(-(-n // BLOCK) * BLOCK, i, t, s["seed"]) for i, n in enumerate(sizes)])
    c = c + (u.reshape(-1, BLOCK) / 65536.0 * (over - under) < v - under)
    c = np.where(v > 0, np.maximum(c, 1), c)
    return {**out, "exp_avg": m.reshape(-1), "exp_avg_sq": (top * (c / 255) ** 4).reshape(-1)}


def _exact_halves(n, tensor, step, seed):
    word, mul = np.uint64(0xFFFFFFFF), (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57))
    i, half = np.arange(n // 8, dtype=np.uint64), np.uint64(32)
    x = [i & word, i >> half, np.full_like(i, tensor), np.full_like(i, step)]
    key = [np.uint64(seed & 0xFFFFFFFF), np.uint64((seed >> 32) & 0xFFFFFFFF)]
    for r in range(10):
        a, b = mul[0] * x[0], mul[1] * x[2]              # 32 x 32 bits fit 64
        x = [(b >> half) ^ x[1] ^ key[0], b & word, (a >> half) ^ x[3] ^ key[1], a & word]
        key = [(key[0] + np.uint64(0x9E3779B9)) & word, (key[1] + np.uint64(0xBB67AE85)) & word]
    out = np.empty((n // 8, 8))
    for j in range(4):
        out[:, 2 * j], out[:, 2 * j + 1] = x[j] & np.uint64(0xFFFF), x[j] >> np.uint64(16)
    return out.reshape(-1)
