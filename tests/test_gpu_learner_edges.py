"""GPU tests of the learner's operators where their inputs leave the ordinary: overflowed ratios, undefined scores, ids
outside the vocabulary, gradients far below their block's, decay below a weight's last bit, long runs of 8-bit moments."""
import math

import numpy as np
import pytest
import torch

from oracle import learner as L
from oracle import objective as o_obj

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2602_02192_b200 import binding
    return binding


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()


def _objective(B, ln, lo, ls, lr, adv, eps=0.2, C=2.0, beta=0.04):
    """(value and gradient of the gradient call, value of the forward call), each [n] or [n][T] fp64."""
    a = [_dev(x) for x in (ln, lo, ls)]
    r = None if lr is None else _dev(lr)
    value, grad = B.echo_grpo_gradient(*a, r, _dev(adv), None, None, eps, C, beta)
    forward = B.echo_grpo_surrogate(*a, _dev(adv), None, eps, C) if r is None else B.echo_grpo_objective(*a, r, _dev(adv), None, eps, C, beta)
    return (x.double().cpu().numpy() for x in (value, grad, forward))


# ---- objective ----------------------------------------------------------------------------------
@pytest.mark.parametrize("T", [1, 4, 300])               # one token, a vector of them; a warp or a CTA per sequence
@pytest.mark.parametrize("kl", [False, True])
def test_zero_advantage_beside_an_overflowed_ratio(B, T, kl):
    """A = 0 makes the clipped term and its slope 0, whatever the ratio: what is left is the KL term, here -beta k and
    beta expm1(d) with d = -1.5 under w = 1."""
    lo = np.full((2, T), -101.0)
    ln = np.full((2, T), -0.5)
    ln[:, 1::2] = -101.5                                  # ordinary tokens among them
    lr = ln - 1.5
    value, grad, forward = _objective(B, ln, lo, lo, lr if kl else None, np.zeros(2))
    beta = float(np.float32(0.04))
    want = L.grpo_gradient(ln, lo, lo, lr if kl else None, np.zeros(2), None, None, float(np.float32(0.2)), 2.0, beta)
    J = -beta * (math.exp(-1.5) + 1.5 - 1.0) if kl else 0.0
    # expm1f is good to 2 steps (4 e), a handful of roundings beside; sums of T equal terms by at least 32 threads
    assert np.all(np.abs(grad - want) <= 16 * E * np.abs(want))
    assert np.all(np.abs(value - J) <= (16 + T / 32 + 16) * E * abs(J))
    assert np.all(np.abs(forward - J) <= (16 + T / 32 + 16) * E * abs(J))


@pytest.mark.parametrize("T", [1, 8, 301])
@pytest.mark.parametrize("kl", [False, True])
@pytest.mark.parametrize("adv", [1.0, -0.5, 0.0])
def test_undefined_log_probabilities_show(B, T, kl, adv):
    """NaN in any log-probability of a token that counts, and -inf beside -inf (scores of rows with nothing left), reach
    that sequence's value and that token's gradient, and no other; the forward calls agree."""
    inf, nan = math.inf, math.nan
    bad = [dict(ln=nan), dict(lo=nan), dict(ls=nan), dict(ln=-inf, lo=-inf), dict(lo=-inf, ls=-inf)]
    if kl:
        bad += [dict(lr=nan), dict(ln=-inf, lr=-inf)]
    n, at = len(bad) + 1, T // 2
    x = {k: np.full((n, T), v) for k, v in (("ln", -1.0), ("lo", -1.1), ("ls", -1.2), ("lr", -0.9))}
    for i, change in enumerate(bad):
        for k, v in change.items():
            x[k][i, at] = v
    args = x["ln"], x["lo"], x["ls"], x["lr"] if kl else None, np.full(n, adv)
    value, grad, forward = _objective(B, *args)
    want = np.zeros((n, T), dtype=bool)
    want[:-1, at] = True
    assert np.array_equal(np.isnan(grad), want) and np.isfinite(grad[~want]).all()
    assert np.isnan(value[:-1]).all() and np.isfinite(value[-1]) and np.isnan(forward[:-1]).all() and np.isfinite(forward[-1])
    mask = np.ones((n, T), np.uint8)
    with np.errstate(invalid="ignore"):
        oracle = L.grpo_gradient(*args, None, None, 0.2, 2.0, 0.04)
        J = o_obj.grpo_objective(*args, mask, 0.2, 2.0, 0.04) if kl else o_obj.grpo_surrogate(*args[:3], args[4], mask, 0.2, 2.0)
    assert np.array_equal(np.isnan(oracle), want)
    assert np.isnan(J[:-1]).all() and np.isfinite(J[-1])


def test_no_weight_on_the_reference_policy(B):
    """beta = 0 is the objective without the KL term, also where exp(logp_ref - logp_new) overflows."""
    rng = np.random.default_rng(8)
    lo = -np.abs(rng.normal(size=(3, 40)))
    ln, ls, adv = lo + 0.1 * rng.normal(size=lo.shape), lo + 0.1 * rng.normal(size=lo.shape), rng.normal(size=3)
    lr = ln + 0.2
    lr[:, ::3] = ln[:, ::3] + 100.0
    with_ref = list(_objective(B, ln, lo, ls, lr, adv, beta=0.0))
    without = list(_objective(B, ln, lo, ls, None, adv))
    assert all(np.isfinite(a).all() and np.array_equal(a, b) for a, b in zip(with_ref, without))


# ---- gradient of the logits ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("how", ["dense", "in place", "strided"])
@pytest.mark.parametrize("entropy", [False, True])
def test_ids_outside_the_vocabulary_have_no_finite_gradient(B, dtype, how, entropy):
    """The forward call scores them NaN; the gradient must not be an ordinary one that pushes the whole row down."""
    R, V = 6, 1003
    gen = torch.Generator(device="cuda").manual_seed(2)
    store = torch.randn((R, V + 5), generator=gen, device="cuda").to(dtype)
    z = store[:, :V]
    z[3] = -math.inf                                      # nothing left, and an id that is none
    y = torch.tensor([V, 2 ** 31 - 1, V, V, 7, -1], dtype=torch.int32, device="cuda")
    a = torch.tensor([1.0, -0.5, 0.0, 1.0, 1.0, 1.0], device="cuda")       # nothing arrives at row 2's score
    b = torch.full((R,), 0.3, device="cuda") if entropy else None
    lp, H, st, _, _ = B.echo_token_logprobs(z, y)
    assert torch.isnan(lp).tolist() == [True] * 4 + [False] * 2
    want = L.token_logprobs_backward(z.double().cpu().numpy(), y.cpu().numpy(), 1.0, a.cpu().numpy(),
                                     b.cpu().numpy() if entropy else None)
    out = {"dense": None, "in place": z, "strided": torch.zeros((R, V + 9), dtype=dtype, device="cuda")[:, 3:V + 3]}[how]
    g = B.echo_token_logprobs_backward(z, y, H, st, a, b, out=out)
    nan = torch.isnan(g).cpu().numpy()
    assert np.array_equal(nan, np.isnan(want))
    assert nan.all(axis=1).tolist() == [True, True, False, True, False, False] and not nan[[2, 4, 5]].any()


# ---- AdamW --------------------------------------------------------------------------------------
@pytest.mark.parametrize("gdtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw_8_keeps_second_moments_far_below_their_block(B, gdtype, offset):
    """(1 - beta2) g^2 of a gradient of 1e-23 is 0 in fp32 and 1e-49 in the definition: code 1 beside gradients of 1e-3,
    code 0 only where there is no gradient.  The same for an old v beside a gradient of 1e16."""
    n = 256 * 3 + 77
    rng = np.random.default_rng(31)
    g = rng.normal(size=n) * 1e-3
    g[rng.random(n) < 0.3] = 0
    small = rng.random(n) < 0.3
    g[small] = rng.choice([-1e-23, 1e-23, 1e-30, 3e-22], size=small.sum())
    codes, vcodes = rng.integers(-127, 128, n).astype(np.int8), rng.integers(0, 3, n).astype(np.uint8)
    scales, vscales = np.full(4, 1e-3, np.float32), np.full(4, 1e-20, np.float32)
    codes[:256], vcodes[:256], scales[0], vscales[0] = 0, 0, 0, 0           # nothing before
    g[512] = 1e16

    def dev(x, dtype):
        store = torch.zeros(n + offset, dtype=dtype, device="cuda")[offset:]
        store.copy_(torch.from_numpy(x))
        return store

    tg = dev(g, gdtype)
    tm, tv, p = dev(codes, torch.int8), dev(vcodes, torch.uint8), dev(np.zeros(n), torch.float32)
    sm, sv = _dev(scales), _dev(vscales)
    B.echo_adamw_step(B.AdamWTensors([p], [tg], [tm], [tv], None, 0.0, [sm], [sv]), 5, 1e-3, seed=4)
    g64 = tg.double().cpu().numpy()
    _, wm, wv = L.adamw(np.zeros(n), g64, L.avg_values(codes, scales), L.sq_values(vcodes, vscales), 5, 1e-3, 0.9, 0.999, 1e-8, 0.0)
    cv, csv = L.quantise_sq(wv, L.halves(n, 0, 5, 4))
    cm, csm = L.quantise_avg(wm)
    assert np.all((cv == 0) == (wv == 0)) and np.all(cv[512:768] >= (wv[512:768] > 0))
    assert np.array_equal(sv.cpu().numpy(), csv) and np.array_equal(tv.cpu().numpy(), cv)
    assert np.array_equal(sm.cpu().numpy(), csm) and np.array_equal(tm.cpu().numpy(), cm)


def _state8(sizes, gdtype, seed, offset):
    """Random weights, gradients, codes and scales of 8-bit moments, `offset` elements into their storage."""
    rng = np.random.default_rng(seed)

    def t(x, dtype):
        store = torch.zeros(len(x) + offset, dtype=dtype, device="cuda")[offset:]
        store.copy_(torch.from_numpy(np.asarray(x)))
        return store

    d = {k: [] for k in ("p", "g", "m", "v", "ms", "vs")}
    for n in sizes:
        nb = -(-n // 256)
        g = rng.normal(size=n) * 1e-3 * np.exp(rng.normal(size=n) * 2)
        g[rng.random(n) < 0.2] = 0
        if nb > 4:
            g[256:512] = 0                                # a block that only decays
            g[512:768] *= 1e-16                           # and one whose v leave fp32's normal numbers
        ms, vs = rng.random(nb) * 1e-3, rng.random(nb) * 1e-6
        if nb > 4:
            ms[2], vs[2] = 1e-33, 1e-35
        d["p"].append(t(rng.normal(size=n) * 0.05, torch.float32))
        d["g"].append(t(g, gdtype))
        d["m"].append(t(rng.integers(-127, 128, n), torch.int8))
        d["v"].append(t(rng.integers(0, 256, n), torch.uint8))
        d["ms"].append(t(ms, torch.float32))
        d["vs"].append(t(vs, torch.float32))
    return d


@pytest.mark.parametrize("gdtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("seed,step,scale,beta1", [(0, 1, None, 0.9), (3, 2, None, 0.9), (0xDEADBEEF12345678, 1000, 2.5, 0.9),
                                                   (9, 7, 0.5, 0.5), (1, 4, 1.0, 0.0)])
def test_adamw_8_random_first_moments(B, gdtype, offset, seed, step, scale, beta1):
    """Codes and scales are those of the 64-bit definition, exactly; the weights are those that nearest codes give."""
    sizes = [1, 255, 256, 257, 3, 2048, 0, 70001, 512, 8, 300_000]
    d = _state8(sizes, gdtype, 6, offset)
    before = {k: [x.double().cpu().numpy() for x in d[k]] for k in ("p", "g")}
    codes = [[x.cpu().numpy() for x in d[k]] for k in ("m", "ms", "v", "vs")]
    other = {k: [x.clone() for x in d[k]] for k in d}
    gs = torch.tensor([scale], device="cuda") if scale else None
    B.echo_adamw_step(B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], None, 0.02, d["ms"], d["vs"], random_avg=True),
                      step, 1e-3, beta1, 0.999, 1e-8, grad_scale=gs, seed=seed)
    B.echo_adamw_step(B.AdamWTensors(other["p"], d["g"], other["m"], other["v"], None, 0.02, other["ms"], other["vs"]),
                      step, 1e-3, beta1, 0.999, 1e-8, grad_scale=gs, seed=seed)
    for i, n in enumerate(sizes):
        if n == 0:
            continue
        m0, v0 = L.avg_values(codes[0][i], codes[1][i]), L.sq_values(codes[2][i], codes[3][i])
        _, wm, wv = L.adamw(before["p"][i], before["g"][i], m0, v0, step, 1e-3, beta1, 0.999, 1e-8, 0.02, scale or 1.0)
        cm, sm = L.quantise_avg(wm, L.halves(n, i, step, seed, 1) if step > 1 else None)
        cv, sv = L.quantise_sq(wv, L.halves(n, i, step, seed))
        assert np.array_equal(d["ms"][i].cpu().numpy(), sm) and np.array_equal(d["vs"][i].cpu().numpy(), sv)
        assert np.array_equal(d["m"][i].cpu().numpy(), cm)
        assert np.array_equal(d["v"][i].cpu().numpy(), cv)
        assert torch.equal(d["p"][i], other["p"][i])
        assert (step == 1) == torch.equal(d["m"][i], other["m"][i]) or n < 256


def test_adamw_8_random_first_moments_where_everything_cancels(B):
    """(1 - beta1) g = -beta1 m up to the last bits in whole blocks: fp32's m is mostly rounding, 64 bits decide."""
    n = 256 * 4
    rng = np.random.default_rng(12)
    codes, scales = rng.integers(-127, 128, n).astype(np.int8), np.full(4, 1e-3, dtype=np.float32)
    vcodes, vscales = rng.integers(1, 256, n).astype(np.uint8), np.full(4, 1e-6, dtype=np.float32)
    m, v = L.avg_values(codes, scales), L.sq_values(vcodes, vscales)
    g = (-9.0 * m * (1 + np.repeat([1e-7, 1e-6, 1e-4, 1e-2], 256) * rng.normal(size=n))).astype(np.float32)
    tm, tv, p = torch.from_numpy(codes).cuda(), torch.from_numpy(vcodes).cuda(), torch.zeros(n, device="cuda")
    sm, sv = _dev(scales), _dev(vscales)
    B.echo_adamw_step(B.AdamWTensors([p], [_dev(g)], [tm], [tv], None, 0.0, [sm], [sv], random_avg=True), 5, 1e-3, seed=77)
    _, wm, wv = L.adamw(np.zeros(n), g, m, v, 5, 1e-3, 0.9, 0.999, 1e-8, 0.0)
    cm, csm = L.quantise_avg(wm, L.halves(n, 0, 5, 77, 1))
    cv, csv = L.quantise_sq(wv, L.halves(n, 0, 5, 77))
    assert np.array_equal(sm.cpu().numpy(), csm) and np.array_equal(tm.cpu().numpy(), cm)
    assert np.array_equal(sv.cpu().numpy(), csv) and np.array_equal(tv.cpu().numpy(), cv)


def _drift(B, random_avg, steps, beta2, ratio):
    """Mean distance, in lr, of 8-bit from 32-bit moments for elements (one in 16) whose gradients are `ratio` of the
    others' (0: as large as the others' up to step 50, then none)."""
    n, lr = 4096, 1e-3
    gen = torch.Generator(device="cuda").manual_seed(1)
    special = torch.arange(n, device="cuda") % 16 == 0
    p32, p8, grad = (torch.zeros(n, device="cuda") for _ in range(3))
    a, b = B.AdamWTensors.zeros([p32], [grad]), B.AdamWTensors.zeros([p8], [grad], state_bits=8, random_avg=random_avg)
    for t in range(1, steps + 1):
        g = torch.randn(n, generator=gen, device="cuda") * 1e-3
        g[special] *= ratio if ratio else float(t <= 50)
        grad.copy_(g)
        B.echo_adamw_step(a, t, lr, 0.9, beta2)
        B.echo_adamw_step(b, t, lr, 0.9, beta2, seed=5)
    return float((p8 - p32)[special].abs().mean()) / lr


def test_adamw_8_lets_go_of_ended_gradients(B):
    """At most about 1 lr of rounding (derived beside the same test of the oracle), at step 500 and for good; nearest codes
    drift by several lr a step."""
    assert _drift(B, True, 500, 0.95, 0) < 2.0 and _drift(B, True, 2000, 0.95, 0) < 2.0
    assert _drift(B, True, 2000, 0.999, 0) < 2.0
    assert _drift(B, False, 500, 0.95, 0) > 100.0


def test_adamw_8_small_gradients_beside_large_ones(B):
    """At 1e-4 of the block's others a first moment is below code 1, whose value is 6e-5 of the block's largest: rounding
    at random is noise without a drift, nearest codes keep whatever once reached one."""
    assert _drift(B, True, 2000, 0.999, 1e-4) < _drift(B, False, 2000, 0.999, 1e-4)
    assert _drift(B, True, 2000, 0.999, 3e-4) < _drift(B, False, 2000, 0.999, 3e-4)


@pytest.mark.parametrize("bits,gdtype", [(32, torch.float32), (32, torch.bfloat16), (8, torch.float32)])
@pytest.mark.parametrize("lr,decay", [(1e-6, 0.01), (1e-6, 0.1), (3e-5, 0.1), (1e-3, 0.0), (0.4, 7.0)])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw_decay_below_a_weights_last_bit(B, bits, gdtype, lr, decay, offset):
    """lr * weight_decay = 1e-8 is a twelfth of the last bit of a weight in [1, 2).  Every weight is the fp32 number next to
    its exact value, up to what comes before that rounding: the update's 20 roundings (of m relative to the sum of its
    terms), one of its sum with the decay's second part, which is at most 2^-24 of the weight, and one of that part."""
    n = 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(17)
    rand = lambda: torch.rand(n + offset, generator=gen, device="cuda")  # noqa: E731
    p, g = (1 + rand())[offset:], (rand() - 0.5).to(gdtype)[offset:]
    if bits == 32:
        m, v, scales = (rand() - 0.5)[offset:], (0.1 + rand())[offset:], ()
        m64, v64 = m.double(), v.double()
    else:
        m = torch.randint(-127, 128, (n + offset,), generator=gen, device="cuda").to(torch.int8)[offset:]
        v = torch.randint(128, 256, (n + offset,), generator=gen, device="cuda").to(torch.uint8)[offset:]
        scales = [torch.full((n // 256,), 0.5, device="cuda")], [torch.full((n // 256,), 1.0, device="cuda")]
        m64, v64 = 0.5 * (m.double() / 127) * (m.double() / 127).abs(), (v.double() / 255) ** 4
    p64, g64 = p.double(), g.double()
    B.echo_adamw_step(B.AdamWTensors([p], [g], [m], [v], None, decay, *scales), 9, lr)
    v64 = 0.999 * v64 + (1 - 0.999) * g64 * g64
    rate = lr / (1 - 0.9 ** 9) / ((v64 / (1 - 0.999 ** 9)).sqrt() + 1e-8)
    want = p64 * (1 - lr * decay) - rate * (0.9 * m64 + (1 - 0.9) * g64)
    before_rounding = 21 * E * rate * (0.9 * m64.abs() + (1 - 0.9) * g64.abs()) + 2 * E * E * p64
    half_step = torch.ldexp(torch.full_like(want, E), torch.frexp(p.double())[1] - 1)
    assert bool(((p.double() - want).abs() <= half_step + before_rounding).all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_adamw_leaves_infinite_weights(B, bits, decay):
    p = torch.tensor([math.inf, -math.inf, 1.0] * 100, device="cuda")
    before, g = p.clone(), torch.zeros(300, device="cuda")
    B.echo_adamw_step(B.AdamWTensors.zeros([p], [g], state_bits=bits, weight_decay=decay), 1, 3e-5)
    assert torch.equal(p[0::3], before[0::3]) and torch.equal(p[1::3], before[1::3]) and torch.isfinite(p[2::3]).all()


def test_adamw_handle_with_autograd(B):
    """The usual loop: gradients that autograd makes anew every step."""
    torch.manual_seed(4)
    model = torch.nn.Linear(64, 8, bias=False, device="cuda")
    p = model.weight
    x = torch.randn(32, 64, device="cuda")

    def backward():
        model.zero_grad()                                  # (set_to_none)
        model(x).pow(2).sum().backward()

    backward()
    plan = B.AdamWTensors.zeros([p], [p.grad])
    w, m, v = p.detach().double().cpu().numpy().ravel(), np.zeros(512), np.zeros(512)
    for t in range(1, 4):
        if t > 1:
            old = p.grad
            backward()
            if p.grad is not old:
                with pytest.raises(RuntimeError):
                    B.echo_adamw_step(plan, t, 1e-2)
            plan.set_grads([p.grad])
        g = p.grad.double().cpu().numpy().ravel()
        B.echo_adamw_step(plan, t, 1e-2)
        w, m, v = L.adamw(w, g, m, v, t, 1e-2, 0.9, 0.999, 1e-8, 0.0)
        got = p.detach().double().cpu().numpy().ravel()
        # moments: 8 e of terms of one size; the update: 14 e more; both at most 10 lr here; three steps
        assert np.abs(got - w).max() <= t * (30 * E * 1e-2 * 10 + E * np.abs(w).max())


def test_adamw_random_first_moments_on_a_stream_and_in_a_graph(B):
    """Three steps, eager on the current stream, on another, and replayed from a graph, end in the same state."""
    sizes = [5000, 1, 300]
    d = _state8(sizes, torch.bfloat16, 2, 0)
    start = {k: [x.clone() for x in d[k]] for k in d}
    plan = B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], None, 0.1, d["ms"], d["vs"], random_avg=True)

    def run():
        for t in (4, 5, 6):
            B.echo_adamw_step(plan, t, 1e-3, seed=9)

    def reset():
        for k in d:
            for x, s in zip(d[k], start[k]):
                x.copy_(s)

    def state():
        torch.cuda.synchronize()
        return [x.clone() for k in d for x in d[k]]

    run()
    want = state()
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    assert all(torch.equal(a, b) for a, b in zip(want, state()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(2):
        reset()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, state()))


def test_objective_with_undefined_scores_reaches_the_weights_as_nan(B):
    """A token that the scoring call cannot score (an id outside the vocabulary) shows in every step after it, in its own
    sequence alone."""
    V, n, T = 500, 4, 8
    gen = torch.Generator(device="cuda").manual_seed(6)
    z = torch.randn((n * T, V), generator=gen, device="cuda")
    y = torch.randint(0, V, (n * T,), generator=gen, device="cuda", dtype=torch.int32)
    y[2 * T + 3] = V
    lp, H, st, _, _ = B.echo_token_logprobs(z, y)
    old = torch.where(torch.isnan(lp), torch.zeros_like(lp), lp).view(n, T)
    value, g = B.echo_grpo_gradient(lp.view(n, T), old, old, None, torch.ones(n, device="cuda"), None, None, 0.2, 2.0, 0.0)
    dz = B.echo_token_logprobs_backward(z, y, H, st, g.view(-1))
    row = torch.zeros(n * T, dtype=torch.bool, device="cuda")
    row[2 * T + 3] = True
    assert torch.isnan(value).tolist() == [False, False, True, False]
    assert torch.equal(torch.isnan(dz).all(dim=1), row) and torch.equal(torch.isnan(dz).any(dim=1), row)


@pytest.mark.parametrize("offset", [0, 1])
def test_adamw_8_on_the_border_between_two_codes(B, offset):
    """|m| a quarter of the block's largest is 127 / 2 on the codes' axis: the even one, 64, is taken (as by rint), for
    blocks of every 8-bit mantissa (in fp32 one over some of them falls short), and beside neighbours one fp32 step away."""
    n = 128 * 256
    largest = np.repeat(1 + np.arange(128) / 128, 256).astype(np.float32)
    g = largest.copy()
    g[1::4] *= np.float32(-0.25)
    g[2::4] = np.nextafter(g[2::4] / 4, np.float32(0))
    g[3::4] = np.nextafter(g[3::4] / 4, np.float32(9))
    store = torch.zeros(n + offset, device="cuda")[offset:]
    store.copy_(torch.from_numpy(g))
    tm, tv = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    sm, sv, p = torch.zeros(128, device="cuda"), torch.zeros(128, device="cuda"), torch.zeros(n, device="cuda")
    B.echo_adamw_step(B.AdamWTensors([p], [store], [tm], [tv], None, 0.0, [sm], [sv]), 1, 1e-3, beta1=0.0)
    want, scale = L.quantise_avg(g.astype(np.float64))
    assert np.array_equal(sm.cpu().numpy(), largest[::256]) and np.array_equal(scale, largest[::256])
    assert np.array_equal(tm.cpu().numpy(), want)
    assert want.reshape(-1, 4).min(axis=0).tolist() == [127, -64, 63, 64] == want.reshape(-1, 4).max(axis=0).tolist()


@pytest.mark.parametrize("T", [1, 4, 300])
@pytest.mark.parametrize("adv", [-1.0, 0.7, 0.0])
def test_ratios_that_overflow_beside_weights_that_underflow(B, T, adv):
    """An old policy that all but rules a token out: rho = exp(ln - lo) overflows, w = exp(lo - ls) underflows, and w rho is
    exp(ln - ls).  The same for the estimate's exp(lr - ln) beside w.  Against the formula with its products formed from
    sums of exponents, in 64 bits; the kernel's exponents are off by 2 e of each difference where it multiplies."""
    cases = [(-1.0, -120.0, -2.0, -1.5), (-1.0, -90.0, -2.0, -1.5), (-0.5, -81.0, -1.0, -0.7), (-0.5, -79.0, -1.0, -0.7),
             (-0.1, -1e4, -3.0, -0.2), (-120.0, -120.5, -2.0, -1.0), (-100.0, -190.0, -3.0, -2.0), (-1.0, -1.1, -1.2, -0.9),
             (-1.0, -120.0, -121.0, -1.1), (-95.0, -1.0, -1.0, -94.0)]
    x = np.array([[c] * T for c in cases], dtype=np.float32).astype(np.float64)          # [cases][T][4]
    ln, lo, ls, lr = (x[..., i] for i in range(4))
    eps, C, beta = float(np.float32(0.2)), 2.0, float(np.float32(0.04))
    lw = np.minimum(lo - ls, math.log(C))
    a, w = np.full(ln.shape, adv), np.exp(lw)
    with np.errstate(over="ignore", invalid="ignore"):
        w_rho, clip = np.exp(ln - lo + lw), np.clip(np.exp(ln - lo), 1 - eps, 1 + eps)
        policy = np.where(a == 0, 0.0, np.minimum(w_rho * a, w * clip * a))
        flat = np.where(a > 0, ln - lo > math.log1p(eps), ln - lo < math.log1p(-eps))
        slope = np.where(flat | (a == 0), 0.0, w_rho * a)
        w_k = np.exp(lr - ln + lw) - w
    for kl in (False, True):
        term = policy - (beta * (w_k - w * (lr - ln)) if kl else 0.0)
        d = slope + (beta * w_k if kl else 0.0)
        size = np.abs(policy) + np.abs(slope) + (beta * (np.abs(w_k) + w * (np.abs(lr - ln) + 1)) if kl else 0.0)
        exponents = np.minimum(np.abs(ln - lo), 80) + np.minimum(np.abs(lo - ls), 100) + np.minimum(np.abs(lr - ln), 80)
        tol = E * (24 + 2 * exponents) * size + 1e-37
        over = (np.abs(term) > 3.4e38) | (np.abs(d) > 3.4e38)                              # what fp32 cannot hold
        value, grad, forward = _objective(B, ln, lo, ls, lr if kl else None, np.full(len(cases), adv))
        assert not np.isnan(grad).any() and not np.isnan(value).any() and not np.isnan(forward).any()
        assert np.all((np.abs(grad * T - d) <= tol + 2 * E * np.abs(d))[~over])
        rows = ~over.any(axis=1)
        mean, mean_tol = term.mean(axis=1), tol.mean(axis=1) + E * (T / 32 + 20) * size.mean(axis=1)
        assert np.all((np.abs(value - mean) <= mean_tol)[rows]) and np.all((np.abs(forward - mean) <= mean_tol)[rows])
        assert rows.sum() >= 8


@pytest.mark.parametrize("adv", [0.7, 0.0])
def test_tokens_that_the_old_policy_rules_out(B, adv):
    """logp_old = -inf: the weight is 0, and so are the clipped term (0.7: at the border) and the KL term, however large."""
    one = np.ones((1, 1))
    for ln, lr in ((-90.0, -0.5), (-120.0, -0.5), (-1.0, -2.0)):
        for ref in (None, lr * one):
            value, grad, forward = _objective(B, ln * one, -math.inf * one, -one, ref, np.array([adv]))
            assert value[0] == 0 and grad[0, 0] == 0 and forward[0] == 0
