"""GPU parity of the learner's operators: token log-probabilities and their gradient, the objective's gradient, AdamW.

Every kernel is compared with the fp64 oracle on the same (already rounded) inputs.  Bounds are sums of roundings:
e = 2^-24 is half a step of fp32; a row of V logits is summed by at least 128 threads, so that a sum of
non-negative terms passes through at most n = V / 128 + 64 additions, each off by at most e relative; ex2 is good to
4 e (its documented 2^-22), its argument x = (z - zmax) log2(e) / T carries three roundings, 3 e |x|.
"""
import math

import numpy as np
import pytest
import torch

from oracle import learner as L
from oracle import objective as o_obj

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: E}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}      # below the normal numbers


@pytest.fixture(scope="module")
def B():
    from paper_2602_02192_b200 import binding
    return binding


def _rows(kind, R, V, dtype, seed, pad=0, offset=0):
    """Logits as a device tensor (rows V + pad apart, offset elements into their storage)."""
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(R, V)) * 2.0
    if kind == "peaked":
        z[np.arange(R), rng.integers(0, V, R)] += 25.0
    elif kind == "offset":
        z += rng.choice([-3e3, 1e3, 2e4], size=(R, 1))
    elif kind == "constant":
        z[:] = rng.normal(size=(R, 1))
    elif kind == "ascending":
        z = np.sort(z, axis=1)
    elif kind == "few":
        z = rng.integers(-2, 3, size=(R, V)).astype(np.float64)       # ties everywhere, -0 among them
        z[z == 0] *= -1.0
    elif kind == "masked":
        z[rng.random((R, V)) < 0.97] = -np.inf
        z[0] = -np.inf                                                 # a row with nothing left
        if R > 1:
            z[1, 1:] = -np.inf                                         # one id left
            z[1, 0] = 1.5
        if R > 2:
            z[2] = float(torch.finfo(dtype).min)                       # the type's lowest value everywhere
        if R > 3:
            z[3, V // 2:] = float(torch.finfo(dtype).min)
    store = torch.zeros(R * (V + pad) + offset, dtype=dtype, device="cuda")
    view = store[offset:].view(R, V + pad)[:, :V]
    view.copy_(torch.from_numpy(z).cuda())
    return view


def _bounds(z64, temperature, V):
    """Per row: bound of log l, of the entropy; and s = (z - zmax) / T (-inf kept)."""
    n = V / 128 + 64
    logp, p, empty, bad = L.log_softmax(z64, temperature)
    p = np.where(empty[:, None], 0.0, p)                 # a row with nothing left: constants, no sums
    with np.errstate(invalid="ignore"):
        s = (z64 - z64.max(axis=1, keepdims=True)) / temperature
    ps = np.where(p > 0, p * np.abs(np.where(p > 0, s, 0.0)), 0.0)
    A, S2 = ps.sum(axis=1), np.where(p > 0, ps * np.abs(np.where(p > 0, s, 0.0)), 0.0).sum(axis=1)
    logl = np.abs(np.where(np.isfinite(s), s, 0.0) - np.where(np.isfinite(logp), logp, 0.0)).max(axis=1)
    d_logl = E * (n + 8 + 3 * A + 2 * logl)
    d_ent = d_logl + E * ((n + 12) * A + 4 * S2 + 4 * logl)
    return s, d_logl, d_ent


CASES = [("plain", 1, 1, 0, 0), ("plain", 3, 2, 0, 1), ("plain", 5, 33, 3, 0), ("plain", 2, 4096, 0, 0),
         ("plain", 1, 151936, 0, 0), ("plain", 5, 50263, 41, 1), ("plain", 700, 1003, 0, 0), ("peaked", 9, 8191, 1, 3),
         ("offset", 6, 4099, 0, 0), ("masked", 7, 20011, 5, 0), ("constant", 4, 151936, 0, 0), ("few", 4, 30011, 0, 1),
         ("ascending", 3, 100003, 0, 0), ("constant", 400, 300, 0, 0), ("masked", 400, 2500, 0, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind,R,V,pad,offset", CASES)
@pytest.mark.parametrize("temperature,top_k", [(1.0, 0), (0.7, 1), (1.3, 32), (1.0, 5)])
def test_token_logprobs(B, kind, R, V, pad, offset, dtype, temperature, top_k):
    z = _rows(kind, R, V, dtype, seed=R * 1000003 + V, pad=pad, offset=offset)
    rng = np.random.default_rng(V + R)
    y = rng.integers(0, V, R)
    y[rng.random(R) < 0.2] = -1
    if R > 4:
        y[4] = V                                        # not an id of the vocabulary
    tokens = torch.from_numpy(y.astype(np.int32)).cuda()
    z64 = z.double().cpu().numpy()
    T = float(np.float32(temperature))
    lp, H, st, ids, top = (x.cpu().numpy() if x is not None else None for x in B.echo_token_logprobs(z, tokens, temperature, top_k))
    wlp, wH, wst, wids, wtop = L.token_logprobs(z64, y, T, top_k)
    s, d_logl, d_ent = _bounds(z64, T, V)
    with np.errstate(invalid="ignore"):
        sy = np.where((y >= 0) & (y < V), np.abs(s[np.arange(R), np.clip(y, 0, V - 1)]), 0.0)
    fin = np.isfinite(wlp) & (np.abs(wlp) < 1e38)
    assert np.array_equal(np.isnan(lp), np.isnan(wlp))
    assert np.all(lp[~fin & ~np.isnan(wlp)] < -1e38)     # -inf, or the lowest value over T: out of fp32's range or next to it
    with np.errstate(invalid="ignore"):
        d_lp = np.abs(lp - wlp)
    assert np.all(d_lp[fin] <= (d_logl + E * (4 * np.where(np.isfinite(sy), sy, 0) + 2 * np.abs(wlp)))[fin])
    assert np.all(np.abs(H - wH) <= d_ent)
    assert np.array_equal(st[:, 0].astype(np.float64), wst[:, 0])        # the maximum is an input
    some = np.isfinite(wst[:, 1])
    assert np.array_equal(np.isneginf(st[:, 1]), ~some) and np.all(np.abs(st[:, 1] - wst[:, 1])[some] <= d_logl[some])
    if top_k:
        assert np.array_equal(ids, wids)
        ok = np.isfinite(wtop) & (np.abs(wtop) < 1e38)
        assert np.all(top[~ok] < -1e38)
        assert np.all(np.abs(top - wtop)[ok] <= (d_logl[:, None] + E * 8 * np.abs(np.where(ok, wtop, 0)))[ok])
    else:
        assert ids is None and top is None


def test_undefined_rows(B):
    z = torch.zeros((4, 3000), device="cuda")
    z[0, 17] = float("nan")
    z[1, 2999] = float("inf")
    z[2] = float("nan")
    z[3, 5] = 2.0
    tokens = torch.tensor([3, 4, 5, -1], dtype=torch.int32, device="cuda")
    lp, H, st, ids, _ = B.echo_token_logprobs(z, tokens, 1.0, 2)
    assert torch.isnan(lp[:3]).all() and torch.isnan(H[:3]).all() and torch.isnan(st[:3, 1]).all()
    assert lp[3] == 0 and torch.isfinite(H[3])
    assert ids.tolist() == [[0, 1], [2999, 0], [-1, -1], [5, 0]]
    g = B.echo_token_logprobs_backward(z, tokens, H, st, torch.ones(4, device="cuda"))
    assert torch.isnan(g[:3]).all() and bool((g[3] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("temperature", [1e-9, 1e-5, 1e4, 1e9, 3e37])
def test_extreme_temperatures_and_magnitudes(B, dtype, temperature):
    """Sharp and flat distributions, rows of huge and of lowest values beside -inf: rows that the one-FMA form leaves."""
    V, T = 2111, float(np.float32(temperature))
    z = _rows("plain", 6, V, dtype, 21)
    big = 6e4 if dtype == torch.float16 else 1e38
    z[1] = z[1] * (big / 16)
    z[2] = -big
    z[2, 5:] = -math.inf
    z[3] = torch.finfo(dtype).min
    z[3, ::2] = -math.inf
    z[4, :2000] = -math.inf
    for r, mask in enumerate((-3e4, -1e4, -1e9, -1e10, -1e20, -1e30)):     # masks of every size, alone and beside logits
        z = torch.cat([z, z[:1]])
        z[-1, 7:] = max(mask, float(torch.finfo(dtype).min))
        z = torch.cat([z, z[-1:]])
        z[-1, :7] = z[-1, 7]
    y = np.array([3, 4, 2, 1, 2100, -1] + [0, 9] * 6)
    z64 = z.double().cpu().numpy()
    lp, H, st, ids, top = (x.cpu().numpy() for x in B.echo_token_logprobs(z, torch.from_numpy(y.astype(np.int32)).cuda(), temperature, 5))
    wlp, wH, wst, wids, wtop = L.token_logprobs(z64, y, T, 5)
    s, d_logl, d_ent = _bounds(z64, T, V)
    assert np.array_equal(ids, wids)
    fin = np.abs(wlp) < 1e38
    assert np.all(lp[~fin] < -1e38)
    assert np.all(np.abs(lp - wlp)[fin] <= (d_logl + E * 6 * np.abs(wlp))[fin]) and np.all(np.abs(H - wH) <= d_ent)
    assert np.all(np.abs(st[:, 1] - wst[:, 1]) <= d_logl)
    fin = np.abs(wtop) < 1e38
    assert np.all(np.abs(top - wtop)[fin] <= (d_logl[:, None] + E * 8 * np.abs(wtop))[fin]) and np.all(top[~fin] < -1e38)


def test_statistics_without_tokens(B):
    z = _rows("plain", 6, 5000, torch.bfloat16, 1)
    lp, H, st, ids, top = B.echo_token_logprobs(z, None, 1.0, 3)
    _, H2, st2, ids2, top2 = B.echo_token_logprobs(z, torch.zeros(6, dtype=torch.int32, device="cuda"), 1.0, 3)
    assert lp is None and torch.equal(H, H2) and torch.equal(st, st2) and torch.equal(ids, ids2) and torch.equal(top, top2)
    lp, H, st, _, _ = B.echo_token_logprobs(z[:0], torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert lp.shape == (0,) and st.shape == (0, 2)


def test_every_split_of_a_row_gives_the_same_alternatives(B):
    """Few rows are cut over several CTAs, many are not: the same row must give the same answer either way."""
    for kind in ("plain", "few", "ascending", "masked"):
        z = _rows(kind, 4, 40009, torch.float16, 77)
        many = z.repeat(160, 1)
        y = torch.arange(4, dtype=torch.int32, device="cuda")
        a = B.echo_token_logprobs(z, y, 0.9, 32)
        b = B.echo_token_logprobs(many, y.repeat(160), 0.9, 32)
        assert torch.equal(a[3], b[3][:4]) and torch.equal(b[3][:4], b[3][-4:])
        for i in (0, 1):
            # the sums run in another order: over other CTAs, or (odd rows) from another 16-byte boundary
            assert torch.allclose(a[i], b[i][:4], rtol=0, atol=E * 800 * 12)
            assert torch.allclose(b[i][:4], b[i][-4:], rtol=0, atol=E * 800 * 12)


def test_rows_past_four_gigabytes(B):
    """The last rows of a matrix whose elements pass 32-bit offsets."""
    V, R = 151936, 30000
    z = torch.empty((R, V), dtype=torch.bfloat16, device="cuda")
    z[-3:] = _rows("plain", 3, V, torch.bfloat16, 5)
    y = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    y[-3:] = torch.tensor([7, 100000, V - 1], dtype=torch.int32)
    lp = torch.empty(R, device="cuda")
    st, H = torch.zeros((R, 2), device="cuda"), torch.zeros(R, device="cuda")
    # log-probabilities alone: rows without a token are not read
    s = torch.cuda.current_stream().cuda_stream
    assert B.lib.echo_token_logprobs(z.data_ptr(), 0, V, R, V, y.data_ptr(), 1.0, 0, lp.data_ptr(), None, None, None, None, s) == 0
    got = B.echo_token_logprobs(z[-3:], y[-3:])
    assert bool((lp[:-3] == 0).all()) and torch.allclose(lp[-3:], got[0], rtol=0, atol=E * 1300 * 12)
    st[-3:], H[-3:] = got[2], got[1]
    ga = torch.zeros(R, device="cuda")
    ga[-3:] = 1.0
    want = B.echo_token_logprobs_backward(z[-3:], y[-3:], got[1], got[2], ga[-3:])
    B.echo_token_logprobs_backward(z, y, H, st, ga, out=z)               # in place: 9 GB of zeros and three rows
    assert torch.equal(z[-3:], want) and bool((z[12345] == 0).all()) and bool((z[-4] == 0).all())
    del z
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind,R,V,pad,offset", [c for c in CASES if c[1] * c[2] < 800_000])
@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("how", ["dense", "in place", "strided"])
def test_token_logprobs_backward(B, kind, R, V, pad, offset, dtype, entropy, how):
    z = _rows(kind, R, V, dtype, seed=R * 1000003 + V, pad=pad, offset=offset)
    rng = np.random.default_rng(V + 3 * R)
    y = rng.integers(0, V, R)
    y[rng.random(R) < 0.2] = -1
    a, b = rng.normal(size=R).astype(np.float32), (rng.normal(size=R) * 0.3).astype(np.float32)
    a[rng.random(R) < 0.1] = 0
    T = 0.8
    tokens = torch.from_numpy(y.astype(np.int32)).cuda()
    z64 = z.double().cpu().numpy()
    _, H, st, _, _ = B.echo_token_logprobs(z, tokens, T)
    out = None
    if how == "in place":
        out = z
    elif how == "strided":
        out = torch.full((R, V + 7), 9.0, dtype=dtype, device="cuda")[:, 3:V + 3]
    g = B.echo_token_logprobs_backward(z, tokens, H, st, torch.from_numpy(a).cuda(),
                                       torch.from_numpy(b).cuda() if entropy else None, T, out=out)
    T = float(np.float32(T))
    want = L.token_logprobs_backward(z64, y, T, a, b if entropy else None)
    s, d_logl, d_ent = _bounds(z64, T, V)
    logp, p, empty, _ = L.log_softmax(z64, T)
    lp_abs = np.where(p > 0, np.abs(np.where(p > 0, logp, 0.0)), 0.0)
    _, wH, _, _, _ = L.token_logprobs(z64, y, T)
    bb = np.abs(b) if entropy else np.zeros(R)
    # p is off by the error of log l and of its own exponent; the bracket by the entropy's and by roundings
    rel = d_logl[:, None] + E * (5 * lp_abs + 3 * np.abs(np.where(np.isfinite(s), s, 0.0)) * (p > 0) + 10)
    bracket = np.abs(a)[:, None] + bb[:, None] * (lp_abs + np.abs(wH)[:, None])
    tol = p * (rel * bracket + bb[:, None] * (d_ent + d_logl)[:, None] + 6 * E * bracket) / T
    tol += (HALF_STEP[dtype] * 1.01 + 4 * E) * np.abs(want) + 3 * E * np.abs(a)[:, None] / T * (np.abs(want) > 0) + TINY[dtype]
    got = g.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()
    if how == "strided":
        base = g._base
        assert bool((base[:, :3] == 9).all()) and bool((base[:, V + 3:] == 9).all())      # what lies beside is untouched
    if how == "dense" and kind == "masked":
        off = torch.isneginf(z)
        off[np.arange(R)[y >= 0], y[y >= 0]] = False      # (a taken token's own entry holds a / T)
        assert bool((g[off] == 0).all())


def test_entropy_gradient_at_the_smallest_temperatures(B):
    """One id takes the whole mass: log p = 0 there, p = 0 elsewhere, so every gradient of the entropy is exactly 0, at -inf
    too, however large 1 / temperature is."""
    z = torch.full((2, 300), -1.0, device="cuda")
    z[:, 17] = 0.0
    z[1, 100:] = -math.inf
    _, H, st, _, _ = B.echo_token_logprobs(z, None, 1e-9)
    g = B.echo_token_logprobs_backward(z, None, H, st, None, torch.ones(2, device="cuda"), 1e-9)
    assert bool((H == 0).all()) and bool((g == 0).all())


def test_backward_leaves_padding_in_place(B):
    store = torch.full((5, 1100), 7.0, dtype=torch.bfloat16, device="cuda")
    z = store[:, 1:1004]
    z.copy_(_rows("plain", 5, 1003, torch.bfloat16, 2))
    y = torch.arange(5, dtype=torch.int32, device="cuda")
    _, H, st, _, _ = B.echo_token_logprobs(z, y)
    B.echo_token_logprobs_backward(z, y, H, st, torch.ones(5, device="cuda"), torch.ones(5, device="cuda"), out=z)
    assert bool((store[:, 0] == 7).all()) and bool((store[:, 1004:] == 7).all())


def test_logits_gradient_against_differences(B):
    """The value of the forward call moves by the gradient: central differences in fp32 logits with a step h large
    enough that the forward error of ~1e-6 over 2 h stays below 1e-3, and small enough for the third derivative."""
    z = _rows("plain", 3, 40, torch.float32, 9)
    y = torch.tensor([0, 39, 7], dtype=torch.int32, device="cuda")
    a, b = torch.tensor([1.0, -0.5, 0.3], device="cuda"), torch.tensor([0.2, 0.0, -1.0], device="cuda")

    def value(zz):
        lp, H, *_ = B.echo_token_logprobs(zz, y, 0.9)
        return (a * lp + b * H).double().cpu().numpy()

    _, H, st, _, _ = B.echo_token_logprobs(z, y, 0.9)
    g = B.echo_token_logprobs_backward(z, y, H, st, a, b, 0.9).cpu().numpy()
    h = 2.0 ** -6
    for v in range(0, 40, 3):
        d = torch.zeros_like(z)
        d[:, v] = h
        assert np.all(np.abs((value(z + d) - value(z - d)) / (2 * h) - g[:, v]) < 1e-3)


# ---- objective ----------------------------------------------------------------------------------
@pytest.mark.parametrize("n,T", [(1, 1), (3, 5), (7, 64), (2, 257), (5, 2048), (1, 8191), (33, 100), (300, 260)])
@pytest.mark.parametrize("mask,kl,up", [(True, True, True), (False, True, False), (True, False, True), (False, False, False)])
def test_grpo_gradient(B, n, T, mask, kl, up):
    rng = np.random.default_rng(n * 10007 + T)
    f = lambda *s: rng.normal(size=s).astype(np.float32)  # noqa: E731
    lo = -np.abs(f(n, T)) * 2
    ln, ls, lr = lo + 0.3 * f(n, T), lo + 0.4 * f(n, T), lo + 0.5 * f(n, T)
    ln, ls, lr = (x.astype(np.float32) for x in (ln, ls, lr))
    adv, go = f(n), f(n)
    if n > 2:
        adv[1] = 0
    m = (rng.random((n, T)) < 0.7).astype(np.uint8) * rng.integers(1, 255, size=(n, T)).astype(np.uint8)
    if n > 1:
        m[0] = 0                                           # an empty response
    if n * T > 4:
        ln.flat[1] = np.float32(lo.flat[1])                # rho = 1
    inf = np.where(m == 0)
    lns = ln.copy()
    if mask and len(inf[0]):                               # what the mask leaves out may hold anything
        lns[inf] = np.array([np.nan, np.inf, -np.inf], dtype=np.float32)[np.arange(len(inf[0])) % 3]
    eps, C, beta = 0.2, 1.3, 0.07
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    value, g = B.echo_grpo_gradient(dev(lns if mask else ln), dev(lo), dev(ls), dev(lr) if kl else None, dev(adv),
                                    dev(m) if mask else None, dev(go) if up else None, eps, C, beta)
    eps64, beta64, C64 = (float(np.float32(x)) for x in (eps, beta, C))
    mm = (m != 0).astype(np.uint8) if mask else np.ones((n, T), np.uint8)
    want = L.grpo_gradient(ln, lo, ls, lr if kl else None, adv, mm, go if up else None, eps64, C64, beta64)
    ref = o_obj.grpo_objective(ln, lo, ls, lr if kl else ln, adv, mm, eps64, C64, beta64 if kl else 0.0)
    rho, w = np.exp((ln - lo).astype(np.float64)), np.minimum(np.exp((lo - ls).astype(np.float64)), C64)
    count = np.maximum(mm.sum(axis=1, keepdims=True), 1)
    kl_size = beta64 * (np.exp(np.abs(lr - ln).astype(np.float64)) + np.abs(lr - ln)) if kl else 0.0
    # expf and expm1f are good to 2 steps (4 e), differences of the inputs to e of themselves; a dozen roundings beside
    size = w * (rho * np.abs(adv)[:, None] + kl_size)
    # the differences ln - lo, lo - ls, lr - ln are off by e of themselves, which is below 4 e here (|d| < 4)
    tol = size * E * 24 / count
    got = g.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol * (np.abs(go)[:, None] if up else 1.0) + 1e-40)
    assert np.all(got[mm == 0] == 0)
    sum_tol = (mm * size).sum(axis=1) / count[:, 0] * E * (24 + T / 32 + 16) + 1e-40
    assert np.all(np.abs(value.double().cpu().numpy() - ref) <= sum_tol)


def test_grpo_gradient_next_to_the_borders(B):
    """rho one fp32 step inside and outside the clipping borders: the slope goes by the exact difference."""
    eps = 0.2
    ln, want = [], []
    for A, border in ((1.0, math.log1p(float(np.float32(eps)))), (-1.0, math.log1p(-float(np.float32(eps))))):
        x = np.float32(border)
        for k in (np.nextafter(x, np.float32(-9)), x, np.nextafter(x, np.float32(9))):
            ln.append((A, k))
            want.append(0.0 if (float(k) > border if A > 0 else float(k) < border) else math.exp(float(k)) * A)
    adv = torch.tensor([a for a, _ in ln], device="cuda")
    new = torch.tensor(np.array([[k] for _, k in ln], dtype=np.float32), device="cuda")
    zero = torch.zeros_like(new)
    _, g = B.echo_grpo_gradient(new, zero, zero, None, adv, None, None, eps, 5.0, 0.0)
    got = g[:, 0].double().cpu().numpy()
    assert np.all((got == 0) == (np.array(want) == 0)) and np.allclose(got, want, rtol=8 * E)


def test_grpo_value_equals_the_forward_calls(B):
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    ln, lo, ls, lr, adv = r(9, 700), r(9, 700), r(9, 700), r(9, 700), r(9)
    mask = (torch.rand((9, 700), generator=g, device="cuda") < 0.5).to(torch.uint8)
    v, _ = B.echo_grpo_gradient(ln, lo, ls, lr, adv, mask, None, 0.2, 2.0, 0.05)
    w = B.echo_grpo_objective(ln, lo, ls, lr, adv, mask, 0.2, 2.0, 0.05)
    # two orders of the same fp32 sums of terms of size |term|
    size = (torch.exp(ln - lo).abs() * adv.abs()[:, None] * 2 + 0.1 * torch.exp((lr - ln).abs())).sum(dim=1) / mask.sum(dim=1)
    assert bool(((v - w).abs() <= size * E * 80).all())
    v, _ = B.echo_grpo_gradient(ln, lo, ls, None, adv, mask, None, 0.2, 2.0, 0.05)
    w = B.echo_grpo_surrogate(ln, lo, ls, adv, mask, 0.2, 2.0)
    assert bool(((v - w).abs() <= size * E * 80).all())


# ---- AdamW --------------------------------------------------------------------------------------
SIZES = [1, 255, 256, 257, 3, 2048, 70001, 0, 512, 8]


def _adamw_inputs(sizes, bits, gdtype, seed, offset=0):
    rng = np.random.default_rng(seed)

    def t(x, dtype):
        x = np.asarray(x)
        store = torch.zeros(len(x) + offset, dtype=dtype, device="cuda")
        store[offset:] = torch.from_numpy(x).cuda().to(dtype)
        return store[offset:]

    d = dict(p=[], g=[], m=[], v=[], ms=[], vs=[])
    for n in sizes:
        nb = -(-n // 256)
        d["p"].append(t(rng.normal(size=n) * 0.05, torch.float32))
        g = rng.normal(size=n) * 1e-3 * np.exp(rng.normal(size=n) * 2)
        g[rng.random(n) < 0.1] = 0
        d["g"].append(t(g, gdtype))
        if bits == 32:
            d["m"].append(t(rng.normal(size=n) * 3e-4, torch.float32))
            d["v"].append(t((rng.normal(size=n) * 1e-3) ** 2, torch.float32))
        else:
            d["m"].append(t(rng.integers(-127, 128, n), torch.int8))
            d["v"].append(t(rng.integers(0, 256, n), torch.uint8))
            ms, vs = rng.random(nb) * 1e-3, rng.random(nb) * 1e-6
            if nb > 2:
                ms[1] = vs[1] = 0.0                        # an untouched block
                d["m"][-1][256:512] = 0
                d["v"][-1][256:512] = 0
                d["g"][-1][256:512] = 0
            d["ms"].append(t(ms, torch.float32))
            d["vs"].append(t(vs, torch.float32))
    return d


def _host(ts):
    return [x.detach().double().cpu().numpy() for x in ts]


@pytest.mark.parametrize("gdtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("copy,scale", [(True, 0.37), (False, None)])
def test_adamw_32(B, gdtype, offset, copy, scale):
    d = _adamw_inputs(SIZES, 32, gdtype, 5, offset)
    copies = [torch.zeros(n + 1, dtype=torch.bfloat16, device="cuda")[offset:n + offset] for n in SIZES] if copy else None
    decay = [0.1 if i % 2 else 0.0 for i in range(len(SIZES))]
    before = {k: _host(d[k]) for k in "pgmv"}
    gs = torch.tensor([scale], device="cuda") if scale else None
    plan = B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], copies, decay)
    lr, b1, b2, eps, step = 1e-3, 0.9, 0.99, 1e-8, 3
    B.echo_adamw_step(plan, step, lr, b1, b2, eps, grad_scale=gs)
    for i in range(len(SIZES)):
        p, m, v = (_host([d[k][i]])[0] for k in "pmv")
        s = float(np.float32(scale)) if scale else 1.0
        wp, wm, wv = L.adamw(before["p"][i], before["g"][i], before["m"][i], before["v"][i], step, lr, b1, b2, eps, decay[i], s)
        gg = np.abs(before["g"][i] * s)
        # constants, products and the sum: four roundings for m, six for v (all of its terms are positive)
        assert np.all(np.abs(m - wm) <= 5 * E * (b1 * np.abs(before["m"][i]) + (1 - b1) * gg) + 1e-44)
        assert np.all(np.abs(v - wv) <= 8 * E * wv + 1e-44)
        upd = lr / (1 - b1 ** step) / (np.sqrt(wv / (1 - b2 ** step)) + eps)
        d_m = 5 * E * (b1 * np.abs(before["m"][i]) + (1 - b1) * gg)
        # update: m's own error; quotient, root, product: 12 e; p: constant, product, sum
        assert np.all(np.abs(p - wp) <= upd * (d_m + 14 * E * np.abs(wm)) + 3 * E * np.abs(before["p"][i]) + 1e-44)
        if copy:
            assert torch.equal(copies[i], d["p"][i].to(torch.bfloat16))


@pytest.mark.parametrize("gdtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("seed,step,scale", [(0, 1, None), (0xDEADBEEF12345678, 1000, 2.5)])
def test_adamw_8(B, gdtype, offset, seed, step, scale):
    """Codes and scales are those of the 64-bit definition, exactly."""
    sizes = SIZES + [300_000]
    d = _adamw_inputs(sizes, 8, gdtype, 6, offset)
    before = {k: _host(d[k]) for k in ("p", "g")}
    mv = [L.avg_values(c.cpu().numpy(), s.cpu().numpy()) for c, s in zip(d["m"], d["ms"])]
    vv = [L.sq_values(c.cpu().numpy(), s.cpu().numpy()) for c, s in zip(d["v"], d["vs"])]
    plan = B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], None, 0.02, d["ms"], d["vs"])
    gs = torch.tensor([scale], device="cuda") if scale else None
    lr, b1, b2, eps = 1e-3, 0.9, 0.999, 1e-8
    B.echo_adamw_step(plan, step, lr, b1, b2, eps, grad_scale=gs, seed=seed)
    out_m = [torch.empty(n, device="cuda") for n in sizes]
    out_v = [torch.empty(n, device="cuda") for n in sizes]
    B.echo_adamw_unpack(plan, out_m, out_v)
    for i, n in enumerate(sizes):
        if n == 0:
            continue
        s = scale or 1.0
        wp, wm, wv = L.adamw(before["p"][i], before["g"][i], mv[i], vv[i], step, lr, b1, b2, eps, 0.02, s)
        cm, sm = L.quantise_avg(wm)
        cv, sv = L.quantise_sq(wv, L.halves(n, i, step, seed))
        assert np.array_equal(d["ms"][i].cpu().numpy(), sm) and np.array_equal(d["vs"][i].cpu().numpy(), sv)
        assert np.array_equal(d["m"][i].cpu().numpy(), cm)
        assert np.array_equal(d["v"][i].cpu().numpy(), cv)
        p = _host([d["p"][i]])[0]
        g = np.abs(before["g"][i] * s)
        d_m = 9 * E * (b1 * np.abs(mv[i]) + (1 - b1) * g)
        upd = lr / (1 - b1 ** step) / (np.sqrt(wv / (1 - b2 ** step)) + eps)
        assert np.all(np.abs(p - wp) <= upd * (d_m + 18 * E * np.abs(wm)) + 3 * E * np.abs(before["p"][i]) + 1e-44)
        # values of the codes: five roundings
        assert np.all(np.abs(_host([out_m[i]])[0] - L.avg_values(cm, sm)) <= 6 * E * np.abs(L.avg_values(cm, sm)) + 1e-44)
        assert np.all(np.abs(_host([out_v[i]])[0] - L.sq_values(cv, sv)) <= 10 * E * L.sq_values(cv, sv) + 1e-44)


def test_adamw_8_where_everything_cancels(B):
    """(1 - b1) g = -b1 m up to the last bits in a whole block: fp32's m is mostly rounding, the codes are the 64-bit
    ones all the same.  And blocks that only decay, where every code stays next to itself; and tiny values."""
    n = 256 * 4
    rng = np.random.default_rng(12)
    codes, scales = rng.integers(-127, 128, n).astype(np.int8), np.full(4, 1e-3, dtype=np.float32)
    vcodes, vscales = rng.integers(1, 256, n).astype(np.uint8), np.array([1e-6, 1e-6, 1e-36, 1e-38], dtype=np.float32)
    m, v = L.avg_values(codes, scales), L.sq_values(vcodes, vscales)
    g = (-9.0 * m * (1 + 1e-6 * rng.normal(size=n))).astype(np.float32)
    g[256:512] = 0
    g[512:768] = rng.normal(size=256) * 1e-19
    g[768:] = 0
    dev = lambda x: torch.from_numpy(x.copy()).cuda()  # noqa: E731
    tm, tv, sm, sv, p = dev(codes), dev(vcodes), dev(scales), dev(vscales), torch.zeros(n, device="cuda")
    plan = B.AdamWTensors([p], [dev(g)], [tm], [tv], None, 0.0, [sm], [sv])
    B.echo_adamw_step(plan, 5, 1e-3, seed=77)
    _, wm, wv = L.adamw(np.zeros(n), g, m, v, 5, 1e-3, 0.9, 0.999, 1e-8, 0.0)
    cm, csm = L.quantise_avg(wm)
    cv, csv = L.quantise_sq(wv, L.halves(n, 0, 5, 77))
    assert np.array_equal(sm.cpu().numpy(), csm) and np.array_equal(sv.cpu().numpy(), csv) and csv[3] == 0
    assert np.array_equal(tm.cpu().numpy(), cm) and np.array_equal(tv.cpu().numpy(), cv)
    assert bool(torch.isfinite(p).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_overflowed_step_changes_nothing(B, bits):
    d = _adamw_inputs([1000, 3], bits, torch.float32, 7)
    plan = B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], None, 0.1, d["ms"], d["vs"])
    keep = [x.clone() for k in d for x in d[k]]
    for bad in (float("inf"), float("nan")):
        B.echo_adamw_step(plan, 1, 1e-3, grad_scale=torch.tensor([bad], device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(keep, [x for k in d for x in d[k]]))


def test_adamw_bad_gradient_stays_in_its_block(B):
    d = _adamw_inputs([1024], 8, torch.float32, 8)
    d["g"][0][300] = float("nan")
    plan = B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], None, 0.0, d["ms"], d["vs"])
    B.echo_adamw_step(plan, 1, 1e-3)
    assert torch.isnan(d["ms"][0][1]) and torch.isfinite(d["ms"][0][[0, 2, 3]]).all()
    bad = torch.isnan(d["p"][0])
    assert bad.sum() == 1 and bool(bad[300])


def test_adamw_many_tensors(B):
    """More tensors than one launch holds."""
    sizes = [1 + (i * 37) % 700 for i in range(905)]
    d = _adamw_inputs(sizes, 32, torch.bfloat16, 9)
    before = {k: _host(d[k]) for k in "pgmv"}
    B.echo_adamw_step(B.AdamWTensors(d["p"], d["g"], d["m"], d["v"]), 2, 1e-2)
    for i in (0, 31, 32, 399, 400, 401, 800, 904):
        wp, wm, _ = L.adamw(before["p"][i], before["g"][i], before["m"][i], before["v"][i], 2, 1e-2, 0.9, 0.999, 1e-8, 0.0)
        assert np.allclose(_host([d["m"][i]])[0], wm, rtol=0, atol=5 * E * 0.2)
        assert np.abs(_host([d["p"][i]])[0] - wp).max() < 1e-5
    assert all(not np.array_equal(a, b) for a, b in zip(before["m"], _host(d["m"])))


def test_adamw_8_follows_adamw_32(B):
    """From zero moments over 300 steps of the same noisy gradients: random rounding has no drift, so v keeps its mean.

    Its spread: a step moves v by about 1 - b2 = 0.001 of itself, the codes around it are 4 / c apart (relative), so
    the upper one is taken with probability f = 0.001 c / 4 and a step adds the variance f (4 / c)^2 = 0.004 / c, which
    dies away over 1 / (2 * 0.001) steps: sqrt(2 / c) relative in v, half of that in the update.  Gradient sizes spread
    by exp(N(0, 1)): the codes of the upper half are above c = 255 exp(-2.8 / 2) = 63 (18 % in v), nearly all above 20
    (16 % in an update, whose error keeps its sign for hundreds of steps).  First moment: codes of 127 sqrt(|m| / M)
    above 16 nearly everywhere, rounding 0.29 * 2 / 16 a step, 2.3 times that after the feedback: 8 %, another sign
    every ten steps.  Together below a quarter of p."""
    n = 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    size = torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-3
    p32, p8 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    grad = torch.zeros(n, device="cuda")
    a, b = B.AdamWTensors.zeros([p32], [grad]), B.AdamWTensors.zeros([p8], [grad], state_bits=8)
    for t in range(1, 301):
        grad.copy_(torch.randn(n, generator=g, device="cuda") * size)
        B.echo_adamw_step(a, t, 1e-3)
        B.echo_adamw_step(b, t, 1e-3, seed=5)
    m, v = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    B.echo_adamw_unpack(b, [m], [v])
    ratio = (v / a.exp_avg_sq[0])[size > size.median()]
    assert abs(float(ratio.mean()) - 1) < 0.05 and float(ratio.min()) > 0.5 and float(ratio.max()) < 2
    assert float((p8 - p32).norm() / p32.norm()) < 0.25


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_past_32_bit_offsets(B, bits):
    """The end of one tensor of more than 2^32 elements (bytes of its fp32 arrays: 17 GB each)."""
    n = (1 << 32) + 5 * 256 + 77 if bits == 8 else (1 << 31) + 300
    tail = 256 * 3 + (77 if bits == 8 else 44)
    rng = np.random.default_rng(4)
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-tail:] = torch.from_numpy(rng.normal(size=tail).astype(np.float32)).cuda()
    g[-tail:] = torch.from_numpy(rng.normal(size=tail).astype(np.float32)).cuda().to(torch.bfloat16)
    before = _host([p[-tail:], g[-tail:]])
    plan = B.AdamWTensors.zeros([p], [g], state_bits=bits)
    B.echo_adamw_step(plan, 1, 1e-2, seed=3)
    wp, wm, wv = L.adamw(before[0], before[1], np.zeros(tail), np.zeros(tail), 1, 1e-2, 0.9, 0.999, 1e-8, 0.0)
    # first step: p moves by lr times the sign of g, through a dozen roundings
    assert np.abs(_host([p[-tail:]])[0] - wp).max() <= 3 * E * np.abs(before[0]).max() + 20 * E * 1e-2
    if bits == 8:
        cm, _ = L.quantise_avg(wm)
        octet = (n - tail) // 8                          # the tail starts on a block
        words = L.philox.philox4x32_10(np.arange(octet, octet + (tail + 7) // 8, dtype=np.uint64) & np.uint64(0xFFFFFFFF),
                                       np.arange(octet, octet + (tail + 7) // 8, dtype=np.uint64) >> np.uint64(32), 0, 1, 3, 0)
        half = np.empty((tail + 7) // 8 * 8, dtype=np.int64)
        for j, w in enumerate(words):
            half[2 * j::8], half[2 * j + 1::8] = w & 0xFFFF, w >> 16
        cv, _ = L.quantise_sq(wv, half[:tail])
        assert np.array_equal(plan.exp_avg[0][-tail:].cpu().numpy(), cm)
        assert np.array_equal(plan.exp_avg_sq[0][-tail:].cpu().numpy(), cv)
    else:
        assert np.abs(_host([plan.exp_avg[0][-tail:]])[0] - wm).max() <= 5 * E
    assert bool((p[:-tail][::4097] == 0).all()) and float(p[1 << 30]) == 0
    del p, g, plan
    torch.cuda.empty_cache()


def test_grpo_past_32_bit_offsets(B):
    n, T = 262160, 8200
    x = torch.zeros((n, T), device="cuda")
    adv = torch.randn(n, device="cuda")
    v, grad = B.echo_grpo_gradient(x, x, x, None, adv, None, None, 0.2, 2.0, 0.0)
    # equal policies: the objective is A (a sum of T equal terms in fp32), the gradient A / T
    assert bool(((v - adv).abs() <= adv.abs() * E * (T / 16 + 16)).all())
    for r in (0, n // 2, n - 1):
        assert torch.allclose(grad[r], adv[r] / T, rtol=4 * E, atol=0)
    del x, grad
    torch.cuda.empty_cache()


# ---- streams, graphs, the whole step --------------------------------------------------------------
def test_repeats_are_equal_and_graphs_replay(B):
    z = _rows("few", 40, 30011, torch.bfloat16, 3)
    y = torch.randint(0, 30011, (40,), dtype=torch.int32, device="cuda")
    ga, gb = torch.randn(40, device="cuda"), torch.randn(40, device="cuda")
    ln, lo, ls, adv = torch.randn(4, 300, device="cuda"), torch.randn(4, 300, device="cuda"), torch.randn(4, 300, device="cuda"), torch.randn(4, device="cuda")
    d = _adamw_inputs([5000, 100], 8, torch.bfloat16, 2)
    start = {k: [x.clone() for x in d[k]] for k in d}
    plan = B.AdamWTensors(d["p"], d["g"], d["m"], d["v"], None, 0.1, d["ms"], d["vs"])

    def run():
        f = B.echo_token_logprobs(z, y, 1.0, 20)
        back = B.echo_token_logprobs_backward(z, y, f[1], f[2], ga, gb)
        o = B.echo_grpo_gradient(ln, lo, ls, None, adv, None, None, 0.2, 2.0, 0.0)
        B.echo_adamw_step(plan, 4, 1e-3, seed=9)
        return [*f, back, *o]

    def reset():
        for k in d:
            for x, s in zip(d[k], start[k]):
                x.copy_(s)

    first = run()
    state = [x.clone() for k in d for x in d[k]]
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    assert all(torch.equal(a, b) for a, b in zip(state, [x for k in d for x in d[k]]))
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = run()
    for _ in range(2):
        reset()
        for t in third:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, third))
        assert all(torch.equal(a, b) for a, b in zip(state, [x for k in d for x in d[k]]))


def _engine(B, vocab, P, G, Lp, T, eos_id=-1, **more):
    from paper_2602_02192_b200 import synth
    shape = synth.DecoderShape("small", 2, 128, 2, 1, 64, 256, vocab)
    w = synth.make_weights(shape, 3, device="cuda", std=0.08)
    eng = B.Engine(B.make_config(shape, P, G, Lp, T, eos_id=eos_id, **more))
    eng.echo_load_policy(w, 1)
    eng.echo_wait_policy()
    prompts = torch.from_numpy(synth.make_prompts(P, Lp, vocab, 5)).cuda()
    return shape, w, eng, prompts


@pytest.mark.parametrize("eos", [-1, 7])
def test_score_detail(B, eos, monkeypatch):
    """With as many alternatives as ids the whole distribution comes back: it has to hold the log-probability that
    echo_score gives, sum to 1 and have the entropy that is reported.  (Fixed-order projections: both calls then see the
    same logits, bit for bit.)"""
    monkeypatch.setenv("ECHO_DETERMINISTIC", "1")
    P, G, Lp, T, V = 3, 2, 9, 12, 32
    shape, w, eng, prompts = _engine(B, V, P, G, Lp, T, eos)
    lens = [9, 4, 1]
    tok, lp, _ = eng.echo_rollout(prompts, lens, G, T, 0.8, 11)
    if eos >= 0:
        tok[0, 0, 3] = eos                               # ends early; what follows is not scored
    want, _ = eng.echo_score(prompts, lens, tok, 0.8)
    got, H, ids, top, ver = eng.echo_score_detail(prompts, lens, tok, 0.8, V)
    _, H0, none_ids, none_top, _ = eng.echo_score_detail(prompts, lens, tok, 0.8)
    _, _, ids5, top5, _ = eng.echo_score_detail(prompts, lens, tok, 0.8, 5)
    eng.echo_sync()
    assert none_ids is None and none_top is None and torch.equal(H, H0)
    assert torch.equal(ids5, ids[..., :5]) and torch.equal(top5, top[..., :5]) and np.all(ver == 1)
    want, got, H, ids, top, tk = (x.cpu().numpy() for x in (want, got, H, ids, top, tok))
    assert np.all(np.abs(got - want) <= E * 64 * np.maximum(1, np.abs(want)))       # two kernels, one formula, 32 ids
    live = np.ones((P, G, T), dtype=bool)
    if eos >= 0:
        for p in range(P):
            for g in range(G):
                at = np.nonzero(tk[p, g] == eos)[0]
                if len(at):
                    live[p, g, at[0] + 1:] = False
        assert not live.all()
        assert np.all(got[~live] == 0) and np.all(H[~live] == 0) and np.all(ids[~live] == -1) and np.isneginf(top[~live]).all()
    assert np.all(np.sort(ids[live], axis=-1) == np.arange(V)) and np.all(np.diff(top[live], axis=-1) <= 0)
    prob = np.exp(top[live].astype(np.float64))
    assert np.abs(prob.sum(axis=-1) - 1).max() < E * 64 * 4
    assert np.abs(-(prob * top[live]).sum(axis=-1) - H[live]).max() < E * 64 * 16
    at = (ids == tk[..., None]) & live[..., None]
    assert np.array_equal(at.sum(axis=-1), live.astype(int)) and np.array_equal(top[at], got[live])
    eng.close()


def test_score_detail_refuses_bad_tokens(B):
    shape, w, eng, prompts = _engine(B, 64, 1, 1, 4, 3)
    tok = torch.tensor([[[1, 64, 2]]], dtype=torch.int32, device="cuda")
    eng.echo_score_detail(prompts, [4], tok, 1.0, 2)
    with pytest.raises(B.EchoError) as e:
        eng.echo_sync()
    assert e.value.code == -7
    eng.close()
    shape, w, eng, prompts = _engine(B, 64, 1, 1, 4, 3)
    tok[0, 0, 1], tok[0, 0, 2] = 2, -1                   # the last token is never fed: only the scoring sees it
    eng.echo_score_detail(prompts, [4], tok, 1.0)
    with pytest.raises(B.EchoError) as e:
        eng.echo_sync()
    assert e.value.code == -7
    eng.close()


def test_score_detail_refuses_bad_tokens_when_nothing_else_is_wanted(B):
    shape, w, eng, prompts = _engine(B, 64, 1, 1, 4, 3)
    tok = torch.tensor([[[1, 2, -1]]], dtype=torch.int32, device="cuda")
    lens, versions = np.array([4], dtype=np.int32), np.zeros(1, dtype=np.int64)
    lp = torch.zeros(3, device="cuda")
    torch.cuda.synchronize()
    assert B.lib.echo_score_detail(eng._ctx, prompts.data_ptr(), lens.ctypes.data, 1, 1, 3, 1.0, tok.data_ptr(), 0,
                                   lp.data_ptr(), None, None, None, versions.ctypes.data) == 0
    with pytest.raises(B.EchoError) as e:
        eng.echo_sync()
    assert e.value.code == -7
    eng.close()


def test_one_learner_step(B):
    """Rollout -> rewards -> log-probabilities of the learner's logits -> objective and gradient -> gradient of the
    logits -> gradient of the lm_head -> AdamW -> next snapshot, as a trainer runs it."""
    P, G, Lp, T, V = 4, 4, 8, 17, 500
    shape, w, eng, prompts = _engine(B, V, P, G, Lp, T)
    n, d = P * G, shape.d_model
    hidden = torch.zeros((T - 1, n, d), device="cuda")
    eng.echo_debug_capture(shape.n_layers - 1, dec_out=hidden)
    tok, lp_sampler, ver = eng.echo_rollout(prompts, [Lp] * P, G, T, 1.0, 21)
    eng.echo_sync()
    eng.echo_debug_capture(-1)
    adv = B.echo_group_advantage(torch.rand((P, G), generator=torch.Generator().manual_seed(0)).cuda()).view(n)
    # the learner's own forward: tokens 1..T-1 from the last layer's output
    h = hidden * torch.rsqrt(hidden.pow(2).mean(dim=-1, keepdim=True) + shape.rms_eps) * w["final_norm"].float()
    h = h.transpose(0, 1).reshape(n * (T - 1), d).contiguous()
    y = tok.view(n, T)[:, 1:].reshape(-1).contiguous()
    sampler = lp_sampler.view(n, T)[:, 1:].contiguous()
    master = w["lm_head"].float().contiguous()

    def objective(weight):
        logits = (h.double() @ weight.double().T).float()
        lp, H, st, _, _ = B.echo_token_logprobs(logits, y)
        value, g = B.echo_grpo_gradient(lp.view(n, T - 1), old, sampler, sampler, adv, None, None, 0.2, 2.0, 0.04)
        return logits, lp, H, st, value, g

    old = sampler
    _, lp, _, _, _, _ = objective(master)
    # the learner's logits are the sampler's up to the engine's 16-bit activations
    assert float((lp.view(n, T - 1) - sampler).abs().max()) < 5e-2
    old = lp.view(n, T - 1).clone()
    logits, lp, H, st, value, g = objective(master)
    bonus = torch.full((n * (T - 1),), 0.01, device="cuda")
    dz = B.echo_token_logprobs_backward(logits, y, H, st, g.view(-1), bonus, out=logits)          # in place
    dW = dz.T @ h
    # the gradient against a difference along a random direction: J is smooth here up to the clipping borders at
    # rho = 0.8 and 1.2, far from rho = 1; h = 2^-8 moves a logit by at most 0.03
    step = torch.randn(master.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    s = 2.0 ** -8 / float((h @ step.T).abs().max())
    values = []
    for sign in (1.0, -1.0):
        _, _, H2, _, v2, _ = objective(master + sign * s * step)
        values.append(float(v2.double().sum() + (bonus.double() * H2.double()).sum()))
    slope, want = (values[0] - values[1]) / (2 * s), float((dW.double() * step.double()).sum())
    # values of ~n terms in fp32 (2^-24 each) over 2 s, and the third derivative's s^2
    noise = 2.0 ** -22 * (float(value.abs().sum()) + 0.01 * float(H.sum())) / s
    assert abs(slope - want) <= noise + 1e-3 * float(dz.abs().sum()) * float((h @ step.T).abs().max())
    # update, snapshot, next version
    copy = torch.empty_like(w["lm_head"])
    plan = B.AdamWTensors.zeros([master], [(-dW).to(torch.bfloat16)], state_bits=8, copies=[copy])
    norm = dW.norm()
    before = master.clone()
    B.echo_adamw_step(plan, 1, 1e-3, grad_scale=(1.0 / norm.clamp(min=1.0)).view(1), seed=1)
    assert torch.equal(copy, master.to(torch.bfloat16)) and float((master - before).abs().max()) <= 1.01e-3
    assert float(((master - before) * dW).sum()) > 0                       # uphill
    w2 = dict(w)
    w2["lm_head"] = copy
    eng.echo_load_policy(w2, 2)
    eng.echo_wait_policy()
    lp2, ver2 = eng.echo_score(prompts, [Lp] * P, tok, 1.0)
    eng.echo_sync()
    assert np.all(ver == 1) and np.all(ver2 == 2)
    _, lp_learner, *_ = objective(copy.float())
    # hidden states are the same; the engine multiplies 16-bit activations
    assert float((lp2.view(n, T)[:, 1:].reshape(-1) - lp_learner).abs().max()) < 5e-2
    eng.close()
