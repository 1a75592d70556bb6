"""Pins of the learner-side oracle, and the refusals of the library's learner entry points (no GPU needed)."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from oracle import learner as L
from oracle import objective


def test_uniform_and_two_valued_rows():
    V = 37
    lp, H, st, ids, top = L.token_logprobs(np.full((1, V), 3.25), np.array([5]), 0.7, 4)
    assert abs(lp[0] + math.log(V)) < 1e-14 and abs(H[0] - math.log(V)) < 1e-14
    assert st[0, 0] == 3.25 and abs(st[0, 1] - math.log(V)) < 1e-14
    assert ids[0].tolist() == [0, 1, 2, 3] and np.allclose(top[0], -math.log(V))
    z = np.array([[0.0, math.log(3.0)]])                 # probabilities 1/4, 3/4
    lp, H, _, ids, _ = L.token_logprobs(z, np.array([0]), 1.0, 3)
    assert abs(lp[0] - math.log(0.25)) < 1e-15
    assert abs(H[0] + 0.25 * math.log(0.25) + 0.75 * math.log(0.75)) < 1e-15
    assert ids[0].tolist() == [1, 0, -1]


def test_masked_and_empty_rows():
    z = np.array([[-np.inf, 1.0, 1.0, -np.inf], [-np.inf] * 4, [np.nan, 0.0, 0.0, 0.0]])
    lp, H, st, ids, top = L.token_logprobs(z, np.array([0, 2, 1]), 1.0, 3)
    assert lp[0] == -np.inf and abs(H[0] - math.log(2)) < 1e-15 and ids[0].tolist() == [1, 2, -1]
    assert lp[1] == -np.inf and H[1] == 0 and ids[1].tolist() == [-1] * 3 and np.isneginf(st[1]).all()
    assert np.isnan(lp[2]) and np.isnan(H[2]) and ids[2].tolist() == [1, 2, 3]
    g = L.token_logprobs_backward(z[:2], np.array([1, 2]), 1.0, np.ones(2), np.ones(2))
    assert g[0, 0] == 0 and np.all(g[1] == 0)


def test_logits_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    R, V, T = 4, 11, 0.8
    z, a, b = rng.normal(size=(R, V)), rng.normal(size=R), rng.normal(size=R)
    y = np.array([3, -1, 0, 10])

    def value(zz):
        lp, H, *_ = L.token_logprobs(zz, y, T)
        return float(np.sum(a * lp) + np.sum(b * H))

    g = L.token_logprobs_backward(z, y, T, a, b)
    for r in range(R):
        for v in range(V):
            d = np.zeros_like(z)
            d[r, v] = 1e-5
            assert abs((value(z + d) - value(z - d)) / 2e-5 - g[r, v]) < 1e-8


def test_objective_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(4)
    n, T = 5, 9
    ln, lo, ls, lr = (-np.abs(rng.normal(size=(n, T))) for _ in range(4))
    adv, up = rng.normal(size=n), rng.normal(size=n)
    mask = (rng.random((n, T)) < 0.6).astype(np.uint8)
    mask[2] = 0
    g = L.grpo_gradient(ln, lo, ls, lr, adv, mask, up, 0.2, 1.5, 0.1)
    assert np.all(g[mask == 0] == 0)
    for i in range(n):
        for t in range(T):
            d = np.zeros_like(ln)
            d[i, t] = 1e-6
            f = [np.sum(up * objective.grpo_objective(ln + s * d, lo, ls, lr, adv, mask, 0.2, 1.5, 0.1)) for s in (1, -1)]
            assert abs((f[0] - f[1]) / 2e-6 - g[i, t]) < 1e-7


def test_codes_reproduce_their_own_values():
    codes = np.arange(-127, 128).astype(np.int8)
    scale = np.array([0.125], dtype=np.float32)
    back, s = L.quantise_avg(L.avg_values(codes, scale))
    assert np.array_equal(back, codes) and s[0] == scale[0]
    codes = np.arange(256).astype(np.uint8)
    for half in (0, 32768, 65535):                       # a value that is a code's is not moved by the random number,
        back, s = L.quantise_sq(L.sq_values(codes, scale), np.full(256, half))
        far = np.abs(back.astype(int) - codes.astype(int))
        assert s[0] == scale[0] and far.max() <= 1       # up to the last bit of the 64-bit quotient
        if half == 32768:
            assert far.max() == 0
    assert L.quantise_avg(np.zeros(300))[1].tolist() == [0, 0]


def test_random_rounding_keeps_the_mean():
    v = np.full(256, 3.3e-7)
    v[0] = 1e-5                                          # the block's largest
    half = np.arange(65536)
    sums = np.zeros(256)
    for i in range(0, 65536, 64):
        c, s = L.quantise_sq(v, np.full(256, half[i]))
        sums += L.sq_values(c, s)
    # 1024 equidistant random numbers: the mean is off by at most a 1024th of the distance of the two codes
    c, _ = L.quantise_sq(v, np.zeros(256))
    step = np.float64(np.float32(1e-5)) * (((c[1] + 1) / 255) ** 4 - ((c[1] - 1) / 255) ** 4)
    assert abs(sums[1] / 1024 - 3.3e-7) <= step / 1024
    tiny = np.full(256, 1e-30)
    tiny[0] = 1.0
    assert L.quantise_sq(tiny, np.full(256, 65535))[0][1] == 1            # never lost


def test_halves_are_the_philox_words():
    from oracle import philox
    h = L.halves(20, 3, 7, 0x123456789ABCDEF0)
    w = philox.philox4x32_10(1, 0, 3, 7, 0x9ABCDEF0, 0x12345678)
    assert h[8] == int(w[0]) & 0xFFFF and h[9] == int(w[0]) >> 16 and h[15] == int(w[3]) >> 16 and len(h) == 20


def test_adamw_by_hand():
    p, m, v = L.adamw([1.0], [0.5], [0.0], [0.0], 1, 0.1, 0.9, 0.999, 1e-8, 0.01)
    assert abs(m[0] - 0.05) < 1e-15 and abs(v[0] - 0.00025) < 1e-15
    assert abs(p[0] - (1.0 - 0.001 - 0.1 * 0.5 / (0.5 + 1e-8))) < 1e-12      # first step: m_hat = g, v_hat = g^2


# ---- refusals: every one is decided on the host, before anything is launched -------------------
INVALID, UNSUPPORTED = -1, -9
P0, P1 = 1 << 20, 1 << 24                               # addresses that nothing reads


def _lib():
    from paper_2602_02192_b200 import binding
    return binding, binding.lib


def _forward(**over):
    b, lib = _lib()
    a = dict(logits=P0, fmt=0, stride=100, R=4, V=100, tokens=P1, T=1.0, k=0, lp=P1, ent=P1, stats=P1, ids=None, top=None)
    a.update(over)
    return lib.echo_token_logprobs(*a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(logits=None), INVALID), (dict(fmt=3), INVALID), (dict(fmt=-1), INVALID), (dict(stride=99), INVALID),
    (dict(R=-1), INVALID), (dict(V=0), INVALID), (dict(T=0.0), INVALID), (dict(T=-1.0), INVALID),
    (dict(T=float("nan")), INVALID), (dict(T=float("inf")), INVALID), (dict(T=1e-39), INVALID), (dict(tokens=None), INVALID),
    (dict(lp=None), INVALID), (dict(k=-1), INVALID), (dict(k=5), INVALID), (dict(k=5, ids=P1), INVALID),
    (dict(k=33, ids=P1, top=P1), UNSUPPORTED), (dict(stats=P1 + 4), INVALID), (dict(logits=P0 + 1), INVALID),
    (dict(fmt=2, logits=P0 + 2), INVALID), (dict(tokens=None, lp=None, ent=None, stats=None), INVALID),
    (dict(V=(1 << 24) + 1, stride=1 << 31), UNSUPPORTED), (dict(R=1 << 30), UNSUPPORTED)])
def test_token_logprobs_refusals(over, code):
    assert _forward(**over) == code


def test_nothing_to_do_is_fine():
    b, lib = _lib()
    assert _forward(R=0, logits=None) == 0
    assert lib.echo_grpo_gradient(P0, P0, P0, None, P0, None, None, 0, 5, 0.2, 1.0, 0.0, None, P1, None) == 0
    opt = b.EchoAdamWOptions(1e-3, 0.9, 0.99, 1e-8, 1, 0, None, 2, 32)
    assert lib.echo_adamw_step(None, 0, C.byref(opt), None) == 0


def _backward(**over):
    b, lib = _lib()
    a = dict(logits=P0, fmt=0, stride=100, R=4, V=100, tokens=P1, T=1.0, ent=P1, stats=P1, ga=P1, gb=P1, out=P1, ostride=100)
    a.update(over)
    return lib.echo_token_logprobs_backward(*a.values(), None)


@pytest.mark.parametrize("over", [
    dict(logits=None), dict(out=None), dict(stats=None), dict(stats=P1 + 4), dict(ostride=99), dict(stride=99),
    dict(ga=None, gb=None), dict(tokens=None), dict(ent=None), dict(fmt=3), dict(T=0.0), dict(out=P1 + 1),
    dict(out=P0 + 2), dict(out=P0 + 798), dict(out=P0, ostride=101), dict(out=P0 - 200)])
def test_token_logprobs_backward_refusals(over):
    assert _backward(**over) == INVALID


@pytest.mark.parametrize("change", ["new", "old", "sampler", "adv", "grad", "n", "T", "eps", "C", "beta"])
def test_grpo_gradient_refusals(change):
    b, lib = _lib()
    a = dict(new=P0, old=P0, sampler=P0, ref=P0, adv=P0, mask=None, up=None, n=2, T=3, eps=0.2, C=1.0, beta=0.1, out=None, grad=P1)
    a[change] = {"n": -1, "T": 0, "eps": -0.1, "C": 0.0, "beta": float("nan")}.get(change)
    assert lib.echo_grpo_gradient(*a.values(), None) == INVALID


def test_grpo_gradient_lengths():
    b, lib = _lib()
    call = lambda p, n, T: lib.echo_grpo_gradient(p, p, p, None, p, None, None, n, T, 0.2, 1.0, 0.0, None, p, None)  # noqa: E731
    assert call(None, 0, 5) == 0                          # empty tensors have no address
    assert call(P0, 1, (1 << 30) + 1) == UNSUPPORTED


def _adamw(bits=32, n_tensors=1, entry=None, second=None, **options):
    b, lib = _lib()
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, grad_scale=None, grad_format=2, state_bits=bits)
    o.update(options)
    table = (b.EchoAdamWTensor * 2)()
    for i, over in enumerate((entry, second)):
        base = P0 + i * (1 << 22)
        e = dict(param=base, grad=base + (1 << 16), exp_avg=base + (2 << 16), exp_avg_sq=base + (3 << 16),
                 avg_scales=base + (4 << 16), sq_scales=base + (5 << 16), param_copy=None, n=1000, weight_decay=0.1)
        e.update(over or {})
        for k, v in e.items():
            setattr(table[i], k, v)
    opt = b.EchoAdamWOptions(*o.values())
    return lib.echo_adamw_step(table, n_tensors, C.byref(opt), None)


@pytest.mark.parametrize("options", [
    dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=float("nan")),
    dict(eps=0.0), dict(eps=1e-60), dict(step=0), dict(step=1 << 32), dict(grad_format=3), dict(state_bits=16),
    dict(n_tensors=-1), dict(grad_scale=P1 + 2)])
def test_adamw_option_refusals(options):
    assert _adamw(**options) == INVALID


@pytest.mark.parametrize("entry,bits", [
    (dict(param=None), 32), (dict(grad=None), 32), (dict(exp_avg=None), 32), (dict(exp_avg_sq=None), 32), (dict(n=-1), 32),
    (dict(param=P0 + 2), 32), (dict(exp_avg=P0 + (2 << 16) + 1), 32), (dict(param_copy=P0 + (6 << 16) + 1), 32),
    (dict(avg_scales=None), 8), (dict(sq_scales=None), 8), (dict(weight_decay=-0.1), 32), (dict(weight_decay=float("nan")), 32),
    (dict(exp_avg=P0), 32), (dict(exp_avg_sq=P0 + (2 << 16) + 3996), 32), (dict(grad=P0 + 3996), 32),
    (dict(param_copy=P0 + 2000), 32), (dict(avg_scales=P0 + (5 << 16) + 12), 8)])
def test_adamw_entry_refusals(entry, bits):
    assert _adamw(bits=bits, entry=entry) == INVALID


def test_adamw_8_wants_an_ordinary_eps():
    assert _adamw(bits=8, eps=1e-13) == UNSUPPORTED


def test_adamw_refuses_a_tensor_listed_twice():
    twice = dict(param=P0)
    assert _adamw(n_tensors=2, second=twice) == INVALID


def test_adamw_unpack_refusals():
    b, lib = _lib()
    table = (b.EchoAdamWTensor * 1)()
    table[0].n, table[0].exp_avg, table[0].exp_avg_sq, table[0].avg_scales, table[0].sq_scales = 10, P0, P0, P0, P0
    out = (C.c_void_p * 1)(P1)
    none = (C.c_void_p * 1)(None)
    odd = (C.c_void_p * 1)(P1 + 2)
    assert lib.echo_adamw_unpack(table, 1, none, out, None) == INVALID
    assert lib.echo_adamw_unpack(table, 1, out, odd, None) == INVALID
    assert lib.echo_adamw_unpack(None, 1, out, out, None) == INVALID
    table[0].avg_scales = None
    assert lib.echo_adamw_unpack(table, 1, out, out, None) == INVALID


def test_adamw_unpack_refuses_overlaps():
    b, lib = _lib()
    table = (b.EchoAdamWTensor * 1)()
    table[0].n, table[0].exp_avg, table[0].exp_avg_sq, table[0].avg_scales, table[0].sq_scales = 10, P0, P0 + 64, P0 + 128, P0 + 192
    call = lambda m, v: lib.echo_adamw_unpack(table, 1, (C.c_void_p * 1)(m), (C.c_void_p * 1)(v), None)  # noqa: E731
    assert call(P1, P1) == INVALID and call(P1, P1 + 36) == INVALID           # the outputs with one another
    assert call(P0 + 8, P1) == INVALID and call(P1, P0 + 192) == INVALID      # with the codes, with a scale


def test_score_detail_refusals_come_first():
    b, lib = _lib()
    f = lambda k, ids, top: lib.echo_score_detail(None, P0, P0, 1, 1, 1, 1.0, P0, k, P1, None, ids, top, P1)  # noqa: E731
    assert f(-1, None, None) == INVALID and f(3, None, P1) == INVALID and f(33, P1, P1) == UNSUPPORTED
    assert f(0, None, None) == INVALID                    # no context


def test_new_struct_layouts_match_the_header(tmp_path):
    import os
    import subprocess
    b, _ = _lib()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {"echo_adamw_tensor": b.EchoAdamWTensor, "echo_adamw_options": b.EchoAdamWOptions}
    lines = []
    for name, cls in fields.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "echo.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    out = dict(x.split() for x in subprocess.check_output([str(exe)], text=True).splitlines())
    for name, cls in fields.items():
        assert int(out[name]) == C.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(out[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)


# ---- first moments of 8 bits, rounded at random ---------------------------------------------------
def test_random_rounding_of_first_moments_keeps_the_mean_and_the_codes():
    scale = np.array([0.125], dtype=np.float32)
    codes = np.arange(-127, 128).astype(np.int8)
    for half in (0, 32768, 65535):
        back, s = L.quantise_avg(L.avg_values(codes, scale), np.full(255, half))
        assert np.array_equal(back, codes) and s[0] == scale[0]
    m = np.full(256, -3.3e-7)
    m[0] = 1e-4                                          # the block's largest
    sums = np.zeros(256)
    for half in range(0, 65536, 64):
        c, s = L.quantise_avg(m, np.full(256, half))
        assert c[0] == 127
        sums += L.avg_values(c, s)
    # 1024 equidistant random numbers: the mean is off by at most a 1024th of the distance of the two codes; 127^2 times
    # 3.3e-3 is 53, between 7^2 and 8^2, which are 15 / 127^2 of the largest apart
    assert abs(sums[1] / 1024 + 3.3e-7) <= 15 * 1e-4 / 127 ** 2 / 1024 * 1.01
    assert not np.array_equal(L.halves(64, 1, 2, 3, 1), L.halves(64, 1, 2, 3))


def _mean_drift(random_avg, steps, beta2):
    """Mean distance, in lr, from exact AdamW of elements (one in 16) whose gradient is 0 after step 50."""
    n, lr = 1024, 1e-3
    rng, dead = np.random.default_rng(0), np.arange(n) % 16 == 0
    z8, zs = np.zeros(n), np.zeros(n // 256, np.float32)
    p, c, s, vc, vs = z8, z8.astype(np.int8), zs, z8.astype(np.uint8), zs
    q, m, v = z8, z8, z8
    for t in range(1, steps + 1):
        g = rng.normal(size=n) * 1e-3
        if t > 50:
            g[dead] = 0
        p, m8, v8 = L.adamw(p, g, L.avg_values(c, s), L.sq_values(vc, vs), t, lr, 0.9, beta2, 1e-8, 0.0)
        c, s = L.quantise_avg(m8, L.halves(n, 0, t, 1, 1) if random_avg and t > 1 else None)
        vc, vs = L.quantise_sq(v8, L.halves(n, 0, t, 1))
        q, m, v = L.adamw(q, g, m, v, t, lr, 0.9, beta2, 1e-8, 0.0)
    return np.abs(p - q)[dead].mean() / lr


def test_first_moments_rounded_at_random_fall_when_the_gradient_ends():
    """Codes around 60 lose 1.7 % a step to rounding, 2.3 times that after the feedback, over 50 steps of updates of 0.6 lr
    whose errors keep their sign for ten: 0.7 lr; second moments (codes around 180, 3.5 % after the feedback) 0.5 lr.
    After the end the moment falls by 0.9 / sqrt(0.95) a step: 12 updates are left, of which the steps at codes below 7,
    where a rounding is of the order of the moment itself, are 4 %.  About 1 lr together.  Nearest codes up to 9 stay."""
    assert _mean_drift(True, 400, 0.95) < 2.0
    assert _mean_drift(False, 400, 0.95) > 100.0


def test_adamw_state_bits():
    random_avg = 256
    assert _adamw(state_bits=32 | random_avg) == INVALID and _adamw(state_bits=8 | 512) == INVALID
    assert _adamw(state_bits=random_avg) == INVALID and _adamw(state_bits=16 | random_avg) == INVALID
    assert _adamw(state_bits=8 | random_avg, eps=1e-13) == UNSUPPORTED
    assert _adamw(state_bits=8 | random_avg, entry=dict(avg_scales=None)) == INVALID
    assert _adamw(state_bits=8 | random_avg, entry=dict(avg_scales=P0 + (5 << 16) + 12)) == INVALID      # overlap
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "echo.h")
    with open(header) as f:
        assert f"#define ECHO_ADAMW_RANDOM_AVG {random_avg}" in f.read()
    assert _lib()[0].ECHO_ADAMW_RANDOM_AVG == random_avg


# ---- the handle of an AdamW step (no GPU: stand-ins for device tensors) ----------------------------
class _Memory:
    pass


class _Tensor:
    is_cuda, is_leaf, grad, device = True, True, None, "cuda:0"

    def __init__(self, address, numel=10, dtype=None):
        import torch
        self.address, self.n, self.dtype, self.memory = address, numel, dtype or torch.float32, _Memory()

    def numel(self):
        return self.n

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return True

    def untyped_storage(self):
        return self.memory


def test_adamw_handle_keeps_what_its_addresses_point_to():
    import gc
    import weakref
    b, _ = _lib()
    lists = [[_Tensor(P0 + 4096 * (2 * i + j)) for j in range(2)] for i in range(4)]
    tensors = [weakref.ref(x) for xs in lists for x in xs]
    memory = [weakref.ref(x.memory) for xs in lists for x in xs]
    plan = b.AdamWTensors(*lists)
    for xs in lists:                                      # the caller's lists move on, and so does a tensor's memory
        xs[1].memory = _Memory()
        xs.clear()
    del lists, xs
    gc.collect()
    assert all(r() is not None for r in tensors) and all(r() is not None for r in memory)
    assert plan.table[1].grad == P0 + 4096 * 3
    del plan
    gc.collect()
    assert all(r() is None for r in tensors) and all(r() is None for r in memory)


def test_adamw_handle_notices_other_gradients(monkeypatch):
    """A backward pass after zero_grad(set_to_none=True) makes new gradients: the step must not apply the old ones again."""
    b, _ = _lib()
    params = [_Tensor(P0 + 4096 * i) for i in range(2)]
    grads = [_Tensor(P1 + 4096 * i) for i in range(2)]
    moments = [[_Tensor(P1 + (k << 16) + 4096 * i) for i in range(2)] for k in (1, 2)]
    for p, g in zip(params, grads):
        p.grad = g
    plan = b.AdamWTensors(params, grads, *moments)
    launched = []
    monkeypatch.setattr(b, "_call", lambda *a: launched.append([plan.table[i].grad for i in range(2)]))
    plan.device = type("Device", (), {"index": 0})()
    b.echo_adamw_step(plan, 1, 1e-3)
    params[1].grad = None                                  # zero_grad
    with pytest.raises(RuntimeError):
        b.echo_adamw_step(plan, 2, 1e-3)
    fresh = params[1].grad = _Tensor(P1 + (9 << 16))       # the next backward pass
    with pytest.raises(RuntimeError):
        b.echo_adamw_step(plan, 2, 1e-3)
    plan.device = "cuda:0"
    plan.set_grads([p.grad for p in params])
    plan.device = type("Device", (), {"index": 0})()
    b.echo_adamw_step(plan, 2, 1e-3)
    assert launched == [[P1, P1 + 4096], [P1, fresh.address]]
    plan.device = "cuda:0"
    import torch
    for bad in ([grads[0]], [grads[0], _Tensor(P1, 11)], [grads[0], _Tensor(P1, dtype=torch.bfloat16)], [grads[0], _Tensor(P1, dtype=torch.int32)]):
        with pytest.raises(AssertionError):
            plan.set_grads(bad)
    assert [plan.table[i].grad for i in range(2)] == [P1, fresh.address]
    # gradients that are not the params' own (pieces of a flat buffer, say) are the caller's to keep up to date
    params[0].grad = None
    plan.set_grads([_Tensor(P1), _Tensor(P1 + 4096)])
    plan.device = type("Device", (), {"index": 0})()
    b.echo_adamw_step(plan, 3, 1e-3)
    assert launched[-1] == [P1, P1 + 4096]
