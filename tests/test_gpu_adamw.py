"""adamw_step against its formula in 64 bits, and the 8-bit moments against a bit-exact restatement of their code."""
import math

import numpy as np
import pytest
import torch

from paper_2312_08728_b200 import operators as ops

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
M32 = 0xFFFFFFFF
SIZES = [1, 3, 255, 256, 257, 1000, 4096, 70001]


def mix(x):
    x = np.asarray(x, dtype=np.uint32).copy()
    x ^= x >> np.uint32(16); x *= np.uint32(0x85EBCA6B)
    x ^= x >> np.uint32(13); x *= np.uint32(0xC2B2AE35)
    return x ^ (x >> np.uint32(16))


def random_bits(seed, t, index, n):
    key = mix(np.uint32((seed + t * 0x9E3779B9) & M32))
    key = mix(key ^ np.uint32(((seed >> 32) + index * 0x9E3779B9) & M32))
    return mix(np.arange(n, dtype=np.uint32) ^ key)


def blocks(x):
    n = -(-len(x) // 256) * 256
    return np.concatenate([x, np.zeros(n - len(x), x.dtype)]).reshape(-1, 256)


def exponents(x, least):
    a = np.abs(blocks(x))
    return np.maximum(np.where(np.isfinite(a), a, np.float32(0)).max(axis=1).view(np.uint32) >> 23, least).astype(np.int64)


def code_values_m():
    """Every e4m3 code's value before scaling, NaN for the two that are none."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 7.0), f / 8 * 2.0 ** -6)
    return np.where((c & 127) == 127, np.nan, np.where(c > 127, -v, v))


def code_values_v():
    c = np.arange(256)
    return np.where(c == 0, 0.0, np.where(c == 255, np.nan, (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 30.0)))


def expect_codes(x, table, scale_exp, r16):
    """Code of each value: the neighbour below, or above with the probability that keeps the mean (16 random bits)."""
    values = table[:127] if np.isnan(table[127]) else table[:255]
    a = np.abs(x.astype(np.float64)) * 2.0 ** -scale_exp.astype(np.float64)
    low = np.searchsorted(values, a, side="right") - 1
    gap = values[np.minimum(low + 1, len(values) - 1)] - values[low]
    # drawn up when the fraction of the gap, in units of 2^-16 plus the draw, reaches one gap
    return low, (a - values[low]) / np.where(gap > 0, gap, 1) + r16 / 65536.0 >= 1.0


class Job:
    def __init__(self, sizes, param, grad, bits, master, seed=0, shift=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def make(scale, dtype):
            out = []
            for n in sizes:  # `shift` values into an allocation: not on a 16-byte boundary
                x = torch.randn(n + shift, generator=gen, device="cuda") * scale * torch.exp2(torch.randint(-8, 5, (n + shift,), generator=gen, device="cuda").float())
                out.append(x.to(dtype)[shift:])
            return out
        self.sizes = sizes
        self.masters = make(0.1, torch.float32) if master else None
        self.params = [x.to(param) for x in self.masters] if master else make(0.1, param)
        self.grads = make(0.01, grad)
        self.state = ops.adamw_state(self.params, bits)
        self.bits, self.seed, self.t = bits, 0x123456789AB + seed, 0
        self.decays = [0.0 if i % 3 == 1 else 0.05 for i in range(len(sizes))]
        if bits == 32 and shift:
            for k in ("m", "v"):
                self.state[k] = [torch.zeros(n + shift, device="cuda")[shift:] for n in sizes]

    def before(self):
        """Everything the next update reads, in 64 bits."""
        if self.bits == 8:
            mv = [ops.decode_moments(m, a, v, b) for m, a, v, b in zip(*(self.state[k] for k in ("m", "m_scale", "v", "v_scale")))]
        else:
            mv = list(zip(self.state["m"], self.state["v"]))
        theta = self.masters or self.params
        return [(p.double().clone(), g.double(), m.double().clone(), v.double().clone()) for p, g, (m, v) in zip(theta, self.grads, mv)]

    def step(self, **kw):
        kw = dict(dict(lr=1e-2, weight_decay=self.decays), **kw)
        ops.adamw_step(self.params, self.grads, self.state["m"], self.state["v"], self.state["control"],
                       m_scale=self.state.get("m_scale"), v_scale=self.state.get("v_scale"), masters=self.masters, seed=self.seed, **kw)

    def check(self, before, lr=1e-2, a=0.9, b=0.999, eps=1e-8, gscale=1.0, step32=None):
        self.t += 1
        c1, c2 = 1 - a ** self.t, 1 - b ** self.t
        for i, (p, g, m, v) in enumerate(before):
            g = g * gscale
            m1, v1 = a * m + (1 - a) * g, b * v + (1 - b) * g * g
            em = 4 * E32 * (a * m.abs() + (1 - a) * g.abs()) + 2.0 ** -148
            ev = 6 * E32 * v1 + 2.0 ** -140
            denom = torch.sqrt(v1 / c2) + eps
            move = lr / c1 * m1 / denom
            q = p * (1 - lr * self.decays[i]) - move
            # in units of 2^-24: v's error halved by the root 3, the root 2, its factor and that factor's rounding 2, the sum
            # with eps 1, the quotient 4, the product with the step length and that one's rounding 2: 14, and second-order terms
            eq = 4 * E32 * p.abs() + move.abs() * 15 * E32 + lr / c1 * em / denom + 2 * E32 * q.abs()
            got = (self.masters or self.params)[i]
            if got.dtype == torch.bfloat16:  # rounded at random: less than one step of bf16, at most 2^-7 of the value
                eq = eq + 2.0 ** -7 * (q.abs() + eq) + 2.0 ** -130
            assert bool(((got.double() - q).abs() <= eq).all()), (i, float((got.double() - q).abs().max()))
            if self.masters:
                want = self.masters[i].to(self.params[i].dtype)
                assert torch.equal(self.params[i], want)
            if self.bits == 32:
                assert bool(((self.state["m"][i].double() - m1).abs() <= em).all())
                assert bool(((self.state["v"][i].double() - v1).abs() <= ev).all())


KINDS = [(torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, False), (torch.bfloat16, torch.bfloat16, False),
         (torch.bfloat16, torch.float32, True), (torch.float16, torch.float16, True), (torch.bfloat16, torch.bfloat16, True)]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{str(k[0])[6:]}-{str(k[1])[6:]}{'-copy' if k[2] else ''}")
def test_update(kind, bits, shift):
    job = Job(SIZES, *kind[:2], bits, kind[2], seed=bits + shift, shift=shift)
    for _ in range(4):
        before = job.before()
        job.step()
        job.check(before)
        for g in job.grads:
            g.mul_(-0.7)
    assert job.state["control"].tolist()[:3] == [4, 0, 0]


def test_moments_in_8_bits_bit_for_bit():
    """The codes and scales of the new moments, from the fp32 moments rounded as stated and the hashed bits."""
    job = Job([5, 256, 3000, 40000], torch.float32, torch.float32, 8, False, seed=3)
    job.grads[2][7] = 0.0
    job.grads[2][256:512] = 0.0
    job.grads[1][9] = 1e-30
    f = np.float32
    a, b, a1, b1 = f(0.9), f(0.999), f(1 - 0.9), f(1 - 0.999)
    old = None
    for t in range(1, 5):
        old = [tuple(x.cpu().numpy() for x in ops.decode_moments(m, s, v, r)) for m, s, v, r in
               zip(*(job.state[k] for k in ("m", "m_scale", "v", "v_scale")))]
        job.step()
        for i, (m, v) in enumerate(old):
            g = job.grads[i].cpu().numpy()
            m1, v1 = m * a + g * a1, v * b + (g * b1) * g
            r = random_bits(job.seed, t, i, len(g))
            sm, sv = exponents(m1, 16), exponents(v1, 40)
            assert np.array_equal(job.state["m_scale"][i].cpu().numpy(), sm) and np.array_equal(job.state["v_scale"][i].cpu().numpy(), sv)
            got = job.state["m"][i].view(torch.uint8).cpu().numpy().astype(np.int64)
            low, up = expect_codes(m1, code_values_m(), np.repeat(sm, 256)[:len(g)] - 134, r & 0xFFFF)
            assert np.array_equal(got & 127, low + up)
            signed = (got & 127) > 0
            assert np.array_equal((got > 127)[signed], (m1 < 0)[signed])
            got = job.state["v"][i].cpu().numpy().astype(np.int64)
            low, up = expect_codes(v1, code_values_v(), np.repeat(sv, 256)[:len(g)] - 127, r >> np.uint32(16))
            want = np.where((low == 0) & (v1 > 0), 1, low + up)  # never down to zero
            assert np.array_equal(got, want)


@pytest.mark.parametrize("param,grad", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_moments_in_8_bits_do_not_depend_on_alignment(param, grad):
    """A sum of products rounded once instead of twice would show in a code of some millions: the forms for aligned and for
    other tensors agree in all of 2^24."""
    n = 1 << 24
    gen = torch.Generator(device="cuda").manual_seed(6)
    p = (torch.randn(n, generator=gen, device="cuda") * 0.1).to(param)
    grads = [(torch.randn(n, generator=gen, device="cuda") * torch.exp2(torch.randint(-6, 6, (n,), generator=gen, device="cuda").float())).to(grad) for _ in range(3)]

    def moved(t):
        out = torch.zeros(n + 1, dtype=t.dtype, device="cuda")[1:]
        out.copy_(t)
        return out
    states = [ops.adamw_state([p], 8) for _ in range(2)]
    params = [p.clone(), moved(p)]
    for g in grads:
        ops.adamw_step([params[0]], [g], lr=1e-3, seed=4, **states[0])
        ops.adamw_step([params[1]], [moved(g)], lr=1e-3, seed=4, **states[1])
        for k in ("m", "v", "m_scale", "v_scale"):
            a, b = (s[k][0].view(torch.uint8) for s in states)
            assert torch.equal(a, b), (k, int((a != b).sum()))


def test_moments_in_8_bits_keep_their_mean():
    """A constant gradient: v must approach its square and m the gradient, although every change is below half a step."""
    n, steps = 1 << 16, 1500
    p, g = [torch.zeros(n, device="cuda")], [torch.full((n,), 0.01, device="cuda")]
    s = ops.adamw_state(p, 8)
    for t in range(steps):
        ops.adamw_step(p, g, lr=0.0, seed=11, **s)
    m, v = ops.decode_moments(s["m"][0], s["m_scale"][0], s["v"][0], s["v_scale"][0])
    # Between updates a value sits on one of the two codes beside the true one, at most 1/8 of the value apart, so the mean
    # of 65,536 has a deviation of at most 1/16 / 256.  The draw has 16 bits: each update rounds down by at most 2^-16 of
    # a step too much, 1/(1-b) of which are remembered: 1000 * 2^-16 / 8 = 0.2 % of v, and far less of m.
    want_v = 1e-4 * (1 - 0.999 ** steps)
    assert abs(float(v.double().mean()) / want_v - 1) < 0.005
    assert abs(float(m.double().mean()) / 0.01 - 1) < 0.005


def test_theta_in_bf16_keeps_its_mean():
    """Steps of a sixteenth of half a bf16 step: rounding to nearest would stand still."""
    n = 1 << 16
    p, g = [torch.ones(n, device="cuda", dtype=torch.bfloat16)], [torch.ones(n, device="cuda", dtype=torch.bfloat16)]
    s = ops.adamw_state(p, 32)
    for _ in range(64):
        ops.adamw_step(p, g, lr=2.0 ** -12, seed=5, **s)
    # theta falls by 2^-12 an update, 2^-6 in all.  One value's variance is at most 64 (2^-8)^2 / 4, so the mean of 65,536
    # has a deviation of at most 8 * 2^-9 / 256 = 2^-14; five of them
    assert abs(float(p[0].double().mean()) - (1 - 2.0 ** -6)) < 5 * 2.0 ** -14


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 12, 13, 400, 800])
def test_clipping_by_the_norm_of_all_gradients(count, bits):
    """Lists that need the small table, the large one, and several launches."""
    sizes = [1 + (i * 37) % 300 for i in range(count)]
    job = Job(sizes, torch.float32, torch.float32, bits, False, seed=count)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in job.grads)) * 0.5
    for max_norm in (norm / 3, norm * 2):
        before = job.before()
        job.step(max_norm=max_norm, grad_scale=0.5)
        job.check(before, gscale=0.5 * min(1.0, max_norm / (norm + 1e-6)))
        got = job.state["control"].cpu().numpy()[3:].view(np.float64)[0]
        assert abs(got / norm - 1) < 1e-12
    assert job.state["control"].tolist()[:3] == [2, 0, 0]


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_update_with_a_norm_that_is_not_finite_is_left_out(bad):
    job = Job([10, 3000], torch.bfloat16, torch.float32, 8, True, seed=8)
    job.step()
    keep = [t.clone() for k in ("m", "v", "m_scale", "v_scale") for t in job.state[k]] + [t.clone() for t in job.params + job.masters]
    job.grads[1][2999] = bad
    job.step(max_norm=1.0)
    now = [t for k in ("m", "v", "m_scale", "v_scale") for t in job.state[k]] + job.params + job.masters
    for x, y in zip(now, keep):
        assert torch.equal(x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x, y.view(torch.uint8) if y.dtype == torch.float8_e4m3fn else y)
    assert job.state["control"].tolist()[:3] == [1, 1, 0]
    job.step()  # without clipping a value that is not finite stays in its place
    m, _ = ops.decode_moments(*(job.state[k][1] for k in ("m", "m_scale", "v", "v_scale")))
    assert torch.isfinite(m[:2999]).all() and torch.isfinite(job.masters[1][:2999]).all()
    assert torch.isnan(m[2999])


def test_large_gradients_do_not_overflow_the_norm():
    job = Job([1000], torch.float32, torch.float32, 32, False)
    job.grads[0].fill_(1e30)
    before = job.before()
    job.step(max_norm=1.0)
    job.check(before, gscale=1.0 / (1e30 * math.sqrt(1000)))


def test_empty_tensors_and_mixed_states():
    p = [torch.randn(n, device="cuda") for n in (0, 600, 0, 77)]
    g = [torch.randn_like(x) for x in p]
    s8, s32 = ops.adamw_state(p, 8), ops.adamw_state(p, 32)
    m, v = [s32["m"][0], s8["m"][1], s32["m"][2], s32["m"][3]], [s32["v"][0], s8["v"][1], s32["v"][2], s32["v"][3]]
    want = [x - 0.1 * y / (y.abs() + 1e-8) for x, y in zip(p, g)]  # first update: m / sqrt(v) = g / |g|
    ops.adamw_step(p, g, m, v, s8["control"], lr=0.1, m_scale=s8["m_scale"], v_scale=s8["v_scale"])
    for x, y in zip(p, want):
        assert torch.allclose(x, y, rtol=0, atol=1e-5)  # m / sqrt(v) from fp32 factors: a few 2^-24 relative of 0.1, and 2^-24 |p|
    only_empty = [torch.zeros(0, device="cuda")]
    s = ops.adamw_state(only_empty)
    ops.adamw_step(only_empty, only_empty, lr=0.1, **s)
    assert s["control"].tolist()[0] == 1


def test_captured_updates_go_on_counting():
    job, twin = (Job([300, 5000], torch.float32, torch.float32, 32, False, seed=4) for _ in range(2))
    for _ in range(3):
        twin.step(max_norm=0.5)
    job.step(max_norm=0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        job.step(max_norm=0.5)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert job.state["control"].tolist() == twin.state["control"].tolist()
    for x, y in zip(job.params + job.state["m"] + job.state["v"], twin.params + twin.state["m"] + twin.state["v"]):
        assert torch.equal(x, y)


def test_another_stream():
    job, twin = (Job([300, 5000], torch.bfloat16, torch.bfloat16, 8, False, seed=4) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    job.step(stream=side, max_norm=0.1)
    twin.step(max_norm=0.1)
    side.synchronize()
    for x, y in zip(job.params, twin.params):
        assert torch.equal(x, y)


def test_refusals():
    p, g = [torch.zeros(300, device="cuda")], [torch.zeros(300, device="cuda")]
    s = ops.adamw_state(p)
    s8 = ops.adamw_state(p, 8)
    h = [p[0].half()]
    calls = [
        lambda: ops.adamw_step(p, [], lr=1.0, **s), lambda: ops.adamw_step(p, [g[0][:299]], lr=1.0, **s), lambda: ops.adamw_step(p, [g[0].double()], lr=1.0, **s),
        lambda: ops.adamw_step(p, [g[0].cpu()], lr=1.0, **s), lambda: ops.adamw_step([torch.zeros(600, device="cuda")[::2]], g, lr=1.0, **s),
        lambda: ops.adamw_step(p, g, s["m"], s8["v"], s["control"], 1.0), lambda: ops.adamw_step(p, g, s8["m"], s8["v"], s["control"], 1.0),
        lambda: ops.adamw_step(p, g, s8["m"], s8["v"], s["control"], 1.0, m_scale=s8["m_scale"], v_scale=[s8["v_scale"][0][:1]]),
        lambda: ops.adamw_step(p, g, s["m"], s["v"], s["control"][:3], 1.0), lambda: ops.adamw_step(p, g, s["m"], s["v"], s["control"].float(), 1.0),
        lambda: ops.adamw_step(h, g, s["m"], s["v"], s["control"], 1.0), lambda: ops.adamw_step(h, g, s["m"], s["v"], s["control"], 1.0, masters=[None]),
        lambda: ops.adamw_step(p, g, s["m"], s["v"], s["control"], 1.0, masters=[torch.zeros(300, device="cuda")]),
        lambda: ops.adamw_step(p, g, s["m"], s["v"], s["control"], 1.0, weight_decay=[0.1, 0.1]),
        lambda: ops.adamw_step(p, g, s["m"], s["v"], s["control"], 1.0, masters=[]),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {k} was not refused")
    from paper_2312_08728_b200.binding import BmgdError
    for call in (lambda: ops.adamw_step(p, p, lr=1.0, **s), lambda: ops.adamw_step(p * 2, g * 2, s["m"] * 2, s["v"] * 2, s["control"], 1.0),
                 lambda: ops.adamw_step(p, g, lr=math.nan, **s), lambda: ops.adamw_step(p, g, lr=1.0, a=1.0, **s), lambda: ops.adamw_step(p, g, lr=1.0, max_norm=-1.0, **s)):
        with pytest.raises(BmgdError):
            call()
    assert s["control"].tolist() == [0, 0, 0, 0]


@pytest.mark.parametrize("b", [0.999, 0.9999999])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,master,shift", [(torch.float32, False, 0), (torch.float32, False, 1), (torch.bfloat16, True, 0)])
def test_first_updates_from_tiny_gradients_with_the_least_eps(param, master, shift, bits, b):
    """eps = 0 counts as 2^-63, and the second moments of gradients of 1e-22 to 1e-15 are subnormal: sqrt(v) / sqrt(1 - b) is not
    small beside eps, so the first update moves theta by up to lr, not by a multiple of it."""
    n, lr, a = 4096 + 37, 0.01, 0.9
    gen = torch.Generator(device="cuda").manual_seed(bits)
    size = 10.0 ** (torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * 7 - 22)
    g = torch.zeros(n + shift, device="cuda")[shift:]
    g.copy_(torch.where(torch.rand(n, generator=gen, device="cuda") < 0.5, -size, size))
    p = [torch.zeros(n + shift, device="cuda", dtype=param)[shift:]]
    masters = [torch.zeros(n, device="cuda")] if master else None
    ops.adamw_step(p, [g], lr=lr, a=a, b=b, eps=0.0, masters=masters, **ops.adamw_state(p, bits))
    gd = g.double()
    v, eps, root = (1 - b) * gd * gd, 2.0 ** -63, (1 - b) ** -0.5
    denom = v.sqrt() * root + eps
    move = lr / (1 - a) * (1 - a) * gd / denom
    # v has a relative error of 4 units of 2^-24 where it is normal and one subnormal step, 2^-149, at most; the rest in units of 2^-24:
    # the root 2 and its factor 2, the sum 1, the quotient 4, m 2, the step length 2, theta 1
    dv = 4 * E32 * v + 2.0 ** -149
    spread = ((v + dv).sqrt() - (v - dv).clamp(min=0).sqrt()) * root / ((v - dv).clamp(min=0).sqrt() * root + eps)
    err = ((masters or p)[0].double() + move).abs()
    assert bool((err <= move.abs() * (spread + 16 * E32) + 2.0 ** -149).all()), float((err / move.abs()).max())
    assert float(move.abs().max()) <= lr
