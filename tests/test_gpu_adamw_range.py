"""The AdamW step where a gradient's square passes binary32's range: v is infinite, so that the update is m / inf = 0 and the weight only decays; an 8-bit
state holds the root at sqrt(FLT_MAX) and comes back down in the steps behind it."""
import numpy as np
import pytest
import torch

import operator_refs as ref

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
F32, BF = torch.float32, torch.bfloat16
LR, B1, B2, EPS, WD = 1e-3, 0.9, 0.95, 1e-8, 0.1
FLT_MAX = float(np.finfo(np.float32).max)
N = 300          # two blocks of 128 and the start of a third, a chunk that is not full
LONG = 2048 + 300  # a full chunk and a short one


@pytest.fixture(scope="module")
def api():
    from paper_2602_01410_b200 import api
    return api


class State:
    def __init__(self, api, n, bits, param, grad):
        self.api, self.bits, self.n = api, bits, n
        gen = torch.Generator(device="cuda").manual_seed(n)
        state = torch.uint8 if bits == 8 else F32
        self.p = (0.5 + torch.rand(n, generator=gen, device="cuda")).to(param)
        self.g = (1e-3 * torch.randn(n, generator=gen, device="cuda")).to(grad)
        self.m, self.v = (torch.zeros(n, dtype=state, device="cuda") for _ in range(2))
        self.ms, self.vs = (torch.zeros(-(-n // 128), device="cuda") for _ in range(2))
        self.c = torch.zeros(n, dtype=BF, device="cuda") if param == F32 else None
        self.t = api.make_adamw_tensors([self.p], [self.g], [self.m], [self.v], m_scales=[self.ms] if bits == 8 else None, v_scales=[self.vs] if bits == 8 else None,
                                        copies=[self.c] if param == F32 else None, weight_decay=WD)

    def step(self, k, sr, grad_scale=None):
        self.api.snip_adamw_step(self.t, LR, B1, B2, EPS, k, rounding=self.api.ROUND_STOCHASTIC if sr else self.api.ROUND_NEAREST_EVEN, seed=11, grad_scale=grad_scale)

    def values(self, name):
        t = getattr(self, name)
        return (t.view(torch.float8_e4m3fn) if self.bits == 8 else t).double().cpu().numpy()

    def moment(self, name):
        x = self.values(name)
        return x if self.bits == 32 else x / np.repeat(getattr(self, name + "s").double().cpu().numpy(), 128)[:self.n]


FORMS = [(bits, param, grad, sr) for bits in (32, 8) for param, grad in ((F32, F32), (F32, BF), (BF, F32), (BF, BF)) for sr in (False, True)]


@pytest.mark.parametrize("bits,param,grad,sr", FORMS)
@pytest.mark.parametrize("n", [N, LONG])
@pytest.mark.parametrize("size", [1e20, -3e38])
def test_a_square_beyond_the_range_leaves_the_weight_to_its_decay(api, bits, param, grad, sr, n, size):
    at = [5, 140, n - 1]
    a, b = State(api, n, bits, param, grad), State(api, n, bits, param, grad)
    a.g[at], b.g[at] = size, 0.0        # b: the same step without these gradients
    before = a.p.double().cpu().numpy()
    a.step(1, sr)
    b.step(1, sr)
    got, others = a.p.double().cpu().numpy(), np.setdiff1d(np.arange(n), at)
    want = before[at] * (1 - LR * float(np.float32(WD)))
    # the factor (one rounding) and the product (one more); a bf16 weight to its neighbours
    slack = 2 * E * want if param == F32 else (2.0 ** -7 if sr else 2.0 ** -8) * want
    assert np.all(np.abs(got[at] - want) <= 1.01 * slack)
    if a.c is not None:
        assert torch.equal(a.c, a.p.to(BF))
    assert torch.equal(a.p[others], b.p[others])       # nobody else's weight
    if bits == 32:
        size = float(a.g[5])
        assert np.all(np.isposinf(a.values("v")[at])) and np.all(np.abs(a.values("m")[at] - (1 - B1) * size) <= 3 * E * abs(size))
        for name in ("m", "v"):
            assert torch.equal(getattr(a, name)[others], getattr(b, name)[others])
    else:
        assert np.all(a.values("v")[at] == 448) and np.all(np.abs(a.values("m")[at]) == 448)
        scale = a.vs.double().cpu().numpy()[[i // 128 for i in at]]
        # 448 times the rounded reciprocal of the rounded root: three roundings
        assert np.all(np.abs(scale * np.sqrt(FLT_MAX) / 448 - 1) <= 4 * E)
        assert np.all(np.isfinite(a.moment("v"))) and np.all(a.values("v") > 0)
        blocks = [k for k in range(-(-n // 128)) if all(i // 128 != k for i in at)]
        for name in ("m", "v"):
            for k in blocks:
                assert torch.equal(getattr(a, name)[128 * k: 128 * k + 128], getattr(b, name)[128 * k: 128 * k + 128])


@pytest.mark.parametrize("bits,param,grad,sr", FORMS)
def test_the_steps_behind_it(api, bits, param, grad, sr):
    a = State(api, N, bits, param, grad)
    a.g[7] = 1e20
    a.step(1, sr)
    a.g[7] = 1e-3
    roots, weights = [], [float(a.p[7])]
    for k in range(2, 200):
        a.step(k, sr)
        roots.append(a.moment("v")[7])
        weights.append(float(a.p[7]))
    assert np.all(np.isfinite(a.p.double().cpu().numpy())) and np.all(np.isfinite(weights))
    if bits == 32:
        # an infinite v stays one: the weight decays and does nothing else
        assert np.all(np.isposinf(roots))
        if param == F32:
            want = weights[0] * (1 - LR * float(np.float32(WD))) ** 198
            assert abs(weights[-1] - want) <= 198 * 2 * E * want
    else:
        # an 8-bit one is finite and falls as beta2^k does: it is its block's largest, which is code 448 of a scale that follows it (and its root is
        # read back within 4 roundings a step), down to 0.95^99 = 6.2e-3 of the largest root there is
        assert np.all(np.isfinite(roots)) and all(y < x for x, y in zip(roots, roots[1:]))
        assert abs(roots[-1] / (np.sqrt(FLT_MAX) * B2 ** 99) - 1) <= 198 * 8 * E


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sr", [False, True])
def test_a_scaled_gradient_counts_as_scaled(api, bits, sr):
    gs = torch.tensor([1e12], device="cuda")
    a, b = State(api, N, bits, F32, F32), State(api, N, bits, F32, F32)
    a.g.zero_()
    b.g.zero_()
    a.g[3] = 1e9
    before = float(a.p[3])
    a.step(1, sr, gs)
    b.step(1, sr, gs)
    want = before * (1 - LR * float(np.float32(WD)))
    assert abs(float(a.p[3]) - want) <= 2.02 * E * want
    others = [i for i in range(N) if i != 3]
    assert torch.equal(a.p[others], b.p[others])


@pytest.mark.parametrize("bits", [32, 8])
def test_a_square_within_the_range_is_an_ordinary_one(api, bits):
    # 1e19: the square is 1e38, v = 5e36; the first step's update is lr whatever the gradient's size
    a = State(api, N, bits, F32, F32)
    a.g[9] = 1e19
    before = float(a.p[9])
    a.step(1, False)
    p, *_ = ref.adamw(np.array([before]), np.array([float(a.g[9])]), np.zeros(1), np.zeros(1), LR, B1, B2, EPS, 1, float(np.float32(WD)))
    assert abs(float(a.p[9]) - p[0]) <= 4 * E * before + 20 * E * LR


@pytest.mark.parametrize("bits,param,grad,sr", FORMS)
@pytest.mark.parametrize("n", [N, LONG])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_no_rounding_hides_what_is_not_a_number(api, bits, param, grad, sr, n, what):
    # outside the documented range, but a step that has diverged must not look like a sound one
    at = [5, 140, n - 1]
    a, b = State(api, n, bits, param, grad), State(api, n, bits, param, grad)
    a.g[at], b.g[at] = what, 0.0
    others = np.setdiff1d(np.arange(n), at)
    for k in (1, 2):                    # and it stays one
        a.step(k, sr)
        b.step(k, sr)
        a.g[at] = 1e-3
        assert np.all(np.isnan(a.p.double().cpu().numpy()[at]))
        if a.c is not None:
            assert np.all(np.isnan(a.c.double().cpu().numpy()[at]))
        if bits == 32 or np.isnan(what):
            assert not np.any(np.isfinite(a.values("m")[at]))
        if bits == 32:
            assert not np.any(np.isfinite(a.values("v")[at]))
        elif np.isnan(what):
            assert np.all(np.isnan(a.values("v")[at]))
        assert torch.equal(a.p[others], b.p[others]) or np.isinf(what)
        if k == 1:
            assert torch.equal(a.p[others], b.p[others])
        if np.isnan(what):
            # the scale is that of the block's numbers: the other elements are what they are without it
            for name in ("m", "v"):
                assert torch.equal(getattr(a, name)[others], getattr(b, name)[others])
            assert torch.equal(a.ms, b.ms) and torch.equal(a.vs, b.vs)


@pytest.mark.parametrize("bits,param,grad,sr", FORMS)
def test_a_weight_that_is_not_a_number_stays_one(api, bits, param, grad, sr):
    a, b = State(api, N, bits, param, grad), State(api, N, bits, param, grad)
    a.p[[5, 299]] = float("nan")
    a.p[6] = float("inf")
    a.step(1, sr)
    b.step(1, sr)
    got = a.p.double().cpu().numpy()
    assert np.all(np.isnan(got[[5, 299]])) and np.isposinf(got[6])
    others = [i for i in range(N) if i not in (5, 6, 299)]
    assert torch.equal(a.p[others], b.p[others]) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v)


@pytest.mark.parametrize("sr", [False, True])
def test_the_largest_weights_round_as_their_type_does(api, sr):
    # no update and no decay: bf16 weights come back as they are, the largest finite ones and both zeros included
    p = torch.tensor([3.3895e38, -3.3895e38, 0.0, -0.0, 1.0, 2.0 ** -126, -2.0 ** -133], device="cuda").to(BF)
    keep = p.clone()
    g, m, v = (torch.zeros(7, device="cuda") for _ in range(3))
    t = api.make_adamw_tensors([p], [g], [m], [v])
    api.snip_adamw_step(t, 0.0, B1, B2, EPS, 1, rounding=api.ROUND_STOCHASTIC if sr else api.ROUND_NEAREST_EVEN, seed=5)
    assert torch.equal(p, keep)
