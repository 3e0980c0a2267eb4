"""The AdamW step over many tensors against the 64-bit form.

Tolerances, e = 2^-24 (half a binary32 step).  m: two products and a sum, 3 e of the magnitudes that enter; v: 4 e, all terms positive; the update: the error
of m, and for sqrt (1 e of its own and half of v's), its product and sum, the division (2 e) and the step size (2 e) together 12 e; p: the product with
1 - lr wd (2 e) and the sum (1 e).  8-bit states are read exactly but for the division by the scale, 2 e (4 e for v)."""
import numpy as np
import pytest
import torch

import operator_refs as ref

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
HY = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8)
SIZES = [1, 3, 4, 127, 128, 129, 0, 500, 4095, 4096, 4097, 70001]


@pytest.fixture(scope="module")
def api():
    from paper_2602_01410_b200 import api
    return api


def f64(t):
    return t.double().cpu().numpy()


class Run:
    """Tensors of a step, with guard elements behind each."""

    def __init__(self, sizes, bits, param, grad, copy, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.bits, self.sizes, self.copy, self.param = bits, sizes, copy, param
        def normal(n):
            return torch.randn(n, generator=g, device="cuda")
        def guarded(t, fill):
            n = t.numel()
            whole = torch.full((n + 32,), fill, dtype=t.dtype, device="cuda")
            whole[:n] = t
            self.guards.append((whole, n, fill))
            return whole[:n]
        self.guards = []
        self.p, self.g, self.m, self.v, self.ms, self.vs, self.c = [], [], [], [], [], [], []
        for n in sizes:
            scale = 1e-3 * torch.exp(2 * normal(n))
            self.p.append(guarded((0.02 * normal(n)).to(param), 9.0))
            self.g.append((normal(n) * scale).to(grad))
            m, v = normal(n) * scale * 0.4, scale ** 2
            if bits == 32:
                self.m.append(guarded(m, 9.0)); self.v.append(guarded(v, 9.0))
            else:
                s = [torch.from_numpy(ref.block_scale(f64(x)).astype(np.float32)).cuda() for x in (m, v.sqrt())]
                for dst, x, sc in ((self.m, m, s[0]), (self.v, v.sqrt(), s[1])):
                    code = (x * sc.repeat_interleave(128)[:n]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                    dst.append(guarded(code, 0x5A))
                self.ms.append(guarded(s[0], 9.0)); self.vs.append(guarded(s[1], 9.0))
            self.c.append(guarded(torch.zeros(n, dtype=torch.bfloat16, device="cuda"), 9.0) if copy else None)
        self.before = self.values()

    def values(self):
        out = []
        for i, n in enumerate(self.sizes):
            if self.bits == 32:
                m, v = f64(self.m[i]), f64(self.v[i])
            else:
                m = ref.code_values(self.m[i].cpu().numpy(), True, 1, n)[0] / np.repeat(f64(self.ms[i]), 128)[:n]
                v = (ref.code_values(self.v[i].cpu().numpy(), True, 1, n)[0] / np.repeat(f64(self.vs[i]), 128)[:n]) ** 2
            out.append((f64(self.p[i]), f64(self.g[i]), m, v))
        return out

    def tensors(self, api, decay=0.1):
        eight = self.bits == 8
        return api.make_adamw_tensors(self.p, self.g, self.m, self.v, m_scales=self.ms if eight else None, v_scales=self.vs if eight else None,
                                      copies=self.c if self.copy else None, weight_decay=decay)

    def check(self, step, decay=0.1, seed=None, grad_scale=1.0, first_tensor=0, hy=HY):
        read = 2 * E if self.bits == 8 else 0
        for i, n in enumerate(self.sizes):
            p0, g, m0, v0 = self.before[i]
            d = decay[i] if isinstance(decay, (list, tuple)) else decay
            p, m, v, up = ref.adamw(p0, g, m0, v0, hy["lr"], hy["beta1"], hy["beta2"], hy["eps"], step, d, grad_scale)
            em = (3 * E + read) * (hy["beta1"] * np.abs(m0) + 2 * (1 - hy["beta1"]) * np.abs(g * grad_scale))
            ev = (4 * E + 2 * read) * v
            root = np.sqrt(v)
            eup = np.abs(up) * (12 * E + read) + em * np.abs(up) / np.where(m == 0, 1, np.abs(m))
            ep = 4 * E * np.abs(p0) + eup
            if seed is None:
                um = uv = up16 = None
            else:
                w = ref.philox(-(-n // 4), first_tensor + i, 2 * step, seed)
                um, uv = ref.uniforms(n, w[:2]), ref.uniforms(n, w[2:])
                up16 = ref.uniforms(n, ref.philox(-(-n // 4), first_tensor + i, 2 * step + 1, seed)[:2])
            if self.bits == 32:
                assert np.all(np.abs(f64(self.m[i]) - m) <= em) and np.all(np.abs(f64(self.v[i]) - v) <= ev)
            elif n:
                for codes, scales, x, ex, u, floor in ((self.m, self.ms, m, em, um, False), (self.v, self.vs, root, 4 * E * root + 2 * read * root, uv, True)):
                    s = ref.block_scale(x)
                    got = f64(scales[i])
                    most = 448 / s
                    worst = np.array([ex[128 * b: 128 * b + 128].max() for b in range(len(s))])
                    assert np.all(np.abs(got - s) <= s * (2 * E + worst / np.where(s == 1, 1, most)))
                    t, q = x * np.repeat(s, 128)[:n], ref.code_values(codes[i].cpu().numpy(), True, 1, n)[0]
                    slack = np.repeat(s, 128)[:n] * ex * 1.01 + np.abs(t) * np.repeat(2 * E + worst / most, 128)[:n] + np.abs(t) * 2 * E
                    ok = ref.between(q, t, slack, ref.E4M3, u)
                    if floor:
                        ok |= (q == 2.0 ** -9) & (x > 0) & ref.between(np.zeros(n), t, slack, ref.E4M3, u)
                        assert np.all(q[x > 0] > 0)
                    assert np.all(ok)
            got = f64(self.p[i])
            if self.param == torch.float32:
                assert np.all(np.abs(got - p) <= ep)
                if self.copy:
                    assert torch.equal(self.c[i], self.p[i].to(torch.bfloat16))
            elif seed is None:
                assert np.all(np.abs(got - p) <= 2.0 ** -8 * np.abs(p) + ep * 1.01)
            else:
                def sr(x):
                    step_ = np.exp2(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126))) - 7)
                    low = np.floor(np.abs(x) / step_)
                    return np.copysign((low + (np.abs(x) / step_ - low > (up16 + 0.5) / 65536)) * step_, x)
                a, b = sr(p - ep), sr(p + ep)
                assert np.all((got >= np.minimum(a, b)) & (got <= np.maximum(a, b)))
        for whole, n, fill in self.guards:
            assert torch.all(whole[n:] == fill)


F32, BF = torch.float32, torch.bfloat16


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,copy", [(F32, F32, True), (F32, BF, False), (F32, BF, True), (BF, F32, False), (BF, BF, False)])
@pytest.mark.parametrize("sr", [False, True])
def test_one_step(api, bits, param, grad, copy, sr):
    r = Run(SIZES, bits, param, grad, copy)
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    api.snip_adamw_step(r.tensors(api, decay), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 7, rounding=api.ROUND_STOCHASTIC if sr else api.ROUND_NEAREST_EVEN, seed=0x123456789ABCDEF0)
    r.check(7, [float(np.float32(d)) for d in decay], 0x123456789ABCDEF0 if sr else None)


@pytest.mark.parametrize("bits", [32, 8])
def test_fresh_states_of_zero_bytes(api, bits):
    r = Run([700, 128, 5], bits, F32, F32, False, seed=3)
    for ts in (r.m, r.v, r.ms, r.vs):
        for t in ts:
            t.zero_()
    r.before = [(p, g, np.zeros_like(p), np.zeros_like(p)) for p, g, _, _ in r.before]
    api.snip_adamw_step(r.tensors(api, 0.0), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 1)
    r.check(1, 0.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_of_zero(api, bits):
    # blocks of zeros: states stay zero, their scale is 1, only the decay moves the weights
    r = Run([300, 4096], bits, F32, F32, True, seed=4)
    for ts in (r.m, r.v, r.g):
        for t in ts:
            t.zero_()
    r.before = r.values()
    api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 5, rounding=api.ROUND_STOCHASTIC)
    for i in range(2):
        assert torch.all(r.m[i] & 0x7F == 0) if bits == 8 else torch.all(r.m[i] == 0)
        assert torch.all(r.v[i] == 0)
        if bits == 8:
            assert torch.all(r.ms[i] == 1) and torch.all(r.vs[i] == 1)
    r.check(5, seed=0 if bits == 8 else None)


def test_more_tensors_than_a_launch_takes(api):
    sizes = [(37 * i) % 300 for i in range(1000)]
    r = Run(sizes, 8, BF, BF, False, seed=5)
    api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 3, rounding=api.ROUND_STOCHASTIC, seed=99)
    r.check(3, float(np.float32(0.1)), 99)


@pytest.mark.parametrize("count", [1, 111, 112, 113, 447, 448, 449])
def test_counts_around_the_tables_sizes(api, count):
    r = Run([1 + (i * 13) % 260 for i in range(count)], 32, F32, BF, True, seed=count)
    api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 2)
    r.check(2, float(np.float32(0.1)))


def test_a_large_tensor_among_small_ones(api):
    # more chunks than the grid: CTAs walk on and across tensors
    r = Run([10, 9_000_001, 0, 129], 8, F32, BF, True, seed=6)
    api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 11, rounding=api.ROUND_STOCHASTIC, seed=(1 << 64) - 1)
    r.check(11, float(np.float32(0.1)), (1 << 64) - 1)


def test_reruns_and_splits_give_the_same_bits(api):
    a, b = (Run([5000, 300], 8, BF, F32, False, seed=8) for _ in range(2))
    for r in (a, b):
        api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 3, rounding=api.ROUND_STOCHASTIC, seed=4)
    for x, y in zip(a.p + a.m + a.v + a.ms + a.vs, b.p + b.m + b.v + b.ms + b.vs):
        assert torch.equal(x, y)
    c = Run([5000, 300], 8, BF, F32, False, seed=8)
    api.snip_adamw_step(c.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 4, rounding=api.ROUND_STOCHASTIC, seed=4)
    assert not torch.equal(a.m[0], c.m[0])      # the step's number enters the generator


def test_gradient_scale_on_the_device(api):
    r = Run([1000, 3], 32, F32, F32, False, seed=9)
    gs = torch.tensor([0.25], device="cuda")
    api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 2, grad_scale=gs)
    r.check(2, float(np.float32(0.1)), grad_scale=0.25)


@pytest.mark.parametrize("param", [F32, BF])
def test_gradient_scale_with_8_bit_states(api, param):
    # no power of two: g' is rounded, which adds 1 e to the new part of m and 2 e to that of v; with the 3 e and 4 e of the two products, the
    # constant and the sum these stay within the bounds for 8 bits (6 e and 8 e)
    r = Run([1000, 3, 4097], 8, param, F32, False, seed=12)
    gs = torch.tensor([0.3], device="cuda")
    api.snip_adamw_step(r.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 3, rounding=api.ROUND_STOCHASTIC, seed=2 ** 63 + 5, grad_scale=gs)
    r.check(3, float(np.float32(0.1)), seed=2 ** 63 + 5, grad_scale=float(np.float32(0.3)))


@pytest.mark.parametrize("on_device", ["rate", "step"])
@pytest.mark.parametrize("bits", [32, 8])
def test_only_the_rate_or_only_the_step_on_the_device(api, on_device, bits):
    a, b = Run([5000, 77], bits, F32, BF, True, seed=13), Run([5000, 77], bits, F32, BF, True, seed=13)
    lr = torch.tensor([1e-3], device="cuda")
    host = float(lr.cpu()[0])
    device = (lr, 6) if on_device == "rate" else (host, torch.tensor([6], dtype=torch.int64, device="cuda"))
    for r, (rate, step) in ((a, device), (b, (host, 6))):
        api.snip_adamw_step(r.tensors(api), rate, 0.9, 0.95, 1e-8, step, rounding=api.ROUND_STOCHASTIC, seed=5)
    for x, y in zip(a.m + a.v + a.ms + a.vs, b.m + b.v + b.ms + b.vs):
        assert torch.equal(x, y)
    for x, y in zip(a.p, b.p):      # as for the captured step: a last place of the bias corrections
        assert torch.all((x - y).abs() <= 4 * E * y.abs() + 1e-3 * 8 * E)


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_reads_step_and_rate_at_each_replay(api, bits):
    r, w = Run([5000, 77], bits, F32, BF, True, seed=10), Run([5000, 77], bits, F32, BF, True, seed=10)
    t, tw = r.tensors(api), w.tensors(api)
    step, lr = torch.tensor([0], dtype=torch.int64, device="cuda"), torch.tensor([1e-3], device="cuda")
    spare = Run([10], bits, F32, BF, True)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):       # the first launch of the kernel, outside the capture
        api.snip_adamw_step(spare.tensors(api), 1e-3, 0.9, 0.95, 1e-8, 1, rounding=api.ROUND_STOCHASTIC)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        api.snip_adamw_step(t, lr, 0.9, 0.95, 1e-8, step, rounding=api.ROUND_STOCHASTIC, seed=21)
    for k in range(1, 4):
        lr.fill_(1e-3 / k)
        for a, b in zip(r.g, w.g):
            a.copy_(torch.randn(a.numel(), device="cuda") * 1e-3); b.copy_(a)
        graph.replay()
        api.snip_adamw_step(tw, float(lr.cpu()[0]), 0.9, 0.95, 1e-8, k, rounding=api.ROUND_STOCHASTIC, seed=21)
        torch.cuda.synchronize()
        # the bias corrections are worked out in 64 bits on either side, but not by the same library: a last place of difference
        for x, y in zip(r.m + r.v + r.ms + r.vs, w.m + w.v + w.ms + w.vs):
            assert torch.equal(x, y)
        for x, y in zip(r.p, w.p):
            assert torch.all((x - y).abs() <= 4 * E * y.abs() + 1e-3 * 8 * E)
            y.copy_(x)


def test_a_long_run_keeps_up_with_32_bits(api):
    # the second moment of constant-size gradients settles at g^2 although a step changes it by less than a code
    n = 1024
    g = torch.full((n,), 0.01, device="cuda")
    p, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    g[::128] = 0.04
    ms, vs = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    t = api.make_adamw_tensors([p], [g], [m], [v], m_scales=[ms], v_scales=[vs])
    for k in range(1, 400):
        api.snip_adamw_step(t, 0.0, 0.9, 0.99, 1e-8, k, rounding=api.ROUND_STOCHASTIC, seed=k)
    root = ref.code_values(v.cpu().numpy(), True, 1, n)[0] / np.repeat(f64(vs), 128)
    want = f64(g) * np.sqrt(1 - 0.99 ** 399)
    # the mean of 1016 elements whose codes scatter by at most a code (1/16 of the value) about it
    assert abs(root[f64(g) < 0.02].mean() / want[1] - 1) < 0.03


def test_two_streams_at_once(api):
    runs = [Run([200_000, 33], 8, F32, BF, True, seed=i) for i in range(2)]
    want = [Run([200_000, 33], 8, F32, BF, True, seed=i) for i in range(2)]
    for i, w in enumerate(want):
        api.snip_adamw_step(w.tensors(api), 1e-3, 0.9, 0.95, 1e-8, 5, rounding=api.ROUND_STOCHASTIC, seed=i)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for i, (s, r) in enumerate(zip(streams, runs)):
        with torch.cuda.stream(s):
            api.snip_adamw_step(r.tensors(api), 1e-3, 0.9, 0.95, 1e-8, 5, rounding=api.ROUND_STOCHASTIC, seed=i)
    torch.cuda.synchronize()
    for a, b in zip(runs, want):
        for x, y in zip(a.p + a.m + a.v + a.ms + a.vs + a.c, b.p + b.m + b.v + b.ms + b.vs + b.c):
            assert torch.equal(x, y)


def test_offsets_beyond_32_bits(api):
    # 8-bit states and bf16 weights of a tensor with more than 2^31 elements; its end is compared with a short tensor of the same values
    n, tail = (1 << 31) + 4096 * 3 + 5, 4096 + 5
    p, g = torch.zeros(n, dtype=BF, device="cuda"), torch.zeros(n, dtype=BF, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(-(-n // 128), device="cuda"), torch.zeros(-(-n // 128), device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    start = n - tail                       # a multiple of 128
    assert start % 128 == 0
    p[start:] = (torch.randn(tail, generator=gen, device="cuda") * 0.02).to(BF)
    g[start:] = (torch.randn(tail, generator=gen, device="cuda") * 1e-3).to(BF)
    q = [t[start:].clone() for t in (p, g, m, v)] + [ms[start // 128:].clone(), vs[start // 128:].clone()]
    api.snip_adamw_step(api.make_adamw_tensors([p], [g], [m], [v], m_scales=[ms], v_scales=[vs]), 1e-3, 0.9, 0.95, 1e-8, 1)
    api.snip_adamw_step(api.make_adamw_tensors([q[0]], [q[1]], [q[2]], [q[3]], m_scales=[q[4]], v_scales=[q[5]]), 1e-3, 0.9, 0.95, 1e-8, 1)
    for a, b in ((p[start:], q[0]), (m[start:], q[2]), (v[start:], q[3]), (ms[start // 128:], q[4]), (vs[start // 128:], q[5])):
        assert torch.equal(a, b)
    assert not torch.any(p[:start]) and torch.all(ms[:start // 128] == 1)


@pytest.mark.parametrize("sr", [False, True])
def test_states_are_the_definitions_bits(api, sr):
    # 8-bit states of a chain of steps, each product and sum in binary32 as the header says: equal bit for bit, scales included (what a step
    # rounds one way or the other is fed back, so that runs which differ in one rounding part company)
    n, seed = 40_000, 77
    g = torch.Generator(device="cuda").manual_seed(2)
    size = torch.exp(2 * torch.randn(n, generator=g, device="cuda")) * 1e-3
    p = torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(-(-n // 128), device="cuda"), torch.zeros(-(-n // 128), device="cuda")
    grad = torch.zeros(n, device="cuda")
    t = api.make_adamw_tensors([p], [grad], [m], [v], m_scales=[ms], v_scales=[vs])
    f = np.float32
    code_m, code_v, s_m, s_v = np.zeros(n, f), np.zeros(n, f), np.ones(len(ms), f), np.ones(len(ms), f)

    def stored(x, u, floor):
        whole = np.zeros(len(ms) * 128, f)
        whole[:n] = np.abs(x)
        most = whole.reshape(-1, 128).max(1)
        s = np.where(most > 0, f(448) * (f(1) / np.where(most > 0, most, f(1))), f(1)).astype(f)
        y = (x * np.repeat(s, 128)[:n]).astype(np.float64)
        c = ref.nearest(y, ref.E4M3) if u is None else ref.stochastic(y, u, ref.E4M3)
        if floor:
            c = np.where((x > 0) & (c == 0), 2.0 ** -9, c)
        return c.astype(f), s

    for step in range(1, 7):
        grad.copy_(torch.randn(n, generator=g, device="cuda") * size)
        gr = grad.cpu().numpy()
        api.snip_adamw_step(t, 1e-3, 0.9, 0.95, 1e-8, step, rounding=api.ROUND_STOCHASTIC if sr else api.ROUND_NEAREST_EVEN, seed=seed)
        om = code_m / np.repeat(s_m, 128)[:n]
        ov = (code_v / np.repeat(s_v, 128)[:n]) ** 2
        nm = f(0.9) * om + f(1 - 0.9) * gr
        nv = f(0.95) * ov + f(1 - 0.95) * (gr * gr)
        um = uv = None
        if sr:
            w = ref.philox(-(-n // 4), 0, 2 * step, seed)
            um, uv = ref.uniforms(n, w[:2]), ref.uniforms(n, w[2:])
        assert nm.dtype == f and nv.dtype == f
        code_m, s_m = stored(nm, um, False)
        code_v, s_v = stored(np.sqrt(nv), uv, True)
        assert np.array_equal(ms.cpu().numpy(), s_m) and np.array_equal(vs.cpu().numpy(), s_v)
        assert np.array_equal(ref.code_values(m.cpu().numpy(), True, 1, n)[0].astype(f), code_m)
        assert np.array_equal(ref.code_values(v.cpu().numpy(), True, 1, n)[0].astype(f), code_v)


def test_a_list_in_one_call_and_in_several(api):
    # the optimizer step to nearest: a tensor's result does not depend on its place in the list, nor on how lists are cut
    for bits in (32, 8):
        a, b = Run(SIZES, bits, F32, BF, True, seed=14), Run(SIZES, bits, F32, BF, True, seed=14)
        api.snip_adamw_step(a.tensors(api), HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 3)
        for at in (slice(5, None), slice(0, 2), slice(2, 5)):
            eight = bits == 8
            t = api.make_adamw_tensors(b.p[at], b.g[at], b.m[at], b.v[at], m_scales=b.ms[at] if eight else None, v_scales=b.vs[at] if eight else None, copies=b.c[at], weight_decay=0.1)
            api.snip_adamw_step(t, HY["lr"], HY["beta1"], HY["beta2"], HY["eps"], 3)
        for x, y in zip(a.p + a.m + a.v + a.ms + a.vs + a.c, b.p + b.m + b.v + b.ms + b.vs + b.c):
            assert np.array_equal(x.float().cpu().numpy(), y.float().cpu().numpy())
