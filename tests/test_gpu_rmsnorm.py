"""RMS norm with residual and quantized outputs, and its backward pass, against the 64-bit forms.

Tolerances.  e = 2^-24 is half a binary32 step.  A sum of n terms whose partial sums are added in a tree of threads with at most n/t + log2(t) + 8
additions on any path is off by at most that many e relative to the sum of magnitudes; 32 vectors of 8 per thread and 10 levels give the 64 e used
for means over a row (a thread holds at most 4 vectors).  rstd takes half of that (square root) and three roundings more: 36 e; y two products
more: 38 e.  A result stored in bf16 adds half a step, 2^-8 relative."""
import numpy as np
import pytest
import torch

import operator_refs as ref

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def api():
    from paper_2602_01410_b200 import api
    return api


def rand(rows, cols, seed, scale=1.0, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(rows, ld or cols, generator=g, device="cuda") * scale
    t[:, ::37] *= 20
    return t.to(torch.bfloat16)[:, :cols]


def gain_of(cols, f32, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    return t if f32 else t.to(torch.bfloat16)


def f64(t):
    return t.double().cpu().numpy()


def check_codes(codes, scales, y, fp8, transposed):
    """Codes and scales against the 64-bit y: scales to the error of a maximum of y, codes what some value that close is rounded to."""
    z = y.T if transposed else y
    lines, along = z.shape
    tiles = -(-along // 128)
    got = ref.code_values(codes.cpu().numpy(), fp8, lines, along)
    s = scales.cpu().numpy().astype(np.float64).reshape(tiles, lines)
    grid = ref.E4M3 if fp8 else ref.E2M1
    for k in range(tiles):
        part = z[:, 128 * k: 128 * k + 128]
        most = np.abs(part).max(1)
        want = np.where(most > 0, grid[-1] / np.where(most > 0, most, 1), 1.0)
        assert np.all(np.abs(s[k] - want) <= 40 * E * want)
        t = part * want[:, None]
        # y, the scale and their product: 38 + 39 + 1 halves of a step
        assert np.all(ref.between(got[:, 128 * k: 128 * k + 128], t, 80 * E * np.abs(t), grid))


SHAPES = [(1, 8), (1, 4096), (2, 128), (3, 136), (5, 264), (7, 512), (33, 520), (9, 1000), (17, 2048), (5, 2056), (4, 4104), (3, 8192), (2, 8200), (2, 16384), (2, 24576), (1, 32768), (1000, 72)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("fp8", [True, False])
def test_row_outputs(api, rows, cols, residual, fp8):
    x, res, gain = rand(rows, cols, 1), rand(rows, cols, 2) if residual else None, gain_of(cols, residual)
    o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3 if fp8 else api.FMT_FP4_E2M1, want_y=True)
    h, rstd, y = ref.norm(f64(x), None if res is None else f64(res), f64(gain), EPS)
    assert np.array_equal(f64(o["h"]), h)
    assert np.all(np.abs(f64(o["rstd"]) - rstd) <= 36 * E * rstd)
    assert np.all(np.abs(f64(o["y"]) - y) <= (2.0 ** -8 + 40 * E) * np.abs(y))
    check_codes(o["codes"], o["scales"], y, fp8, False)
    # fewer outputs: the same values
    only = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res)
    assert only["codes"] is None and torch.equal(only["y"], o["y"]) and torch.equal(only["rstd"], o["rstd"])


@pytest.mark.parametrize("rows,cols", [(64, 64), (128, 128), (64, 192), (192, 320), (320, 576), (128, 4096), (1024, 512)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("fp8,fp8_t", [(True, True), (False, True), (True, False), (False, False)])
def test_both_copies(api, rows, cols, residual, fp8, fp8_t):
    fmts = {True: api.FMT_FP8_E4M3, False: api.FMT_FP4_E2M1}
    x, res, gain = rand(rows, cols, 3), rand(rows, cols, 4) if residual else None, gain_of(cols, not residual)
    o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=fmts[fp8], fmt_t=fmts[fp8_t])
    h, rstd, y = ref.norm(f64(x), None if res is None else f64(res), f64(gain), EPS)
    assert o["y"] is None and np.array_equal(f64(o["h"]), h)
    check_codes(o["codes"], o["scales"], y, fp8, False)
    check_codes(o["codes_t"], o["scales_t"], y, fp8_t, True)
    n = rows * cols if fp8 else rows * cols // 2
    row = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=fmts[fp8])
    assert torch.equal(row["codes"][:n], o["codes"][:n]) and torch.equal(row["scales"], o["scales"]) and torch.equal(row["rstd"], o["rstd"])
    # the transposed copy alone, beside y: a layer whose forward product keeps BF16
    n = rows * cols if fp8_t else rows * cols // 2
    t = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt_t=fmts[fp8_t], want_y=True)
    assert t["codes"] is None and torch.equal(t["codes_t"][:n], o["codes_t"][:n]) and torch.equal(t["scales_t"], o["scales_t"])
    assert np.all(np.abs(f64(t["y"]) - y) <= (2.0 ** -8 + 40 * E) * np.abs(y))


@pytest.mark.parametrize("rows,cols", [(64, 192), (320, 576), (448, 4096)])
@pytest.mark.parametrize("residual", [False, True])
def test_everything_at_once(api, rows, cols, residual):
    x, res, gain = rand(rows, cols, 8), rand(rows, cols, 9) if residual else None, gain_of(cols, True)
    o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP4_E2M1, fmt_t=api.FMT_FP8_E4M3, want_y=True)
    h, rstd, y = ref.norm(f64(x), None if res is None else f64(res), f64(gain), EPS)
    assert np.array_equal(f64(o["h"]), h) and np.all(np.abs(f64(o["rstd"]) - rstd) <= 36 * E * rstd)
    assert np.all(np.abs(f64(o["y"]) - y) <= (2.0 ** -8 + 40 * E) * np.abs(y))
    check_codes(o["codes"], o["scales"], y, False, False)
    check_codes(o["codes_t"], o["scales_t"], y, True, True)


@pytest.mark.parametrize("rows,cols,form", [(257, 512, "row"), (5000, 4096, "row"), (2049, 200, "row"), (4096, 1024, "dual"), (20480, 128, "dual")])
def test_many_rows(api, rows, cols, form):
    # more rows than the grid holds at a time: groups walk on; a few rows and columns of the result are compared
    x, res, gain = rand(rows, cols, 6), rand(rows, cols, 7), gain_of(cols, False)
    o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP8_E4M3 if form == "dual" else None)
    h, rstd, y = ref.norm(f64(x), f64(res), f64(gain), EPS)
    assert np.array_equal(f64(o["h"]), h)
    assert np.all(np.abs(f64(o["rstd"]) - rstd) <= 36 * E * rstd)
    check_codes(o["codes"], o["scales"], y, True, False)
    if form == "dual":
        check_codes(o["codes_t"], o["scales_t"], y, True, True)


def test_strides_and_what_lies_between_rows(api):
    rows, cols, ld = 70, 264, 304
    def strided(seed):
        t = rand(rows, ld, seed)
        return t, t[:, :cols]
    (_, x), (_, res) = strided(1), strided(2)
    hb, yb = torch.full((rows + 1, ld), 7.0, device="cuda", dtype=torch.bfloat16), torch.full((rows + 1, ld), 7.0, device="cuda", dtype=torch.bfloat16)
    gain = gain_of(cols, True)
    codes, scales = torch.full((rows * cols + 64,), 0x5A, dtype=torch.uint8, device="cuda"), torch.zeros(3 * rows, device="cuda")
    rstd = torch.full((rows + 8,), -1.0, device="cuda")
    o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3,
                             out={"h": hb[:rows, :cols], "y": yb[:rows, :cols], "rstd": rstd[:rows], "codes": codes, "scales": scales})
    want = api.snip_rmsnorm_fwd(x.contiguous(), gain, EPS, residual=res.contiguous(), fmt=api.FMT_FP8_E4M3, want_y=True)
    assert torch.equal(o["h"], want["h"]) and torch.equal(o["y"], want["y"]) and torch.equal(codes[:rows * cols], want["codes"]) and torch.equal(scales, want["scales"])
    for b in (hb, yb):
        assert torch.all(b[:rows, cols:] == 7) and torch.all(b[rows] == 7)
    assert torch.all(codes[rows * cols:] == 0x5A) and torch.all(rstd[rows:] == -1)


@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("target", ["residual", "x"])
def test_sum_in_place(api, dual, target):
    x, res, gain = rand(192, 448, 1), rand(192, 448, 2), gain_of(448, True)
    kw = dict(fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP8_E4M3 if dual else None)
    want = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, **kw)
    x2, res2 = x.clone(), res.clone()
    bufs = {k: torch.empty_like(v) for k, v in want.items() if v is not None and k != "h"}
    o = api.snip_rmsnorm_fwd(x2, gain, EPS, residual=res2, out={**bufs, "h": res2 if target == "residual" else x2}, **kw)
    for k in bufs:
        assert torch.equal(o[k], want[k]), k
    assert torch.equal(res2 if target == "residual" else x2, want["h"]) and torch.equal(x2 if target == "residual" else res2, x if target == "residual" else res)


def test_rows_of_zeros_and_extreme_magnitudes(api):
    cols = 256
    x = rand(8, cols, 1)
    x[0] = 0
    x[1] *= 2.0 ** -60          # far below eps: the norm is x / sqrt(eps)
    x[2] *= 2.0 ** 50
    x[3] = 0
    x[3, 200] = 3.0             # one entry: the other tile is empty
    x[4] = 2.0 ** -130          # subnormal in binary32
    gain = gain_of(cols, True)
    gain[:128] = 0.0            # every first tile is empty
    o = api.snip_rmsnorm_fwd(x, gain, EPS, fmt=api.FMT_FP8_E4M3, want_y=True)
    h, rstd, y = ref.norm(f64(x), None, f64(gain), EPS)
    assert np.all(np.abs(f64(o["rstd"]) - rstd) <= 36 * E * rstd)
    assert torch.all(o["y"][0] == 0) and torch.all(o["scales"].view(2, 8)[0] == 1) and torch.all(o["scales"].view(2, 8)[:, 0] == 1)
    assert torch.all(o["codes"].view(8, cols)[0] == 0) and torch.all(o["codes"].view(8, cols)[:, :128] & 127 == 0)
    keep = [0, 1, 2, 3, 5, 6, 7]
    check_codes(o["codes"].view(8, cols)[keep].reshape(-1), o["scales"].view(2, 8)[:, keep].reshape(-1), y[keep], True, False)
    # row 4: y of about 2^-121: 448 / y passes the largest binary32 number, at which the scale is clamped
    most = np.abs(y[4]).max()
    assert 448 / most > np.finfo(np.float32).max and float(o["scales"].view(2, 8)[1, 4]) == np.finfo(np.float32).max


def test_zero_rows_and_no_output_behind_the_last_row(api):
    gain = gain_of(128, True)
    o = api.snip_rmsnorm_fwd(torch.empty(0, 128, dtype=torch.bfloat16, device="cuda"), gain, EPS, fmt=api.FMT_FP8_E4M3, want_y=True)
    assert o["y"].shape == (0, 128)
    dgain = torch.full((128,), 3.0, device="cuda")
    none = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda")
    api.snip_rmsnorm_bwd(none, none, gain, torch.empty(0, device="cuda"), dgain=dgain, accumulate=True)
    assert torch.all(dgain == 3)
    api.snip_rmsnorm_bwd(none, none, gain, torch.empty(0, device="cuda"), dgain=dgain)
    assert torch.all(dgain == 0)


@pytest.mark.parametrize("rows,cols", SHAPES + [(300, 4096), (700, 1536), (4000, 256), (2500, 8192)])
@pytest.mark.parametrize("residual", [False, True])
def test_backward(api, rows, cols, residual):
    dy, h, gain = rand(rows, cols, 8, 1e-3), rand(rows, cols, 9), gain_of(cols, not residual)
    dres = rand(rows, cols, 10, 1e-3) if residual else None
    rstd = torch.from_numpy((1 / np.sqrt(np.mean(f64(h) ** 2, axis=1) + EPS)).astype(np.float32)).cuda()
    dx, dgain = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres)
    want, wgain = ref.norm_bwd(f64(dy), f64(h), f64(gain), f64(rstd), None if dres is None else f64(dres))
    g, u, r = np.abs(f64(dy) * f64(gain)), np.abs(f64(h) * f64(rstd)[:, None]), f64(rstd)[:, None]
    # g: one rounding; u: one; mean: 64 + those; the rest three
    slack = E * r * (4 * g + u * 70 * np.mean(g * u, axis=1, keepdims=True)) + 2 * E * np.abs(0 if dres is None else f64(dres))
    assert np.all(np.abs(f64(dx) - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * slack)
    # a column's sum: a group of rows adds its share (148 groups or more where there are as many rows), 32 threads add the groups, one the threads;
    # each term has three roundings of its own
    assert np.all(np.abs(f64(dgain) - wgain) <= (rows / 148 + rows / 32 + 40) * E * (np.abs(f64(dy)) * u).sum(0))
    again = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres, dgain=dgain.clone(), accumulate=True)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain + dgain)
    frozen = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres, want_dgain=False)
    assert frozen[1] is None and torch.equal(frozen[0], dx)


def test_backward_in_place_and_strides(api):
    rows, cols, ld = 130, 520, 640
    gain, rstd = gain_of(cols, False), torch.rand(rows, device="cuda") + 0.5
    dy, h, dres = rand(rows, ld, 1, 1e-3)[:, :cols], rand(rows, ld, 2)[:, :cols], rand(rows, ld, 3, 1e-3)[:, :cols]
    want = api.snip_rmsnorm_bwd(dy.contiguous(), h.contiguous(), gain, rstd, dresidual=dres.contiguous())
    out = torch.full((rows + 1, ld), 7.0, device="cuda", dtype=torch.bfloat16)
    got = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres, dx=out[:rows, :cols])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.all(out[:rows, cols:] == 7) and torch.all(out[rows] == 7)
    for place in ("dy", "dres"):
        a, b = dy.clone(), dres.clone()
        got = api.snip_rmsnorm_bwd(a, h, gain, rstd, dresidual=b, dx=a if place == "dy" else b)
        assert torch.equal(a if place == "dy" else b, want[0]) and torch.equal(got[1], want[1])


def test_gradient_by_differences(api):
    # the loss sum(dy y) of the forward kernel's own bf16-free quantity, the 64-bit form, moved by one step of x in bf16
    rows, cols = 4, 320
    x, dy, gain = rand(rows, cols, 1), rand(rows, cols, 2, 0.1), gain_of(cols, True)
    o = api.snip_rmsnorm_fwd(x, gain, EPS)
    dx, dgain = api.snip_rmsnorm_bwd(dy, x, gain, o["rstd"])
    X, DY, G = f64(x), f64(dy), f64(gain)
    for r, c in ((0, 0), (1, 111), (3, 319)):
        e = np.zeros_like(X)
        e[r, c] = 1e-5
        num = ((DY * ref.norm(X + e, None, G, EPS)[2]).sum() - (DY * ref.norm(X - e, None, G, EPS)[2]).sum()) / 2e-5
        # the difference itself is good to 1e-9; dx is rounded to bf16, and rstd to binary32
        assert abs(num - f64(dx)[r, c]) <= 2.0 ** -8 * abs(num) + 1e-6 * np.abs(DY[r] * G).max()
    e = np.zeros_like(G)
    e[7] = 1e-5
    num = ((DY * ref.norm(X, None, G + e, EPS)[2]).sum() - (DY * ref.norm(X, None, G - e, EPS)[2]).sum()) / 2e-5
    assert abs(num - f64(dgain)[7]) <= 1e-5 * (np.abs(DY[:, 7]) * 10).sum()


def test_captured_replays_read_new_inputs(api):
    rows, cols = 256, 512
    gain = gain_of(cols, False)
    x, res, dy = rand(rows, cols, 1), rand(rows, cols, 2), rand(rows, cols, 3, 1e-3)
    out = {k: v for k, v in api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP8_E4M3).items() if v is not None}
    ws = torch.empty(api.snip_rmsnorm_bwd_workspace(rows, cols), dtype=torch.uint8, device="cuda")
    dx, dgain = torch.empty_like(x), torch.empty(cols, device="cuda")
    def step():
        api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP8_E4M3, out=out)
        api.snip_rmsnorm_bwd(dy, out["h"], gain, out["rstd"], dresidual=res, dx=dx, dgain=dgain, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (11, 12):
        x.copy_(rand(rows, cols, seed)); dy.copy_(rand(rows, cols, seed + 50, 1e-3))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        gdx, gg = dx.clone(), dgain.clone()
        want = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP8_E4M3)
        wdx, wg = api.snip_rmsnorm_bwd(dy, want["h"], gain, want["rstd"], dresidual=res)
        for k in got:
            assert torch.equal(got[k], want[k]), k
        assert torch.equal(gdx, wdx) and torch.equal(gg, wg)


def test_two_streams_at_once(api):
    rows, cols = 2048, 1024
    gain = gain_of(cols, True)
    ins = [(rand(rows, cols, 20 + i), rand(rows, cols, 30 + i), rand(rows, cols, 40 + i, 1e-3)) for i in range(2)]
    def both(x, res, dy):
        o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP4_E2M1)
        return [o[k] for k in ("h", "rstd", "codes", "scales", "codes_t", "scales_t")] + list(api.snip_rmsnorm_bwd(dy, o["h"], gain, o["rstd"], dresidual=res))
    want = [both(*i) for i in ins]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ins]
    got = []
    for _ in range(3):
        got = []
        for s, i in zip(streams, ins):
            with torch.cuda.stream(s):
                got.append(both(*i))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for p, q in zip(a, b):
            assert torch.equal(p, q)


def test_offsets_beyond_32_bits(api):
    # rows a long way apart: element offsets pass 2^31
    rows, cols, ld = 70000, 64, 32768 + 64
    flat = torch.zeros(rows * ld, dtype=torch.bfloat16, device="cuda")
    x = flat.view(rows, ld)[:, :cols]
    x.copy_(rand(rows, cols, 1))
    gain = gain_of(cols, True)
    o = api.snip_rmsnorm_fwd(x, gain, EPS, out={"y": flat.view(rows, ld)[:, 128:128 + cols]})
    want = api.snip_rmsnorm_fwd(x.contiguous(), gain, EPS)
    assert torch.equal(o["y"], want["y"])
    dx, dgain = api.snip_rmsnorm_bwd(x, o["y"], gain, want["rstd"], dx=flat.view(rows, ld)[:, 256:256 + cols])
    dx2, dgain2 = api.snip_rmsnorm_bwd(x.contiguous(), want["y"], gain, want["rstd"])
    assert torch.equal(dx, dx2) and torch.equal(dgain, dgain2)


def test_refusals_of_the_library_reach_the_caller(api):
    x, gain = rand(100, 128, 1), gain_of(128, True)
    with pytest.raises(api.SnipError):
        api.snip_rmsnorm_fwd(x, gain, EPS, fmt_t=api.FMT_FP8_E4M3)          # 100 rows have no 128x1 tiles for the products
    with pytest.raises(api.SnipError):
        api.snip_rmsnorm_fwd(x, gain, 0.0)
    with pytest.raises(api.SnipError):
        api.snip_rmsnorm_bwd(x, x, gain, torch.ones(100, device="cuda"), ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(api.SnipError):
        api.snip_rmsnorm_bwd(x[:1].expand(100, 128), x, gain, torch.ones(100, device="cuda"))   # a broadcast gradient: row stride 0
    with pytest.raises(ValueError):
        api.snip_rmsnorm_fwd(x, gain.cpu(), EPS)
