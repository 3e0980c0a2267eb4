"""Every kernel of the norm over rows enough for a CTA to come back to its ring's slots, against the 64-bit forms.

The 64-bit forms are computed on the device here (the numpy ones of the other tests would take minutes).  Tolerances as there: with e = 2^-24, rstd 36 e,
y 38 e and half a bf16 step, a scale 39 e, a code what some value within 80 e is rounded to."""
import pytest
import torch

import norm_forms as nf
import operator_refs as ref

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def api():
    from paper_2602_01410_b200 import api
    return api


def rand(rows, cols, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(rows, cols, generator=g, device="cuda") * scale
    t[:, ::37] *= 20
    # rows differ in size, so that one row's sum in the place of another's shows
    return (t * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(torch.bfloat16)


def gain_of(cols, f32):
    g = torch.Generator(device="cuda").manual_seed(5)
    t = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    return t if f32 else t.to(torch.bfloat16)


def nearest(t, grid):
    """ref.nearest on the device."""
    a = t.abs().clamp(max=grid[-1].item())
    hi = torch.searchsorted(grid, a).clamp(1, len(grid) - 1)
    up, down = grid[hi] - a, a - grid[hi - 1]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return torch.copysign(grid[pick], t)


def check_codes(codes, scales, y, fmt):
    """Row codes and scales against the 64-bit y, some rows at a time."""
    rows, cols = y.shape
    fp8 = fmt == 1
    grid = torch.from_numpy(ref.E4M3 if fp8 else ref.E2M1).cuda()
    if fp8:
        got = codes[:rows * cols].view(torch.float8_e4m3fn).view(rows, cols)
        assert not torch.any(codes[:rows * cols] & 127 == 127)
    else:
        c = codes[:rows * cols // 2].view(rows, cols // 2)
        c = torch.stack([c & 15, c >> 4], -1).view(rows, cols).long()
        got = torch.where(c & 8 > 0, -1.0, 1.0) * grid[c & 7]
    tiles = -(-cols // 128)
    s = scales.view(tiles, rows).double()
    for a in range(0, rows, 1024):
        part = torch.nn.functional.pad(y[a: a + 1024], (0, tiles * 128 - cols)).view(-1, tiles, 128)
        most = part.abs().amax(2)
        want = torch.where(most > 0, grid[-1] / most, 1.0)
        assert torch.all((s[:, a: a + 1024].t() - want).abs() <= 40 * E * want)
        t = (part * want[:, :, None]).view(-1, tiles * 128)[:, :cols]
        lo, hi = nearest(t * (1 - 80 * E), grid), nearest(t * (1 + 80 * E), grid)
        q = got[a: a + 1024].double()
        assert torch.all((q >= torch.minimum(lo, hi)) & (q <= torch.maximum(lo, hi)))


@pytest.mark.parametrize("rows,cols,residual,y,fmt", nf.FORWARD)
def test_forward(api, rows, cols, residual, y, fmt):
    x, res, gain = rand(rows, cols, 1), rand(rows, cols, 2) if residual else None, gain_of(cols, rows % 2 == 0)
    guard = 64
    out = {"rstd": torch.full((rows + guard,), -1.0, device="cuda")[:rows]}
    whole = {}

    def buffer(name, n, dtype, fill):
        whole[name] = (torch.full((n + guard,), fill, dtype=dtype, device="cuda"), n, fill)
        return whole[name][0][:n]

    if residual:
        out["h"] = buffer("h", rows * cols, torch.bfloat16, 7.0).view(rows, cols)
    if y:
        out["y"] = buffer("y", rows * cols, torch.bfloat16, 7.0).view(rows, cols)
    tiles = -(-cols // 128)
    if fmt:
        n = api.snip_quantize_sizes(rows, cols, fmt, api.BLOCK_ROW)[0] if rows % 64 == 0 and cols % 64 == 0 else (rows * cols if fmt == 1 else rows * cols // 2 + 64)
        out["codes"], out["scales"] = buffer("codes", n, torch.uint8, 0x5A), buffer("scales", tiles * rows, torch.float32, -1.0)
    api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=fmt or None, out=out)
    h = x.double() if res is None else (x.double() + res.double()).to(torch.bfloat16).double()
    if residual:
        assert torch.equal(out["h"].double(), h)
    rstd = (h.square().mean(1) + EPS) ** -0.5
    assert torch.all((out["rstd"].double() - rstd).abs() <= 36 * E * rstd)
    z = h * rstd[:, None] * gain.double()
    del h
    if y:
        assert torch.all((out["y"].double() - z).abs() <= (2.0 ** -8 + 40 * E) * z.abs())
    if fmt:
        check_codes(out["codes"], out["scales"], z, fmt)
    for name, (t, n, fill) in whole.items():
        assert torch.all(t[n:] == fill), name
    # the same call again: the same bits
    again = {k: torch.empty_like(t) for k, t in out.items()}
    api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=fmt or None, out=again)
    for k in out:
        n = rows * cols // 2 if k == "codes" and fmt == 2 else None
        assert torch.equal(out[k].view(-1)[:n], again[k].view(-1)[:n]), k


@pytest.mark.parametrize("rows,cols,residual", nf.BACKWARD)
def test_backward(api, rows, cols, residual):
    dy, h, gain = rand(rows, cols, 8, 1e-3), rand(rows, cols, 9), gain_of(cols, rows % 2 == 0)
    dres = rand(rows, cols, 10, 1e-3) if residual else None
    rstd = ((h.double().square().mean(1) + EPS) ** -0.5).float()
    # exactly the bytes that were asked for, with a guard behind them
    size = api.snip_rmsnorm_bwd_workspace(rows, cols)
    ws = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    dx_whole = torch.full((rows * cols + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    dgain_whole = torch.full((cols + 64,), 7.0, device="cuda")
    dx, dgain = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres, dx=dx_whole[:rows * cols].view(rows, cols), dgain=dgain_whole[:cols], ws=ws[:size])
    assert torch.all(ws[size:] == 0xA5) and torch.all(dx_whole[rows * cols:] == 7) and torch.all(dgain_whole[cols:] == 7)
    r = rstd.double()[:, None]
    u, g = h.double() * r, dy.double() * gain.double()
    want = r * (g - u * (g * u).mean(1, keepdim=True))
    # g: one rounding; u: one; mean: 64 + those; the rest three (as in the other test of the backward pass)
    slack = E * r * (4 * g.abs() + u.abs() * 70 * (g * u).abs().mean(1, keepdim=True))
    if residual:
        want += dres.double()
        slack += 2 * E * dres.double().abs()
    assert torch.all((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * slack)
    del want, slack, g
    dyu = dy.double() * u
    assert torch.all((dgain.double() - dyu.sum(0)).abs() <= (rows / 148 + rows / 32 + 40) * E * dyu.abs().sum(0))
    del dyu, u
    again = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres, dgain=dgain.clone(), accumulate=True)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dgain + dgain)
    frozen = api.snip_rmsnorm_bwd(dy, h, gain, rstd, dresidual=dres, want_dgain=False)
    assert frozen[1] is None and torch.equal(frozen[0], dx)


@pytest.mark.parametrize("rows,cols", [(2048, 8192), (1216, 5120), (4096, 3200), (1216, 16384), (640, 32768)])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("fmt,fmt_t", [(1, 1), (2, 1), (None, 2)])
def test_both_copies(api, rows, cols, residual, fmt, fmt_t):
    x, res, gain = rand(rows, cols, 3), rand(rows, cols, 4) if residual else None, gain_of(cols, residual)
    o = api.snip_rmsnorm_fwd(x, gain, EPS, residual=res, fmt=fmt, fmt_t=fmt_t)
    h = x.double() if res is None else (x.double() + res.double()).to(torch.bfloat16).double()
    assert torch.equal(o["h"].double(), h)
    z = h * ((h.square().mean(1) + EPS) ** -0.5)[:, None] * gain.double()
    del h
    if fmt:
        check_codes(o["codes"], o["scales"], z, fmt)
    check_codes(o["codes_t"], o["scales_t"], z.t().contiguous(), fmt_t)
