"""What the norm and the optimizer step refuse, on the host and before anything is enqueued (no device is needed, none is touched)."""
import ctypes
import math

import pytest
import torch

P, Q = 0x10000, 0x20000


@pytest.fixture(scope="module")
def api():
    from paper_2602_01410_b200 import build
    build.build()
    from paper_2602_01410_b200 import api
    return api


def fwd(api, **kw):
    a = api.RmsNorm(x=P, gain=P, y=Q, rows=128, cols=128, ld_x=128, ld_residual=128, ld_h=128, ld_y=128, eps=1e-5, gain_dtype=0, fmt=1, fmt_t=1)
    for k, v in kw.items():
        setattr(a, k, v)
    return api._lib.snip_rmsnorm_fwd(ctypes.byref(a), None)


def test_norm_forward(api):
    assert api._lib.snip_rmsnorm_fwd(None, None) == api.ERR_ARG
    for kw in (dict(x=None), dict(gain=None), dict(gain_dtype=2), dict(y=None), dict(residual=P), dict(h=Q), dict(codes=Q), dict(scales=Q), dict(codes_t=Q),
               dict(codes=Q, scales=Q, fmt=0), dict(codes=Q, scales=Q, fmt=3), dict(codes_t=Q, scales_t=Q, rstd=Q, fmt_t=0), dict(codes_t=Q, scales_t=Q),
               dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan)):
        assert fwd(api, **kw) == api.ERR_ARG, kw
    for kw in (dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=-8), dict(cols=100), dict(cols=32776, ld_x=32776, ld_y=32776), dict(ld_x=120), dict(ld_x=132),
               dict(ld_y=64), dict(residual=P, h=Q, ld_residual=0), dict(residual=P, h=Q, ld_h=127), dict(codes_t=Q, scales_t=Q, rstd=Q, rows=100),
               dict(codes_t=Q, scales_t=Q, rstd=Q, cols=136, ld_x=136, ld_y=136)):
        assert fwd(api, **kw) == api.ERR_SHAPE, kw
    for name in ("x", "gain", "y", "rstd"):
        assert fwd(api, **{name: P + 8}) == api.ERR_ALIGN, name
    for kw in (dict(residual=P + 2, h=Q), dict(residual=P, h=Q + 4), dict(codes=Q + 8, scales=Q), dict(codes=Q, scales=Q + 4), dict(codes_t=Q, scales_t=Q + 8, rstd=Q)):
        assert fwd(api, **kw) == api.ERR_ALIGN, kw
    assert fwd(api, ld_x=1 << 31) == api.ERR_SHAPE
    assert fwd(api, rows=0) == api.OK      # nothing to do


def test_norm_forward_refuses_one_address_for_two(api):
    full = dict(residual=0x30000, h=0x40000, rstd=0x50000, codes=0x60000, scales=0x70000, codes_t=0x80000, scales_t=0x90000, x=0xA0000, gain=0xB0000, y=0xC0000)
    outs = ("h", "y", "rstd", "codes", "scales", "codes_t", "scales_t")
    for i, a in enumerate(outs):
        for b in outs[i + 1:]:
            assert fwd(api, **{**full, a: full[b]}) == api.ERR_ARG, (a, b)
        for b in ("x", "residual", "gain"):
            if a != "h" or b == "gain":
                assert fwd(api, **{**full, a: full[b]}) == api.ERR_ARG, (a, b)
    # the sum in place: with the same stride only
    assert fwd(api, **{**full, "h": full["x"], "ld_x": 136}) == api.ERR_ARG
    assert fwd(api, **{**full, "h": full["residual"], "ld_residual": 136}) == api.ERR_ARG


def test_norm_backward_refuses_one_address_for_two(api):
    full = dict(dy=0x30000, h=0x40000, gain=0x50000, rstd=0x60000, dresidual=0x70000, dx=0x80000, dgain=0x90000)
    for a, b in (("dx", "h"), ("dx", "gain"), ("dx", "rstd"), ("dgain", "gain"), ("dgain", "rstd"), ("dgain", "dy"), ("dgain", "h"), ("dgain", "dresidual"), ("dgain", "dx")):
        assert bwd(api, **{**full, a: full[b]}) == api.ERR_ARG, (a, b)
    assert bwd(api, ws=full["dgain"], **full) == api.ERR_ARG
    assert bwd(api, **{**full, "dx": full["dy"], "ld_dy": 136}) == api.ERR_ARG
    assert bwd(api, **{**full, "dx": full["dresidual"], "ld_dresidual": 136}) == api.ERR_ARG


def bwd(api, ws=P, size=1 << 40, **kw):
    a = api.RmsNormBwd(dy=P, h=P, gain=P, rstd=P, dx=Q, dgain=Q + 0x8000, rows=128, cols=128, ld_dy=128, ld_h=128, ld_dresidual=128, ld_dx=128, gain_dtype=1)
    for k, v in kw.items():
        setattr(a, k, v)
    return api._lib.snip_rmsnorm_bwd(ctypes.byref(a), ws, size, None)


def test_norm_backward(api):
    assert api._lib.snip_rmsnorm_bwd(None, None, 0, None) == api.ERR_ARG
    for name in ("dy", "h", "gain", "rstd", "dx"):
        assert bwd(api, **{name: None}) == api.ERR_ARG, name
    assert bwd(api, gain_dtype=-1) == api.ERR_ARG
    for kw in (dict(rows=-1), dict(cols=12), dict(cols=0), dict(ld_dy=8), dict(ld_h=130), dict(ld_dx=0), dict(dresidual=P, ld_dresidual=100)):
        assert bwd(api, **kw) == api.ERR_SHAPE, kw
    for kw in (dict(dy=P + 8), dict(h=P + 2), dict(gain=P + 4), dict(rstd=P + 4), dict(dx=Q + 8), dict(dgain=Q + 0x8004), dict(dresidual=P + 8), dict(ws=P + 8)):
        assert bwd(api, **kw) == api.ERR_ALIGN, kw
    need = api.snip_rmsnorm_bwd_workspace(128, 128)
    assert need >= 4 * 128 and need % 256 == 0
    assert bwd(api, ws=None, size=0) == api.ERR_WORKSPACE
    assert bwd(api, size=need - 1) == api.ERR_WORKSPACE
    n = ctypes.c_size_t()
    assert api._lib.snip_rmsnorm_bwd_workspace(128, 128, None) == api.ERR_ARG
    assert api._lib.snip_rmsnorm_bwd_workspace(128, 100, ctypes.byref(n)) == api.ERR_SHAPE
    assert api.snip_rmsnorm_bwd_workspace(0, 128) == 0


def test_norm_backward_workspace_covers_every_row_group(api):
    # never less than one partial of all columns, and bounded however many rows there are
    for cols in (8, 256, 512, 2048, 4096, 8192, 32768):
        few, many = api.snip_rmsnorm_bwd_workspace(1, cols), api.snip_rmsnorm_bwd_workspace(1 << 30, cols)
        assert few >= 4 * cols and many <= 1 << 30


def adamw(api, count=1, tensor=None, **kw):
    t = api.AdamwTensor(param=P, grad=P + 0x1000, m=P + 0x2000, v=P + 0x3000, n=64)
    for k, v in (tensor or {}).items():
        setattr(t, k, v)
    a = api.Adamw(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1, param_dtype=1, grad_dtype=1, state_bits=32)
    for k, v in kw.items():
        setattr(a, k, v)
    return api._lib.snip_adamw_step(ctypes.byref(t), count, ctypes.byref(a), None)


def test_optimizer_step(api):
    assert api._lib.snip_adamw_step(None, 0, None, None) == api.ERR_ARG
    assert adamw(api, count=-1) == api.ERR_ARG
    assert adamw(api, count=0) == api.OK
    for kw in (dict(param_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(rounding=2), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1),
               dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=math.inf), dict(step=0), dict(step=-3), dict(state_bits=8),
               dict(tensor=dict(param=None)), dict(tensor=dict(grad=None)), dict(tensor=dict(m=None)), dict(tensor=dict(v=None)), dict(tensor=dict(m_scale=P)),
               dict(state_bits=8, tensor=dict(m_scale=P)), dict(param_dtype=0, tensor=dict(param_bf16=P)), dict(tensor=dict(weight_decay=math.nan))):
        assert adamw(api, **kw) == api.ERR_ARG, kw
    for n in (-1, 1 << 41):
        assert adamw(api, tensor=dict(n=n)) == api.ERR_SHAPE
    for kw in (dict(tensor=dict(param=P + 4)), dict(tensor=dict(grad=P + 8)), dict(tensor=dict(m=P + 2)), dict(tensor=dict(v=P + 8)), dict(tensor=dict(param_bf16=P + 2)),
               dict(state_bits=8, tensor=dict(m_scale=P + 2, v_scale=P)), dict(step_device=P + 4), dict(lr_device=P + 2), dict(grad_scale=P + 1)):
        assert adamw(api, **kw) == api.ERR_ALIGN, kw
    assert api.snip_adamw_state_sizes(129, 8) == (129, 8)
    assert api.snip_adamw_state_sizes(129, 32) == (516, 0)
    assert api.snip_adamw_state_sizes(0, 8) == (0, 0)
    with pytest.raises(api.SnipError):
        api.snip_adamw_state_sizes(5, 4)
    with pytest.raises(api.SnipError):
        api.snip_adamw_state_sizes(-1, 8)


def test_more_chunks_than_a_launch_counts_are_refused(api):
    ts = (api.AdamwTensor * 40)(*[api.AdamwTensor(param=P, grad=P, m=P, v=P, n=1 << 40) for _ in range(40)])
    a = api.Adamw(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1, param_dtype=1, grad_dtype=1, state_bits=32)
    assert api._lib.snip_adamw_step(ts, 40, ctypes.byref(a), None) == api.ERR_SHAPE


def test_binding_refuses_host_tensors_and_wrong_types(api):
    bf = torch.bfloat16
    x, gain = torch.zeros(4, 64, dtype=bf), torch.ones(64)
    for call in (lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5),                                        # on the host
                 lambda: api.snip_rmsnorm_fwd(x.float(), gain, 1e-5),
                 lambda: api.snip_rmsnorm_fwd(x[0], gain, 1e-5),
                 lambda: api.snip_rmsnorm_fwd(x.t(), torch.ones(4), 1e-5),                           # rows not contiguous
                 lambda: api.snip_rmsnorm_fwd(x, gain[:32], 1e-5),
                 lambda: api.snip_rmsnorm_fwd(x, gain.double(), 1e-5),
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, residual=x[:2]),
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, fmt=7),
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, out={"codes_t": None, "norm": x}),
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, out={"h": x.clone()}),                  # no residual
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, residual=x, out={"y": x.clone()}),      # nowhere for the sum
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, fmt=1, out={"codes": torch.zeros(256, dtype=torch.uint8)}),
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, fmt=1, out={"codes": torch.zeros(255, dtype=torch.uint8), "scales": torch.zeros(4)}),
                 lambda: api.snip_rmsnorm_fwd(x, gain, 1e-5, fmt=1, out={"codes": torch.zeros(256, dtype=torch.uint8), "scales": torch.zeros(5)}),
                 lambda: api.snip_rmsnorm_bwd(x, x, gain, torch.zeros(4)),
                 lambda: api.snip_rmsnorm_bwd(x, x, gain, torch.zeros(5)),
                 lambda: api.snip_rmsnorm_bwd(x, x.half(), gain, torch.zeros(4)),
                 lambda: api.snip_rmsnorm_bwd(x, x, gain, torch.zeros(4), accumulate=True)):
        with pytest.raises(ValueError):
            call()


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device, for the checks of lists (nothing is launched)."""
    is_cuda = True

    def get_device(self):
        return 0


def test_binding_refuses_overlapping_and_mismatched_lists(api):
    def t(n, dtype=torch.float32):
        return torch.zeros(n, dtype=dtype).as_subclass(OnDevice)

    whole = t(256)
    ok = api.make_adamw_tensors([whole[:128], whole[128:]], [t(128), t(128)], [t(128), t(128)], [t(128), t(128)], copies=[t(128, torch.bfloat16), None], weight_decay=[0.1, 0.0])
    assert ok.count == 2 and ok.state_bits == 32 and abs(ok.table[0].weight_decay - 0.1) < 1e-7 and ok.table[1].param_bf16 is None
    shared = t(64)
    u8 = lambda n: t(n, torch.uint8)  # noqa: E731
    for args, kw in ((([whole[:128], whole[64:192]], [t(128)] * 2, [t(128), t(128)], [t(128), t(128)]), {}),       # parameters overlap
                     (([shared, shared], [t(64)] * 2, [t(64), t(64)], [t(64), t(64)]), {}),                        # the same one twice
                     (([shared], [t(64)], [t(64)], [shared]), {}),                                                  # a state on a parameter
                     (([shared], [shared], [t(64)], [t(64)]), {}),                                                  # its own gradient
                     (([t(64)], [t(63)], [t(64)], [t(64)]), {}),
                     (([t(64)], [t(64)], [t(64)], []), {}),
                     (([t(64), t(64, torch.bfloat16)], [t(64), t(64)], [t(64), t(64)], [t(64), t(64)]), {}),
                     (([t(64)], [t(64)], [u8(64)], [u8(64)]), {}),                                                  # no scales
                     (([t(64)], [t(64)], [u8(64)], [u8(64)]), dict(m_scales=[t(1)], v_scales=[t(2)])),
                     (([t(64)], [t(64)], [t(64)], [t(64)]), dict(m_scales=[t(1)], v_scales=[t(1)])),
                     (([t(64, torch.bfloat16)], [t(64)], [t(64)], [t(64)]), dict(copies=[t(64, torch.bfloat16)])),
                     (([t(64)], [t(64)], [t(64)], [t(64)]), dict(weight_decay=[0.1, 0.2])),
                     (([t(128)[::2]], [t(64)], [t(64)], [t(64)]), {})):
        with pytest.raises(ValueError):
            api.make_adamw_tensors(*args, **kw)
    api.make_adamw_tensors([t(64), t(64)], [shared, shared], [t(64), t(64)], [t(64), t(64)])    # gradients may be shared: they are only read
    assert api.make_adamw_tensors([], [], [], []).count == 0
    for kw in (dict(seed=-1), dict(seed=1 << 64), dict(grad_scale=torch.ones(1))):
        with pytest.raises(ValueError):
            api.snip_adamw_step(ok, 1e-3, 0.9, 0.95, 1e-8, 1, **kw)


def test_packed_arguments_have_the_structures_layout(api):
    # what the binding packs is read back field by field through the structure
    a = api.RmsNorm.from_buffer_copy(api._RMSNORM_ARGS(*range(1, 17), 0.5, 17, 18, 19))
    assert ctypes.sizeof(a) == 144 and [getattr(a, n) for n, _ in a._fields_] == list(range(1, 17)) + [0.5, 17, 18, 19]
    b = api.RmsNormBwd.from_buffer_copy(api._RMSNORM_BWD_ARGS(*range(1, 16)))
    assert ctypes.sizeof(b) == 112 and [getattr(b, n) for n, _ in b._fields_] == list(range(1, 16))
    c = api.Adamw.from_buffer_copy(api._ADAMW_ARGS(0.5, 0.25, 0.125, 2.0, 5, 6, 7, 8, (1 << 64) - 1, 10, 11, 12, 13))
    assert ctypes.sizeof(c) == 88 and [getattr(c, n) for n, _ in c._fields_] == [0.5, 0.25, 0.125, 2.0, 5, 6, 7, 8, (1 << 64) - 1, 10, 11, 12, 13]
