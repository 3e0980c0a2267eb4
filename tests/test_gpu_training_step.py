"""The operators as a training step uses them: norm with both quantized copies -> products of a linear layer -> norm backward -> AdamW on the weight and the
gain.  Every stage is compared with its 64-bit form on the values that the stage before it left on the device."""
import numpy as np
import pytest
import torch

import operator_refs as ref

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


def f64(t):
    return t.double().cpu().numpy()


def dequantized(codes, scales, lines, along, fp8):
    s = f64(scales).reshape(-(-along // 128), lines)
    return ref.code_values(codes.cpu().numpy(), fp8, lines, along) / np.repeat(s, 128, axis=0)[:along].T


def rel(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


@pytest.mark.parametrize("M,K,N,fp8,bits", [(256, 512, 384, True, 8), (320, 448, 256, True, 32), (256, 512, 256, False, 8)])
def test_a_layer_step(M, K, N, fp8, bits):
    from paper_2602_01410_b200 import api
    fmt = api.FMT_FP8_E4M3 if fp8 else api.FMT_FP4_E2M1
    g = torch.Generator(device="cuda").manual_seed(M)
    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")
    x, residual = normal(M, K).to(torch.bfloat16), normal(M, K).to(torch.bfloat16)
    master = 0.02 * normal(N, K)
    weight = master.to(torch.bfloat16)
    gain = 1 + 0.1 * normal(K)
    dy = (1e-3 * normal(M, N)).to(torch.bfloat16)
    dres = (1e-3 * normal(M, K)).to(torch.bfloat16)

    # forward: the norm's codes go to the product as they are
    o = api.snip_rmsnorm_fwd(x, gain, 1e-5, residual=residual, fmt=fmt, fmt_t=fmt)
    wq, wqt = api.snip_quantize_dual(weight, api.DUAL_BLK_BLKT, fmt, fmt, want_stats=False)
    X = api.make_qtensor(o["codes"], o["scales"], M, K, fmt, api.BLOCK_ROW)
    W = api.make_qtensor(wq["codes"], wq["scales"], N, K, fmt, api.BLOCK_BLK)
    y = api.snip_gemm_quantized(api.OP_FWD, X, W, (M, N), api.OUT_FP32)
    xhat = dequantized(o["codes"], o["scales"], M, K, fp8)
    ws = np.repeat(np.repeat(f64(wq["scales"]).reshape(-(-N // 128), -(-K // 128)), 128, 0)[:N], 128, 1)[:, :K]
    what = ref.code_values(wq["codes"].cpu().numpy(), fp8, N, K) / ws
    assert rel(f64(y), xhat @ what.T) <= 1e-5
    # and stand for the normalised activations: the quantization error of the format, about 2.6 % (FP8) and 11 % (FP4) of a normal tile
    h, rstd, yn = ref.norm(f64(x), f64(residual), f64(gain), 1e-5)
    assert rel(xhat, yn) <= (0.04 if fp8 else 0.16)

    # backward: input gradient -> norm backward, weight gradient from the transposed copy
    dq, dqt = api.snip_quantize_dual(dy, api.DUAL_ROW_COLT, fmt, fmt, want_stats=False)
    dX = api.snip_gemm_quantized(api.OP_DGRAD, api.make_qtensor(dq["codes"], dq["scales"], M, N, fmt, api.BLOCK_ROW),
                                 api.make_qtensor(wqt["codes"], wqt["scales"], N, K, fmt, api.BLOCK_BLK, True), (M, K))
    dW = api.snip_gemm_quantized(api.OP_WGRAD, api.make_qtensor(dqt["codes"], dqt["scales"], M, N, fmt, api.BLOCK_COL, True),
                                 api.make_qtensor(o["codes_t"], o["scales_t"], M, K, fmt, api.BLOCK_COL, True), (N, K), api.OUT_FP32)
    xhat_t, dyhat_t = dequantized(o["codes_t"], o["scales_t"], K, M, fp8), dequantized(dqt["codes"], dqt["scales"], N, M, fp8)
    assert rel(f64(dW), dyhat_t @ xhat_t.T) <= 1e-5
    dx, dgain = api.snip_rmsnorm_bwd(dX, o["h"], gain, o["rstd"], dresidual=dres)
    want, wgain = ref.norm_bwd(f64(dX), h, f64(gain), f64(o["rstd"]), f64(dres))
    assert rel(f64(dx), want) <= 2.0 ** -8 and rel(f64(dgain), wgain) <= 1e-5

    # the step: weight (with the bf16 copy that the next forward pass quantizes) and gain
    params, grads = [master, gain], [dW, dgain]
    before = [f64(p) for p in params]
    copies = [weight, None]
    state = torch.uint8 if bits == 8 else torch.float32
    m, v = ([torch.zeros(p.numel(), dtype=state, device="cuda") for p in params] for _ in range(2))
    ms, vs = ([torch.zeros(-(-p.numel() // 128), device="cuda") for p in params] if bits == 8 else None for _ in range(2))
    t = api.make_adamw_tensors(params, grads, m, v, m_scales=ms, v_scales=vs, copies=copies, weight_decay=[0.1, 0.0])
    api.snip_adamw_step(t, 1e-3, 0.9, 0.95, 1e-8, 1, rounding=api.ROUND_STOCHASTIC, seed=1)
    for p, q, gr, wd in zip(params, before, grads, (float(np.float32(0.1)), 0.0)):
        want, *_ = ref.adamw(q, f64(gr), np.zeros(q.shape), np.zeros(q.shape), 1e-3, 0.9, 0.95, 1e-8, 1, wd)
        # an update of 1e-3 or less, good to 20 halves of a step, and the weight's own rounding
        assert np.all(np.abs(f64(p) - want) <= 4 * E * np.abs(q) + 20 * E * 1e-3)
    assert torch.equal(weight, master.to(torch.bfloat16))

    # the next step's forward pass starts from the written copy
    again, _ = api.snip_quantize_dual(weight, api.DUAL_BLK_BLKT, fmt, fmt, want_stats=False)
    assert not torch.equal(again["codes"], wq["codes"])


def test_the_step_in_one_graph():
    # everything above captured once and replayed: the same bits as call by call
    from paper_2602_01410_b200 import api
    M, K, N, F8 = 256, 256, 256, api.FMT_FP8_E4M3
    g = torch.Generator(device="cuda").manual_seed(5)
    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")
    x, residual, dy = normal(M, K).to(torch.bfloat16), normal(M, K).to(torch.bfloat16), (1e-3 * normal(M, N)).to(torch.bfloat16)

    class State:
        def __init__(self):
            gg = torch.Generator(device="cuda").manual_seed(9)
            self.master = 0.02 * torch.randn(N, K, generator=gg, device="cuda")
            self.gain = torch.ones(K, device="cuda")
            self.weight = self.master.to(torch.bfloat16)
            self.dW, self.dgain = torch.zeros(N, K, device="cuda"), torch.zeros(K, device="cuda")
            self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
            ps = [self.master, self.gain]
            self.m, self.v = ([torch.zeros(p.numel(), dtype=torch.uint8, device="cuda") for p in ps] for _ in range(2))
            self.ms, self.vs = ([torch.zeros(-(-p.numel() // 128), device="cuda") for p in ps] for _ in range(2))
            self.t = api.make_adamw_tensors(ps, [self.dW, self.dgain], self.m, self.v, m_scales=self.ms, v_scales=self.vs, copies=[self.weight, None])
            self.o = {k: t for k, t in api.snip_rmsnorm_fwd(x, self.gain, 1e-5, residual=residual, fmt=F8, fmt_t=F8).items() if t is not None}
            self.bufs = api.snip_quantize_dual(self.weight, api.DUAL_BLK_BLKT, F8, F8, want_stats=False)
            self.dbufs = api.snip_quantize_dual(dy, api.DUAL_ROW_COLT, F8, F8, want_stats=False)
            self.y, self.dX, self.dx = torch.empty(M, N, device="cuda"), torch.empty(M, K, dtype=torch.bfloat16, device="cuda"), torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
            size = max(api.snip_workspace_size(op, M, N, K, F8, F8)[0] for op in (0, 1, 2))
            self.ws, self.nws = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(api.snip_rmsnorm_bwd_workspace(M, K), dtype=torch.uint8, device="cuda")

        def run(self):
            q = api.make_qtensor
            o = api.snip_rmsnorm_fwd(x, self.gain, 1e-5, residual=residual, fmt=F8, fmt_t=F8, out=self.o)
            wq, wqt = api.snip_quantize_dual(self.weight, api.DUAL_BLK_BLKT, F8, F8, want_stats=False, bufs=self.bufs)
            dq, dqt = api.snip_quantize_dual(dy, api.DUAL_ROW_COLT, F8, F8, want_stats=False, bufs=self.dbufs)
            api.snip_gemm_quantized(api.OP_FWD, q(o["codes"], o["scales"], M, K, F8, 0), q(wq["codes"], wq["scales"], N, K, F8, 2), (M, N), 1, out=self.y, ws=self.ws)
            api.snip_gemm_quantized(api.OP_DGRAD, q(dq["codes"], dq["scales"], M, N, F8, 0), q(wqt["codes"], wqt["scales"], N, K, F8, 2, True), (M, K), out=self.dX, ws=self.ws)
            api.snip_gemm_quantized(api.OP_WGRAD, q(dqt["codes"], dqt["scales"], M, N, F8, 1, True), q(o["codes_t"], o["scales_t"], M, K, F8, 1, True), (N, K), 1, out=self.dW, ws=self.ws)
            api.snip_rmsnorm_bwd(self.dX, o["h"], self.gain, o["rstd"], dx=self.dx, dgain=self.dgain, ws=self.nws)
            self.step.add_(1)
            api.snip_adamw_step(self.t, 1e-3, 0.9, 0.95, 1e-8, self.step, rounding=api.ROUND_STOCHASTIC, seed=3)

        def tensors(self):
            return [self.master, self.gain, self.weight, self.dW, self.dgain, self.y, self.dx] + self.m + self.v + self.ms + self.vs + list(self.o.values())

    warm, eager, replayed = State(), State(), State()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed.run()
    for _ in range(4):
        eager.run()
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager.tensors(), replayed.tensors()):
        assert torch.equal(a, b)
    assert not torch.equal(eager.master, warm.master)
