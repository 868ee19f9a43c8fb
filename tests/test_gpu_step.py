"""The operators of a token's step together, as a program strings them up: residual and norm into 8 bits, gate and up, down with the
residual, norm again, logits from 4-bit weights, the next token.  Every stage is checked on what the stage before left, eagerly and
captured into a graph that is replayed with other inputs while eager work goes on."""
import numpy as np
import pytest

from test_gpu_add_norm import check as check_norm, check_8_bits, reference as norm_reference
from test_gpu_sample import reference as sample_reference
from test_gpu_w4 import dense

pytestmark = pytest.mark.gpu

D, F, V, G = 512, 1408, 5003, 64


@pytest.fixture(scope="module")
def cas():
    import torch
    assert torch.cuda.is_available()
    import paper_2507_05228_amd as cas
    cas.load_library()
    return cas


class Step:
    def __init__(self, cas, rows, dtype, fmt, seed=0):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.cas, self.rows, self.dtype, self.fmt, self.g = cas, rows, dtype, fmt, g

        def weights(n, k, spread):
            codes = torch.randint(0, 16, (n, k), device="cuda", generator=g, dtype=torch.uint8)
            scales = (spread * (0.5 + torch.rand((n, k // G), device="cuda", generator=g)) / (4.6 * k ** 0.5)).to(dtype)
            zeros = torch.randint(6, 11, (n, k // G), device="cuda", generator=g, dtype=torch.uint8)
            return (codes, scales, zeros), cas.make_w4_weights(codes, scales, zeros)

        self.mats = {n: weights(*s) for n, s in (("gate", (F, D, 1.0)), ("up", (F, D, 1.0)), ("down", (D, F, 1.0)), ("head", (V, D, 3.0)))}
        new = lambda *s, dt=dtype: torch.empty(s, device="cuda", dtype=dt)  # noqa: E731
        self.gain = [(1 + 0.1 * torch.randn(D, device="cuda", generator=g)).to(dtype) for _ in range(2)]
        self.h, self.delta, self.h1, self.mid, self.logits = new(rows, D), new(rows, D), new(rows, D), new(rows, F), new(rows, V)
        self.q, self.s, self.q2, self.s2 = new(rows, D, dt=fmt), new(rows, D // G, dt=torch.float32), new(rows, D, dt=fmt), new(rows, dt=torch.float32)
        self.u, self.token, self.prob = new(rows, dt=torch.float32), new(rows, dt=torch.int32), new(rows, dt=torch.float32)
        self.t, self.k, self.p = (torch.full((rows,), v, device="cuda") for v in (0.8, 40, 0.9))
        self.k = self.k.int()
        self.ws = cas.new_workspace(max([cas.cascade_sample_workspace_bytes(rows, V, dtype), cas.cascade_w4_gemm_workspace_bytes(self.w("gate"), self.q, self.w("up")),
                                         cas.cascade_w4_gemm_workspace_bytes(self.w("down"), self.mid), cas.cascade_w4_gemm_workspace_bytes(self.w("head"), self.q2)]))
        self.fill()

    def w(self, name):
        return self.mats[name][1]

    def fill(self):
        import torch
        self.h.copy_(torch.randn(self.h.shape, device="cuda", generator=self.g))
        self.delta.copy_(torch.randn(self.h.shape, device="cuda", generator=self.g))
        self.u.copy_(torch.rand(self.rows, device="cuda", generator=self.g))

    def run(self):
        cas = self.cas
        cas.cascade_add_norm(self.h, self.gain[0], cas.NORM_RMSNORM, 1e-5, delta=self.delta, sum=self.h1, q=self.q, q_scale=self.s)
        cas.cascade_w4_gemm(self.w("gate"), self.q, self.mid, x_scale=self.s, weights_up=self.w("up"), epilogue=cas.EPI_SWIGLU, workspace=self.ws)
        cas.cascade_w4_gemm(self.w("down"), self.mid, self.h1, residual=self.h1, epilogue=cas.EPI_RESIDUAL, workspace=self.ws)
        cas.cascade_add_norm(self.h1, self.gain[1], cas.NORM_RMSNORM, 1e-5, q=self.q2, q_scale=self.s2)
        cas.cascade_w4_gemm(self.w("head"), self.q2, self.logits, x_scale=self.s2, workspace=self.ws)
        cas.cascade_sample(self.logits, self.u, self.token, temperature=self.t, top_k=self.k, top_p=self.p, prob=self.prob, workspace=self.ws)

    def check(self):
        import torch
        half = torch.finfo(self.dtype).eps / 2
        s, y, slack = norm_reference(self.h, self.delta, self.gain[0], None, False, 1e-5)
        most = 127 if self.fmt == torch.int8 else 448
        check_8_bits(self.q, self.s, y, slack, most, D)
        x = (self.q.double().view(self.rows, -1, G) * self.s.double()[..., None]).view(self.rows, D)
        gate, up, down, head = ((self.mats[n][0], dense(*self.mats[n][0], G)) for n in ("gate", "up", "down", "head"))

        def slack_of(x, m):                                # as derived beside the products' own tests
            return 62 * 2.0 ** -15 * (x.abs() @ m[0][1].double().repeat_interleave(G, 1).t())

        a, b = x @ gate[1].t(), x @ up[1].t()
        silu = a * torch.sigmoid(a)
        sa, sb = slack_of(x, gate), slack_of(x, up)
        check_norm("gate and up", self.mid, silu * b, 1.1 * sa * (b.abs() + sb) + silu.abs() * sb + 2.0 ** -12 * (silu * b).abs(), half)
        h1 = s.to(self.dtype).double() + self.mid.double() @ down[1].t()      # (the sum as it was rounded: half a step at the most apart)
        check_norm("down", self.h1, h1, slack_of(self.mid.double(), down) + half * s.abs() + 2.0 ** -22 * h1.abs(), half)
        _, y, slack = norm_reference(self.h1, None, self.gain[1], None, False, 1e-5)
        check_8_bits(self.q2, self.s2, y, slack, most, D)
        x = self.q2.double() * self.s2.double()[:, None]
        check_norm("logits", self.logits, x @ head[1].t(), slack_of(x, head), half)
        l, u = self.logits.float().cpu().numpy(), self.u.cpu().numpy()
        for r in range(self.rows):
            token, prob = sample_reference(l[r], u[r], np.float32(0.8), 40, np.float32(0.9), 0.0)
            assert int(self.token[r]) == token and abs(float(self.prob[r]) - prob) <= 2.0 ** -22 * prob


@pytest.mark.parametrize("rows", [1, 6, 40])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("fmt", ["int8", "float8_e4m3fn"])
def test_a_step(cas, rows, dtype, fmt):
    import torch
    step = Step(cas, rows, getattr(torch, dtype), getattr(torch, fmt))
    step.run()
    torch.cuda.synchronize()
    step.check()


@pytest.mark.parametrize("rows", [3, 33])
def test_a_captured_step_is_replayed(cas, rows):
    import torch
    step, eager = Step(cas, rows, torch.bfloat16, torch.int8, seed=1), Step(cas, rows, torch.bfloat16, torch.int8, seed=1)
    other = Step(cas, rows, torch.bfloat16, torch.int8, seed=2)
    other.ws = step.ws                                     # graphs that run one after the other may share a workspace
    graphs = []
    for one in (step, other):
        one.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            one.run()
        graphs.append(graph)
    for _ in range(4):
        for one in (step, other):
            one.fill()
        for name in ("h", "delta", "u"):
            getattr(eager, name).copy_(getattr(step, name))
        step.ws.fill_(0x5a)
        graphs[0].replay()
        graphs[1].replay()
        eager.run()
        torch.cuda.synchronize()
        step.check()
        other.check()
        for name in ("h1", "q", "s", "mid", "q2", "s2", "logits", "token", "prob"):
            assert torch.equal(getattr(step, name).view(torch.uint8) if name in ("q", "q2") else getattr(step, name),
                               getattr(eager, name).view(torch.uint8) if name in ("q", "q2") else getattr(eager, name)), name


def test_two_streams_at_once(cas):
    import torch
    steps, streams = [Step(cas, 8, torch.bfloat16, torch.float8_e4m3fn, seed=s) for s in (3, 4)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for step, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                step.run()
    torch.cuda.synchronize()
    for step in steps:
        step.check()
