"""AdamW over many tensors and the global gradient norm: HIP path vs the oracle.

32-bit moments, codes and scales are bit-exact (their arithmetic is part of the format).  Weights: the update is a quotient of
fp32 values with a relative error below 2^-20, and the sum is rounded to fp32 (2^-24 of the result), then to bf16 (2^-8).
"""
import numpy as np
import pytest
import torch

from oracle import slope_oracle as so
from oracle import surroundings_oracle as oo
from paper_2405_16325_amd import binding as sl
from paper_2405_16325_amd import inputs

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS = 1e-2, 0.9, 0.95, 1e-8
# a chunk is 4096 elements, a block 128, a lane's piece 8
SIZES = [1, 7, 8, 9, 127, 128, 129, 1000, 2048, 4095, 4096, 4097, 50257]


def say(msg):
    print(msg, flush=True)


def bf16_bits(x):
    return inputs.f32_to_bf16_bits(np.asarray(x, np.float32))


class Set:
    """Tensors of a step on host and device."""

    def __init__(self, sizes, bits, master, grad_bits, param=True, seed=0, decay=None):
        g = np.random.default_rng(seed)
        self.sizes, self.bits, self.master, self.grad_bits = sizes, bits, master, grad_bits
        self.decay = decay if decay is not None else [0.1 if i % 2 == 0 else 0.0 for i in range(len(sizes))]
        self.p = [(0.1 * g.standard_normal(n)).astype(np.float32) for n in sizes]
        if not master:
            self.p = [inputs.bf16_bits_to_f32(bf16_bits(p)) for p in self.p]
        self.m = [(1e-3 * g.standard_normal(n)).astype(np.float32) for n in sizes]
        self.v = [((1e-3 * g.standard_normal(n)) ** 2).astype(np.float32) for n in sizes]
        if bits == 8:
            self.mq = [oo.store_states(m, 5, False) for m in self.m]
            self.rq = [oo.store_states(np.sqrt(v), 5, True) for v in self.v]
        self.new_grads(g)
        dev = lambda x: torch.from_numpy(np.array(x)).cuda()                                       # noqa: E731
        self.params = [sl.bf16_to_device(bf16_bits(p)) for p in self.p] if param else None
        self.masters = [dev(p) for p in self.p] if master else None
        if bits == 8:
            self.dm, self.dv = ([dev(c).view(sl.E4M3) for c, _ in q] for q in (self.mq, self.rq))
            self.dms, self.dvs = ([dev(s) for _, s in q] for q in (self.mq, self.rq))
        else:
            self.dm, self.dv, self.dms, self.dvs = [dev(m) for m in self.m], [dev(v) for v in self.v], None, None
        self.grads = [dev(x) if grad_bits == 32 else sl.bf16_to_device(bf16_bits(x)) for x in self.g]
        self.plan = sl.slope_adamw_plan(self.params, self.grads, self.dm, self.dv, masters=self.masters, m_scales=self.dms,
                                        v_scales=self.dvs, weight_decay=self.decay)

    def new_grads(self, g):
        self.g = [(1e-3 * g.standard_normal(n)).astype(np.float32) for n in self.sizes]
        if self.grad_bits == 16:
            self.g = [inputs.bf16_bits_to_f32(bf16_bits(x)) for x in self.g]

    def check(self, coef, step):
        for i, n in enumerate(self.sizes):
            m, v = self.m[i], self.v[i]
            if self.bits == 8:
                m, r = oo.load_states(*self.mq[i]), oo.load_states(*self.rq[i])
                v = r * r
            p, m2, v2 = oo.adamw(self.p[i], self.g[i], m, v, coef, LR, B1, B2, EPS, self.decay[i], step)
            what = (i, n)
            if self.bits == 8:
                for x, root, codes, scales in ((m2, False, self.dm[i], self.dms[i]), (np.sqrt(v2), True, self.dv[i], self.dvs[i])):
                    want, scale = oo.store_states(x, step, root)
                    assert (scales.cpu().numpy() == scale).all(), what
                    got = codes.view(torch.uint8).cpu().numpy()
                    assert (oo.e4m3_value(got) == oo.e4m3_value(want)).all(), what
            else:
                assert (self.dm[i].cpu().numpy() == m2).all() and (self.dv[i].cpu().numpy() == v2).all(), what
            bound = 2.0 ** -23 * np.abs(self.p[i]) + 2.0 ** -19 * np.abs(p - self.p[i]) + 2.0 ** -23 * np.abs(p) + 1e-30
            if self.masters is not None:
                assert (np.abs(self.masters[i].cpu().numpy() - p) <= bound).all(), what
            if self.params is not None:
                got = so.bf16_to_f64(sl.bf16_to_host(self.params[i]))
                assert (np.abs(got - p) <= bound + 2.0 ** -8 * 1.01 * np.abs(p)).all(), what


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master,param,grad_bits", [(True, True, 16), (True, True, 32), (True, False, 32), (False, True, 16), (False, True, 32)])
def test_step(bits, master, param, grad_bits):
    say(f"adamw bits={bits} master={master} param={param} grad={grad_bits}")
    s = Set(SIZES, bits, master, grad_bits, param, seed=bits + grad_bits)
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, step=7, grad_scale=0.5)
    torch.cuda.synchronize()
    s.check(0.5, 7)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[1], [128], [0, 5, 0], [300000], [8] * 500, [4096 * 3 + 1, 2]])
def test_sets_of_tensors(bits, sizes):
    say(f"adamw bits={bits} sizes={sizes[:4]} x{len(sizes)}")
    s = Set(sizes, bits, True, 16, seed=3)
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, step=1)
    torch.cuda.synchronize()
    s.check(1.0, 1)


def test_a_set_of_empty_tensors():
    s = Set([0, 0], 32, True, 16)
    control = torch.zeros(4, device="cuda")
    sl.slope_grad_norm(s.plan, control)
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, control=control)
    assert control.tolist() == [0.0, 1.0, 1.0, 0.0]


@pytest.mark.parametrize("bits", [32, 8])
def test_extreme_states(bits):
    """Blocks of zeros; a gradient of zero on zero states; values at both ends of fp32."""
    s = Set([256, 384], bits, True, 32, seed=4)
    for t in s.grads:
        t.zero_()
    s.g = [np.zeros_like(x) for x in s.g]
    for t in s.dm + s.dv:
        t.view(torch.uint8).zero_()
    s.m, s.v = [np.zeros_like(x) for x in s.m], [np.zeros_like(x) for x in s.v]
    for q in ("mq", "rq"):
        if bits == 8:
            setattr(s, q, [(np.zeros_like(c), sc) for c, sc in getattr(s, q)])
    big = np.float32(1e15)
    s.g[1][:] = np.float32(1e-25)
    s.g[1][130] = big
    s.grads[1].copy_(torch.from_numpy(s.g[1]))
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, step=3)
    torch.cuda.synchronize()
    s.check(1.0, 3)
    if bits == 8:
        assert (s.dms[0] == 0).all() and (s.dm[0].view(torch.uint8) & 0x7F == 0).all()


@pytest.mark.parametrize("max_norm", [1e9, 0.01, float("inf")])
@pytest.mark.parametrize("grad_bits", [16, 32])
def test_norm_clip_and_step_from_the_device(max_norm, grad_bits):
    say(f"grad_norm max={max_norm} grad={grad_bits}")
    s = Set(SIZES, 32, True, grad_bits, seed=6)
    control = torch.zeros(4, device="cuda")
    for step in (1, 2):
        sl.slope_grad_norm(s.plan, control, 0.25, max_norm)
        norm, coef = oo.grad_norm(s.g, 0.25, max_norm)
        got = control.tolist()
        assert abs(got[0] - norm) <= 2.0 ** -18 * norm and abs(got[1] - coef) <= 2.0 ** -17 * coef and got[2] == step
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, control=control)
    torch.cuda.synchronize()
    s.check(np.float32(got[1]), 2)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_step_that_is_not_finite_is_left_out(bits, bad):
    say(f"adamw bits={bits} gradient {bad}")
    s = Set([5000, 129], bits, True, 16, seed=8)
    s.grads[1][128] = bad
    tensors = s.params + s.masters + s.dm + s.dv + (s.dms + s.dvs if bits == 8 else [])
    before = [t.view(torch.uint8).clone() for t in tensors]
    control = torch.tensor([0.0, 0.0, 4.0, 0.0], device="cuda")
    sl.slope_grad_norm(s.plan, control, 1.0, 1.0)
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, control=control)
    torch.cuda.synchronize()
    got = control.tolist()
    assert not np.isfinite(got[0]) and got[1] == 0.0 and got[2] == 4.0
    assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(before, tensors))
    # and the next one is taken
    s.grads[1][128] = 0.0
    s.g[1][128] = 0.0
    sl.slope_grad_norm(s.plan, control, 1.0, float("inf"))
    sl.slope_adamw_step(s.plan, LR, B1, B2, EPS, control=control)
    torch.cuda.synchronize()
    assert control[2] == 5.0
    s.check(1.0, 5)


def test_nothing_between_tensors_is_written():
    sizes = [129, 7, 1000]
    for bits in (32, 8):
        state = torch.uint8 if bits == 8 else torch.float32
        pool = {k: torch.full((8192,), 85, dtype=d, device="cuda") for k, d in
                (("p", sl.BF16), ("w", torch.float32), ("m", state), ("v", state), ("ms", torch.float32), ("vs", torch.float32))}
        at = [256, 1024, 4096]
        cut = lambda k: [pool[k][a:a + n] for a, n in zip(at, sizes)]                                  # noqa: E731
        states = lambda k: [t.view(sl.E4M3) for t in cut(k)] if bits == 8 else cut(k)                  # noqa: E731
        scales = lambda k: [pool[k][a // 128:a // 128 + (n + 127) // 128] for a, n in zip(at, sizes)] if bits == 8 else None  # noqa: E731
        plan = sl.slope_adamw_plan(cut("p"), [torch.ones(n, device="cuda") for n in sizes], states("m"), states("v"), masters=cut("w"),
                                   m_scales=scales("ms"), v_scales=scales("vs"))
        sl.slope_adamw_step(plan, LR, B1, B2, EPS, step=1)
        torch.cuda.synchronize()
        for k, t in pool.items():
            inside = torch.zeros(8192, dtype=torch.bool, device="cuda")
            for a, n in zip(at, sizes):
                inside[slice(a, a + n) if k not in ("ms", "vs") else slice(a // 128, a // 128 + (n + 127) // 128)] = True
            assert (t[~inside] == 85).all(), (bits, k)


def test_another_stream_and_graph_replays():
    """Graph replays take the step's number and the clipping factor from the device: they equal eager steps one by one."""
    sets = [Set(SIZES, 8, True, 16, seed=9) for _ in range(2)]
    controls = [torch.zeros(4, device="cuda") for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())

    def step(i):
        sl.slope_grad_norm(sets[i].plan, controls[i], 1.0, 0.05)
        sl.slope_adamw_step(sets[i].plan, LR, B1, B2, EPS, control=controls[i])

    with torch.cuda.stream(stream):
        step(0)
        step(1)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for turn in range(4):
        for a, b in zip(sets[0].grads, sets[1].grads):
            a.copy_(torch.randn(a.shape, device="cuda") * 1e-3)
            b.copy_(a)
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(controls[0], controls[1]) and controls[0][2] == 2 + turn
        for k in ("masters", "params", "dm", "dv", "dms", "dvs"):
            for a, b in zip(getattr(sets[0], k), getattr(sets[1], k)):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (turn, k)


def test_many_steps_reach_a_minimum_with_either_kind_of_state():
    """A quadratic bowl of badly scaled directions: 8-bit states end as near the minimum as 32-bit ones do, up to a factor two."""
    n, ends = 4096, {}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    curve = 10.0 ** (torch.rand(n, generator=gen, device="cuda") * 4 - 2)
    for bits in (32, 8):
        w = torch.ones(n, device="cuda")
        g = torch.zeros(n, device="cuda")
        if bits == 8:
            m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(sl.E4M3) for _ in range(2))
            scales = [torch.zeros(n // 128, device="cuda") for _ in range(2)]
            plan = sl.slope_adamw_plan(None, [g], [m], [v], masters=[w], m_scales=[scales[0]], v_scales=[scales[1]])
        else:
            plan = sl.slope_adamw_plan(None, [g], [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")], masters=[w])
        for t in range(1, 1001):
            g.copy_(curve * w)
            sl.slope_adamw_step(plan, 1e-2 * (1 - t / 1001), B1, 0.99, EPS, step=t)
        ends[bits] = float((0.5 * curve * w * w).sum())
    assert ends[32] < 1e-2 and ends[8] < max(2 * ends[32], 1e-2), ends


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [2.0 ** -126, 2.0 ** 125])
def test_elements_without_a_gradient_at_the_ends_of_eps(bits, eps):
    """Zero gradients on zero states: 0 / eps leaves the weights to their decay, p (1 - lr wd) rounded to fp32 and then to bf16."""
    say(f"adamw bits={bits} eps={eps}")
    s = Set([300, 4097], bits, True, 32, seed=12)
    for t in s.grads + s.dm + s.dv:
        t.view(torch.uint8).zero_()
    sl.slope_adamw_step(s.plan, LR, B1, B2, eps, step=1)
    torch.cuda.synchronize()
    for p, decay, master, param in zip(s.p, s.decay, s.masters, s.params):
        want = p.astype(np.float64) * (1.0 - LR * decay)
        assert (np.abs(master.cpu().numpy() - want) <= 2.0 ** -22 * np.abs(want)).all()
        assert (np.abs(so.bf16_to_f64(sl.bf16_to_host(param)) - want) <= 2.0 ** -8 * 1.01 * np.abs(want)).all()
    assert all((t.view(torch.uint8) & (0x7F if bits == 8 else 0xFF) == 0).all() for t in s.dm + s.dv)
