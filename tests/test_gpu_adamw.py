"""AdamW steps over many tensors on the GPU, through the C ABI, against oracle/adamw.py.

Tolerances, derived from the arithmetic (u = 2^-24):
* m and v in 32 bits: three roundings each of terms that may cancel: 4 u (beta1 |m| + |g|), 4 u v;
* the step: m, 1 / (1 - beta^t) (the exponential's argument is rounded: up to 4 u |t log beta| more, far
  below what beta^t then is), the root and the division within 16 u of it, so |dp| <= lr (32 u |update| + 4 u (beta1
  |m| + |g|) / (c1 denominator)) + 3 u |p|; a bf16 parameter adds 2^-8 |p|;
* codes of 8-bit states: exact, given m and v with each operation rounded to float32 in the formulas' order.
"""

import numpy as np
import pytest

from oracle import adamw as A

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _dev(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _host(t):
    return t.float().cpu().numpy()


def _flat(values, dtype, skew=0):
    """A tensor on the device, `skew` elements past an aligned place, and its surroundings."""
    import torch

    t = torch.float32 if dtype == "f32" else torch.bfloat16
    whole = torch.full((len(values) + skew + 9,), 768.0, dtype=t, device="cuda")
    part = whole[skew:skew + len(values)]
    part.copy_(_dev(np.asarray(values, np.float32)).to(t))
    return part, whole


def _bytes(n, skew=0, fill=0xAB):
    import torch

    whole = torch.full((n + skew + 9,), fill, dtype=torch.uint8, device="cuda")
    return whole[skew:skew + n], whole


class One:
    def __init__(self, rng, n, bits, param="bf16", master=True, grad="bf16", decay=0.1, skew=0, size=None, zeros=False):
        size = np.exp2(rng.integers(-20, 3, max(n, 1)))[:n] if size is None else size
        self.n, self.bits, self.decay, self.param_type, self.grad_type = n, bits, decay, param, grad
        g = rng.standard_normal(n) * size
        m, v = rng.standard_normal(n) * size * 0.3, (rng.standard_normal(n) * size) ** 2
        if zeros:
            g, m, v = 0 * g, 0 * m, 0 * v
        p = (rng.standard_normal(n) * 0.05).astype(np.float32)
        self.parts = {}
        self.param, self.parts["param"] = _flat(p, param, skew)
        self.grad, self.parts["grad"] = _flat(g, grad, skew)
        self.master = None
        if master:
            self.master, self.parts["master"] = _flat(p, "f32", skew)
        if bits == 32:
            self.m, self.parts["m"] = _flat(m, "f32", skew)
            self.v, self.parts["v"] = _flat(v, "f32", skew)
            self.ms = self.vs = None
            self.m0, self.v0 = _host(self.m), _host(self.v)
        else:
            none = [0] * n
            mc, ms, vc, vs = A.codes(m.astype(np.float32), np.sqrt(v).astype(np.float32), none)
            self.m, self.parts["m"] = _bytes(n, skew)
            self.v, self.parts["v"] = _bytes(n, skew)
            self.ms, self.parts["ms"] = _bytes(len(ms), skew)
            self.vs, self.parts["vs"] = _bytes(len(vs), skew)
            for t, a in ((self.m, mc), (self.v, vc), (self.ms, ms), (self.vs, vs)):
                t.copy_(_dev(a))
            self.m0 = A.values_m(mc, ms).astype(np.float32)
            root = A.values_root(vc, vs).astype(np.float32)
            self.v0 = root * root
        self.p0 = _host(self.master if master else self.param)
        self.g0 = _host(self.grad)
        self.around = {k: w.clone() for k, w in self.parts.items()}

    def entry(self):
        from paper_2609_00993_amd import moepd as M

        code = {"f32": M.MOE_DTYPE_F32, "bf16": M.MOE_DTYPE_BF16}
        return M.adamw_tensor(self.param, code[self.param_type], self.master, self.grad, code[self.grad_type], self.m, self.v,
                              self.ms, self.vs, self.n, self.decay)

    def check(self, number, lr, t, b1, b2, eps, scale, seed):
        p, m, v = A.step(self.p0, self.g0, self.m0, self.v0, lr, t, b1, b2, eps, self.decay, scale)
        g = np.abs(self.g0.astype(np.float64) * scale)
        c1, c2 = 1 - b1 ** t, 1 - b2 ** t
        em = 4 * U * (b1 * np.abs(self.m0) + g)
        den = np.sqrt(v / c2) + eps
        with np.errstate(divide="ignore", invalid="ignore"):
            update = np.where(den > 0, np.abs(m) / c1 / den, 0.0)
            slack = np.where(den > 0, em / c1 / den, 0.0)
        tol = lr * (32 * U * update + slack + 4 * U * np.abs(self.decay * self.p0)) + 3 * U * np.abs(p) + 1e-37
        got = _host(self.master if self.master is not None else self.param)
        rounding = 0.0 if self.master is not None or self.param_type == "f32" else 2.0 ** -8
        assert (np.abs(got - p) <= tol + rounding * np.abs(p)).all()
        if self.master is not None and self.n:
            assert (self.param == self.master.to(self.param.dtype)).all()
        if self.bits == 32:
            assert (np.abs(_host(self.m) - m) <= em + 1e-37).all()
            assert (np.abs(_host(self.v) - v) <= 4 * U * v + 1e-37).all()
        else:
            m32, v32 = A.states32(self.g0, self.m0, self.v0, b1, b2, scale)
            mc, ms, vc, vs = A.codes(m32, np.sqrt(v32), A.words(seed, t, number, self.n))
            assert (_host(self.ms) == ms).all() and (_host(self.vs) == vs).all()
            assert (_host(self.m) == mc).all()
            assert (_host(self.v) == vc).all()
        for k, w in self.parts.items():  # nothing beside the tensors
            part = getattr(self, k)
            lo = (part.data_ptr() - w.data_ptr()) // w.element_size()
            assert (w[:lo] == self.around[k][:lo]).all() and (w[lo + part.numel():] == self.around[k][lo + part.numel():]).all(), k
        assert (self.parts["grad"] == self.around["grad"]).all()


def _step(tensors, bits, lr=1e-3, t=7, b1=0.9, b2=0.99, eps=1e-8, scale=None, seed=12345, stream=None):
    import torch

    from paper_2609_00993_amd import moepd as M

    s = stream or torch.cuda.Stream()
    st, h = M.moe_adamw_create([x.entry() for x in tensors], bits)
    M.check(st)
    d = [torch.tensor([lr], device="cuda"), torch.tensor([t], dtype=torch.int32, device="cuda"),
         None if scale is None else torch.tensor([scale], device="cuda")]
    torch.cuda.synchronize()
    M.check(M.moe_adamw_step(h, b1, b2, eps, *d, seed, s))
    torch.cuda.synchronize()
    M.check(M.moe_adamw_destroy(h))
    return dict(lr=float(np.float32(lr)), t=t, b1=b1, b2=b2, eps=eps, scale=1.0 if scale is None else scale, seed=seed)


SIZES = [1, 7, 31, 32, 33, 255, 2047, 2048, 2049, 0, 5000]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,master,grad", [("bf16", True, "bf16"), ("bf16", False, "f32"), ("f32", False, "f32"),
                                               ("f32", True, "bf16"), ("f32", False, "bf16")])
def test_many_tensors(bits, param, master, grad):
    rng = np.random.default_rng(bits)
    ts = [One(rng, n, bits, param, master, grad, decay=0.1 * (i % 2)) for i, n in enumerate(SIZES)]
    how = _step(ts, bits, scale=0.5)
    for i, x in enumerate(ts):
        x.check(i, **how)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("skew", [1, 3, 5])
def test_any_alignment(bits, skew):
    rng = np.random.default_rng(skew)
    ts = [One(rng, n, bits, skew=skew) for n in (1, 40, 2055)]
    how = _step(ts, bits)
    for i, x in enumerate(ts):
        x.check(i, **how)


@pytest.mark.parametrize("t,b1,b2", [(1, 0.9, 0.999), (2, 0.0, 0.0), (100000, 0.9, 0.999), (3, 0.95, 0.9999)])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps_and_betas(bits, t, b1, b2):
    x = One(np.random.default_rng(t), 300, bits)
    x.check(0, **_step([x], bits, t=t, b1=b1, b2=b2))


@pytest.mark.parametrize("bits", [32, 8])
def test_zeros_and_small(bits):
    rng = np.random.default_rng(8)
    ts = [One(rng, 100, bits, zeros=True), One(rng, 100, bits, size=1e-17), One(rng, 64, bits, size=np.exp2(-np.arange(64.0)))]
    how = _step(ts, bits)
    for i, x in enumerate(ts):
        x.check(i, **how)


def test_smallest_scales():
    """m near and below the smallest normal float32: scale byte 0, and codes in steps of 2^-136."""
    rng = np.random.default_rng(9)
    ts = [One(rng, 64, 8, grad="f32", size=s) for s in (1e-36, 1e-37, 1e-38, 3e-39)]
    how = _step(ts, 8)
    for i, x in enumerate(ts):
        x.check(i, **how)
    assert (ts[2].ms == 0).all() and (ts[2].m != 0).any()


def test_states_that_are_not_finite():
    """A NaN or an infinity makes its block's codes NaN, and no other's."""
    import torch

    x = One(np.random.default_rng(1), 128, 8, grad="f32")
    x.grad[40] = float("nan")
    x.grad[70] = float("inf")
    x.g0 = _host(x.grad)
    _step([x], 8)
    assert x.ms.tolist()[1:3] == [255, 255] and x.vs.tolist()[1:3] == [255, 255]
    assert 255 not in (x.ms.tolist()[0], x.ms.tolist()[3], x.vs.tolist()[0], x.vs.tolist()[3])
    assert (x.m[32:96] == 0).all()
    bad = ~torch.isfinite(x.master)
    assert bad.sum() == 2 and bad[40] and bad[70]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), -float("inf")])
def test_scale_that_is_not_finite_changes_nothing(bits, scale):
    x = One(np.random.default_rng(2), 500, bits)
    _step([x], bits, scale=scale)
    for k, w in x.parts.items():
        assert (w == x.around[k]).all(), k


@pytest.mark.parametrize("bits", [32, 8])
def test_long_table(bits):
    """Chunks of several passes, and more tensors than workgroups run at a time."""
    import torch

    from paper_2609_00993_amd import moepd as M

    rng = np.random.default_rng(3)
    small = [One(rng, n, bits) for n in (3000, 1)]
    n = 17_000 * 2048 + 11
    big = {k: torch.zeros(n, dtype=t, device="cuda") for k, t in (
        ("param", torch.bfloat16), ("master", torch.float32), ("grad", torch.bfloat16),
        ("m", torch.float32 if bits == 32 else torch.uint8), ("v", torch.float32 if bits == 32 else torch.uint8))}
    scales = [None, None] if bits == 32 else [torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    big["grad"].fill_(1.0)
    entry = M.adamw_tensor(big["param"], M.MOE_DTYPE_BF16, big["master"], big["grad"], M.MOE_DTYPE_BF16, big["m"], big["v"],
                           *scales, n, 0.0)
    st, h = M.moe_adamw_create([small[0].entry(), entry, small[1].entry()], bits)
    M.check(st)
    s = torch.cuda.Stream()
    lr, t = torch.tensor([0.5], device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    M.check(M.moe_adamw_step(h, 0.9, 0.99, 1e-8, lr, t, None, 5, s))
    torch.cuda.synchronize()
    # m / c1 = 1 and sqrt(v / c2) = 1 everywhere
    assert ((big["master"] + 0.5).abs() <= 0.5 * 64 * U).all() and (big["param"] == big["master"].to(torch.bfloat16)).all()
    m = torch.empty(n, device="cuda")
    r = torch.empty(n, device="cuda")
    M.check(M.moe_adamw_read(h, 1, m, r, M.MOE_DTYPE_F32, s))
    torch.cuda.synchronize()
    step = 8 * U if bits == 32 else 1 / 8
    assert ((m - 0.1).abs() <= 0.1 * step).all() and ((r - 0.1).abs() <= 0.1 * step).all()
    how = dict(lr=0.5, t=1, b1=0.9, b2=0.99, eps=1e-8, scale=1.0, seed=5)
    small[0].check(0, **how)
    small[1].check(2, **how)
    M.check(M.moe_adamw_destroy(h))


def test_rounding_is_fair():
    """Over many elements and steps the codes' mean is the value, though no code is; v that decays by a part of a
    code's step goes down."""
    import torch

    from paper_2609_00993_amd import moepd as M

    n = 1 << 16
    z = lambda t: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
    master, grad = z(torch.float32), z(torch.float32)
    grad.fill_(1.0)
    m, v = z(torch.uint8), z(torch.uint8)
    ms, vs = (torch.zeros(n // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    st, h = M.moe_adamw_create([M.adamw_tensor(master, M.MOE_DTYPE_F32, None, grad, M.MOE_DTYPE_F32, m, v, ms, vs, n)], 8)
    M.check(st)
    s = torch.cuda.Stream()
    lr, t = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = [torch.empty(n, device="cuda") for _ in range(2)]
    steps = 40
    want_m = want_v = 0.0
    for i in range(steps):
        if i == 20:
            grad.fill_(0.0)
        t.fill_(i + 1)
        torch.cuda.synchronize()
        M.check(M.moe_adamw_step(h, 0.9, 0.99, 1e-8, lr, t, None, 77, s))
        torch.cuda.synchronize()
        g = float(i < 20)
        want_m, want_v = 0.9 * want_m + 0.1 * g, 0.99 * want_v + 0.01 * g
    M.check(M.moe_adamw_read(h, 0, *out, M.MOE_DTYPE_F32, s))
    torch.cuda.synchronize()
    # each step adds at most an eighth of the value, evenly spread: (1/8)^2 / 12 each, summed over the steps that are kept
    # (m: sum 0.81^i < 5.3; v's root: at most all 40), over n elements: six deviations of the mean
    dev = 1 / 8 / 12 ** 0.5
    assert abs(out[0].mean().item() / want_m - 1) < 6 * dev * 5.3 ** 0.5 / n ** 0.5
    # the mean of v is that of the root squared plus its variance: the root is unbiased step by step, so v grows by at most
    # (1/8)^2 / 12 of itself a step
    v_mean = out[1].double().square().mean().item()
    grow = (1 + dev ** 2) ** steps
    noise = 6 * 2 * dev * steps ** 0.5 / n ** 0.5
    assert want_v * (1 - noise) <= v_mean <= want_v * grow * (1 + noise)
    M.check(M.moe_adamw_destroy(h))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_read(bits, dtype):
    import torch

    from paper_2609_00993_amd import moepd as M

    rng = np.random.default_rng(4)
    ts = [One(rng, n, bits, skew=k) for n, k in ((100, 0), (2051, 3), (1, 1))]
    st, h = M.moe_adamw_create([x.entry() for x in ts], bits)
    M.check(st)
    s = torch.cuda.Stream()
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    code = M.MOE_DTYPE_F32 if dtype == "f32" else M.MOE_DTYPE_BF16
    for i, x in enumerate(ts):
        m, r = (torch.full((x.n + 8,), 768.0, dtype=t, device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        M.check(M.moe_adamw_read(h, i, m, None, code, s))
        M.check(M.moe_adamw_read(h, i, None, r, code, s))
        torch.cuda.synchronize()
        assert (m[x.n:] == 768).all() and (r[x.n:] == 768).all()
        if bits == 8:
            assert (_host(m)[:x.n] == A.values_m(x.m.cpu().numpy(), x.ms.cpu().numpy())).all()
            assert (_host(r)[:x.n] == A.values_root(x.v.cpu().numpy(), x.vs.cpu().numpy())).all()
        else:
            assert (m[:x.n] == x.m.to(t)).all()
            tol = (U if dtype == "f32" else 2.0 ** -8) * 1.01
            assert (np.abs(_host(r)[:x.n] - np.sqrt(x.v0.astype(np.float64))) <= tol * np.sqrt(x.v0.astype(np.float64))).all()
    M.check(M.moe_adamw_destroy(h))


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_follow_step_and_rate(bits):
    """Replays of one captured step, with the step's number and the rate changed between them, give what eager steps give."""
    import torch

    from paper_2609_00993_amd import moepd as M

    def make():
        rng = np.random.default_rng(11)
        return [One(rng, n, bits) for n in (100, 2500)]

    s = torch.cuda.Stream()
    results = []
    for captured in (False, True):
        ts = make()
        st, h = M.moe_adamw_create([x.entry() for x in ts], bits)
        M.check(st)
        lr, t = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        go = lambda: M.check(M.moe_adamw_step(h, 0.9, 0.99, 1e-8, lr, t, None, 3, s))  # noqa: E731
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(s):
                graph.capture_begin()
                go()
                graph.capture_end()
        for i in range(1, 5):
            t.fill_(i)
            lr.fill_(1e-3 / i)
            torch.cuda.synchronize()
            graph.replay() if captured else go()
            torch.cuda.synchronize()
        if captured:
            del graph
        M.check(M.moe_adamw_destroy(h))
        results.append([w.clone().view(torch.uint8) for x in ts for w in x.parts.values()])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_refused_on_another_table_or_index():
    import torch

    from paper_2609_00993_amd import moepd as M

    x = One(np.random.default_rng(0), 40, 8)
    st, h = M.moe_adamw_create([x.entry()], 8)
    M.check(st)
    s = torch.cuda.Stream()
    m = torch.empty(40, device="cuda")
    for i in (-1, 1):
        assert M.moe_adamw_read(h, i, m, None, M.MOE_DTYPE_F32, s) == M.MOE_ERR_INVALID_ARG
    assert M.moe_adamw_read(h, 0, m, None, M.MOE_DTYPE_FP8, s) == M.MOE_ERR_INVALID_ARG
    lr, t = torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ok = dict(beta1=0.9, beta2=0.99, eps=1e-8, lr=lr, step=t, grad_scale=None, seed=0, stream=s)
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=float("nan")), dict(eps=-1.0), dict(eps=float("inf")), dict(lr=None),
               dict(step=None), dict(stream=None)):
        assert M.moe_adamw_step(h, **{**ok, **kw}) == M.MOE_ERR_INVALID_ARG
    for k, w in x.parts.items():
        assert (w == x.around[k]).all(), k
    M.check(M.moe_adamw_destroy(h))


@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-30])
@pytest.mark.parametrize("bits", [32, 8])
def test_smallest_roots(bits, eps):
    """v from 1e-36 down below the normal numbers, without an eps that hides it. Each of v's three operations (and the square of an
    8-bit state's root) rounds to steps of 2^-149 there: four halves of one, and half of their share of v in the root."""
    rng = np.random.default_rng(21)
    ts = [One(rng, 200, bits, "f32", False, "f32", size=s) for s in (1e-17, 1e-18, 1e-19, 4e-20, 2e-20)]
    for x in ts:  # no gradient or state near 0, so that v stays above 2^-141
        x.grad.copy_(x.grad.sign() * x.grad.abs().clamp(min=x.grad.abs().max().item() / 4))
        x.g0 = _host(x.grad)
    how = _step(ts, bits, lr=1e-2, eps=eps)
    for x in ts:
        p, m, v = A.step(x.p0, x.g0, x.m0, x.v0, how["lr"], how["t"], how["b1"], how["b2"], eps, x.decay, 1.0)
        assert v.min() > 2.0 ** -141 and (ts[0] is x or v.min() < 2.0 ** -126)
        c1, c2 = 1 - how["b1"] ** how["t"], 1 - how["b2"] ** how["t"]
        den = np.sqrt(v / c2) + eps
        update, slack = np.abs(m) / c1 / den, 4 * U * (how["b1"] * np.abs(x.m0) + np.abs(x.g0)) / c1 / den
        tol = how["lr"] * ((32 * U + 2.0 ** -148 / v) * update + slack + 4 * U * np.abs(x.decay * x.p0)) + 3 * U * np.abs(p)
        got = _host(x.param)
        assert np.isfinite(got).all() and (np.abs(got - p) <= tol).all() and (np.abs(got - x.p0) > 1e-4).any()


@pytest.mark.parametrize("eps", [1e-38, 1e-40, 1e-44, 1e-60])
@pytest.mark.parametrize("bits", [32, 8])
def test_zeros_over_the_smallest_eps(bits, eps):
    """Elements that never had a gradient decay, and nothing else."""
    x = One(np.random.default_rng(22), 100, bits, "f32", False, zeros=True)
    how = _step([x], bits, lr=0.5, eps=eps)
    want = x.p0.astype(np.float64) * (1 - how["lr"] * float(np.float32(x.decay)))
    assert (np.abs(_host(x.param) - want) <= 3 * U * np.abs(x.p0)).all()
