"""AdamW over a set of tensors (ff_adamw_set_*) against the fp64 optimizer oracle, one step at a time from the GPU's own
previous state, element by element.

fp32 states, u = 2^-24 (each rounding at most u relative): m takes b1's rounding, the product's inside the fma and the result's
(3 u b1 |m|), and those of 1 - b1, the scaled gradient, their product and the result (5 u (1 - b1) |g|); v the same with the
gradient's twice and the square's (7 u).  The step's denominator takes half of v's 7 u, of the bias correction's u and
its product's u, the root's own u and the sum's u, the numerator the correction's u and its product's u, then division, rate and
product u each: under 16 u of the step, beside what m's own error moves it by.  c takes the decay's, its product's and the
difference's rounding: 3 u |c|, 1 u |step|.
8-bit states: the codes are the oracle's (both compute in fp64 and compare with a random fraction that no short number meets);
c as above with m and v off by their one rounding to fp32."""
import numpy as np
import pytest

from oracle import optim_oracle as OO
from paper_2608_26430_amd import inputs
from tests.parity_util import to_np

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BETAS, EPS = (0.9, 0.999), 1e-8
LENGTHS = [1, 3, 4, 255, 256, 257, 0, 1000, 4096, 4097, 10007]


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def _grad(rng, n, std, dtype):
    x = inputs.gaussian(rng, (n,), std=std)
    return inputs.bf16_round(x) if dtype is torch.bfloat16 else x


def _check_c(c0, c1, m, em, v, t, lr, wd):
    """c1 against c0 stepped with the exact moments m, v, of which the GPU's m is off by at most em."""
    den = np.sqrt(v / (1 - BETAS[1] ** t)) + EPS
    step = lr * (m / (1 - BETAS[0] ** t)) / den
    want = c0 * (1 - lr * wd) - step
    bound = 3 * U * np.abs(c0) + 17 * U * np.abs(step) + lr / (1 - BETAS[0] ** t) * em / den
    assert np.all(np.abs(c1 - want) <= bound * 1.01 + 1e-37), float((np.abs(c1 - want) / (bound + 1e-37)).max())


class _Run:
    """A set with its oracle-side view; tensors start `at` elements into their buffers, and nothing around them is written."""

    def __init__(self, dev, lengths, states, gdt, at=0, copies=True, seed=1, decay=0.01):
        self.gdt, self.lengths, self.states, self.seed = gdt, lengths, states, seed
        rng = inputs.rng(sum(lengths) + at)
        self.rng = rng
        self.decay = [decay if i % 2 == 0 else 0.0 for i in range(len(lengths))]
        self.buf = [torch.full((n + at + 5,), 7.0, device=dev) for n in lengths]
        self.wbuf = [torch.full((n + at + 5,), 7.0, device=dev, dtype=torch.bfloat16) for n in lengths]
        self.gbuf = [torch.full((n + at + 5,), float("nan"), device=dev, dtype=gdt) for n in lengths]
        self.c = [b[at:at + n] for b, n in zip(self.buf, lengths)]
        self.w = [b[at:at + n] for b, n in zip(self.wbuf, lengths)] if copies else None
        self.g = [b[at:at + n] for b, n in zip(self.gbuf, lengths)]
        self.at = at
        for c in self.c:
            c.copy_(torch.from_numpy(inputs.gaussian(rng, (c.numel(),), std=0.02)))
        self.set = ff.AdamWSet(self.c, weight_decay=self.decay, states=states, copies=self.w, grad_dtype=gdt, betas=BETAS,
                               eps=EPS, seed=seed)

    def state(self, i):
        s = self.set
        if self.states == "f32":
            return to_np(s.m[i]), to_np(s.v[i])
        return [to_np(t) for t in (s.m[i], s.v[i], s.m_exp[i], s.v_exp[i])]

    def step(self, t, lr, scale=1.0, std=1.0, skip=(), call=None):
        gs = []
        for i, n in enumerate(self.lengths):
            x = _grad(self.rng, n, std * 10.0 ** (i % 3 - 1), self.gdt)
            self.g[i].copy_(torch.from_numpy(x))
            gs.append(x.astype(np.float64) * scale)
        before = [(to_np(self.c[i]),) + tuple(self.state(i)) for i in range(len(self.lengths))]
        call = call or self.set.step
        call([None if i in skip else g for i, g in enumerate(self.g)], lr, t, grad_scale=scale)
        torch.cuda.synchronize()
        for i, n in enumerate(self.lengths):
            if n == 0:
                continue
            c0, *old = before[i]
            new, c1 = self.state(i), to_np(self.c[i])
            if i in skip:
                assert np.array_equal(c0, c1) and all(np.array_equal(a, b) for a, b in zip(old, new))
                continue
            if self.states == "f32":
                m0, v0 = old
                _, m, v = OO.adamw_step(c0, gs[i], m0, v0, t, lr, *BETAS, EPS, self.decay[i])
                b1, b2 = BETAS
                em = U * (3 * b1 * np.abs(m0) + 5 * (1 - b1) * np.abs(gs[i])) + 1e-38
                ev = U * (3 * b2 * v0 + 7 * (1 - b2) * gs[i] ** 2) + 1e-38
                assert np.all(np.abs(new[0] - m) <= em * 1.01) and np.all(np.abs(new[1] - v) <= ev * 1.01)
            else:
                m0, v0, mx0, vx0 = old
                _, m, v = OO.adamw_step(c0, gs[i], OO.state_values(m0, mx0, True), OO.state_values(v0, vx0, False), t, lr, *BETAS,
                                        EPS, self.decay[i])
                want = OO.adamw8_step(c0, gs[i], m0, v0, mx0, vx0, t, i, self.seed, lr, *BETAS, EPS, self.decay[i])[1:]
                for a, b, name in zip(new, (want[0], want[1], want[2], want[3]), ("m", "v", "m_exp", "v_exp")):
                    assert np.array_equal(a, b), (i, n, name, int((a != b).sum()))
                em = U * np.abs(m)
            _check_c(c0, c1, m, em, v, t, lr, self.decay[i])
            if self.w is not None:
                assert torch.equal(self.w[i], self.c[i].to(torch.bfloat16))
        for b, n in zip(self.buf + self.wbuf, self.lengths * 2):
            assert bool((b[:self.at] == 7).all()) and bool((b[self.at + n:] == 7).all())


@pytest.mark.parametrize("at", [0, 1])
@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_steps_match_the_oracle(dev, states, gdt, at):
    """Ragged lengths, one of them zero, tensors off 16-byte alignment, four steps with gradients of other sizes each."""
    run = _Run(dev, LENGTHS, states, gdt, at)
    for t, std in ((1, 1.0), (2, 1e-3), (3, 0.5), (4, 1e-6)):
        run.step(t, 0.1 / t, scale=0.25, std=std)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_more_tensors_than_one_launch_takes(dev, states):
    """900 tensors of 1 to 900 elements; some without a gradient stay as they are."""
    run = _Run(dev, [1 + (i * 37) % 900 for i in range(900)], states, torch.float32, copies=False)
    run.step(1, 0.05, skip={0, 5, 383, 384, 899})
    run.step(2, 0.05)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_extreme_gradients(dev, states):
    """Blocks of zeros, gradients of 1e-30 beside 1e4, and alone; those whose square leaves fp32, infinities and NaN."""
    n = 1024
    c = torch.from_numpy(inputs.gaussian(inputs.rng(3), (n,))).to(dev)
    s = ff.AdamWSet([c], states=states, betas=BETAS, eps=EPS, seed=9)
    g = np.zeros(n, dtype=np.float32)
    g[256:512] = inputs.gaussian(inputs.rng(4), (256,)) * 1e-30
    g[512:768] = np.where(np.arange(256) % 2, 1e4, 1e-30)
    g[768:] = inputs.gaussian(inputs.rng(5), (256,))
    g[[800, 801, 802, 803]] = np.inf, np.nan, 1e30, -np.inf
    c0 = to_np(c)
    s.step([torch.from_numpy(g).to(dev)], 0.01, 1)
    m, v = s.read()
    torch.cuda.synchronize()
    c1, m, v = to_np(c), to_np(m), to_np(v)
    odd = np.array([800, 801, 802, 803])
    rest = np.setdiff1d(np.arange(n), odd)
    assert np.isfinite(c1[rest]).all() and np.isnan(c1[[801]]).all()
    assert np.array_equal(c1[:256], c0[:256])
    with np.errstate(all="ignore"):
        em = 0.1 * g.astype(np.float64)
    if states == "f32":
        assert np.all(np.abs(m[rest] - em[rest]) <= 5 * U * np.abs(em[rest]) + 1e-38)
        return
    # four significant bits, and nothing above a step of the block's unit below that
    assert not m[odd].any() and not v[odd].any()
    for b in range(4):
        k = np.arange(256 * b, 256 * b + 256)
        k = k[~np.isin(k, odd)]
        for got, want, units in ((m, em, 2.0 ** 18), (v, 1e-3 * g.astype(np.float64) ** 2, 2.0 ** 34)):
            step = np.maximum(np.abs(want[k]) / 8, max(np.abs(want[k]).max() / units * 4, 2.0 ** -120))
            assert np.all(np.abs(got[k] - want[k]) <= step)
    assert np.all(v[512:768] > 0) and not v[:256].any()
    # another step without gradients: nothing forgotten is brought back, nothing is divided by zero
    s.step([torch.zeros(n, device=dev)], 0.01, 2)
    torch.cuda.synchronize()
    assert np.isfinite(to_np(c)[rest]).all()


def test_device_values_and_captured_steps(dev):
    """lr, the gradients' scale and the step number from the device: a captured step, replayed between eager work, equals eager
    steps with the same values, in both kinds of states."""
    for states in ("f32", "8bit"):
        runs = []
        for captured in (True, False):
            rng = inputs.rng(11)
            c = [torch.from_numpy(inputs.gaussian(rng, (n,))).to(dev) for n in (700, 5000)]
            g = [torch.from_numpy(inputs.gaussian(rng, (n,))).to(dev) for n in (700, 5000)]
            s = ff.AdamWSet(c, weight_decay=0.01, states=states, seed=5)
            lr, sc = torch.ones(1, device=dev), torch.ones(1, device=dev)
            step = torch.zeros(1, dtype=torch.int64, device=dev)
            if captured:
                s.step(s.grads(g), 0.0, 1, lr_dev=lr)        # loads the kernels; lr = 0 and ...
                for t in s.m + s.v + (s.m_exp + s.v_exp if s.m_exp else []):
                    t.zero_()                                # ... cleared moments leave the start
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    s.step(s.grads(g), 0.5, 1, grad_scale=2.0, lr_dev=lr, grad_scale_dev=sc, step_dev=step)
            for t in range(4):
                for x in g:
                    x.mul_(-0.7)
                lr.fill_(0.125 / (t + 1))
                sc.fill_(0.25 * (t + 1))
                step.fill_(t)
                if captured:
                    graph.replay()
                else:
                    s.step(g, 0.5 * 0.125 / (t + 1) if t != 2 else 0.5 * float(np.float32(0.125 / 3)), t + 1,
                           grad_scale=2.0 * 0.25 * (t + 1))
                torch.cuda.synchronize()
            m, v = s.read()
            runs.append([x.clone() for x in c] + [m.clone(), v.clone()])
        for a, b in zip(*runs):
            # the bias corrections come from another pow: one rounding of the factors
            assert torch.allclose(a.float(), b.float(), rtol=4 * U, atol=1e-7 * float(b.float().abs().max())), states


def test_equal_inputs_give_equal_bits_on_any_stream(dev):
    out = []
    for other in (False, True):
        rng = inputs.rng(21)
        c = [torch.from_numpy(inputs.gaussian(rng, (n,))).to(dev) for n in (3000, 70)]
        g = [torch.from_numpy(inputs.gaussian(rng, (n,))).to(dev) for n in (3000, 70)]
        s = ff.AdamWSet(c, states="8bit", seed=2 ** 63 + 5)
        stream = torch.cuda.Stream() if other else None
        if other:
            stream.wait_stream(torch.cuda.current_stream())
        for t in (1, 2, 3):
            s.step(g, 0.01, t, stream=stream)
        m, v = s.read(stream=stream)
        torch.cuda.synchronize()
        out.append([*c, m, v])
    assert all(torch.equal(a, b) for a, b in zip(*out))
    # the second tensor's draws are its own
    assert not torch.equal(out[0][2][:70], out[0][2][s.offsets[1]:s.offsets[1] + 70])


def test_read_gives_the_codes_values_and_zeros_behind_the_end(dev):
    run = _Run(dev, [300, 1, 256], "8bit", torch.float32)
    run.step(1, 0.1)
    m, v = run.set.read()
    torch.cuda.synchronize()
    assert m.dtype is torch.bfloat16 and m.numel() == 512 + 256 + 256
    m, v = to_np(m), to_np(v)
    for i, (o, n) in enumerate(zip(run.set.offsets, run.lengths)):
        cm, cv, xm, xv = run.state(i)
        assert np.array_equal(m[o:o + n], OO.state_values(cm, xm, True))
        assert np.array_equal(v[o:o + n], OO.state_values(cv, xv, False))
        end = o + -(-n // 256) * 256
        assert not m[o + n:end].any() and not v[o + n:end].any()


def test_offsets_past_32_bits(dev):
    """One tensor of 2^31 + 300 elements: its last elements step as a tensor of their own would."""
    n = 2 ** 31 + 300
    if torch.cuda.mem_get_info()[0] < 30 * 2 ** 30:
        pytest.skip("needs 30 GiB")
    tail = 300 + 256        # whole blocks
    x = torch.from_numpy(inputs.gaussian(inputs.rng(8), (tail,))).to(dev)
    gx = torch.from_numpy(inputs.bf16_round(inputs.gaussian(inputs.rng(9), (tail,)))).to(dev, torch.bfloat16)
    c, g = torch.zeros(n, device=dev), torch.zeros(n, device=dev, dtype=torch.bfloat16)
    c[-tail:] = x
    g[-tail:] = gx
    s = ff.AdamWSet([c], states="8bit", grad_dtype=torch.bfloat16, seed=4)
    s.step([g], 0.1, 1)
    torch.cuda.synchronize()
    m = 0.1 * to_np(gx)
    v = 0.001 * to_np(gx) ** 2
    _check_c(to_np(x), to_np(c[-tail:]), m, U * np.abs(m), v, 1, 0.1, 0.0)
    from oracle.train_oracle import philox4x32
    e = np.arange(n - tail, n)
    b = (e // 4).astype(np.uint64)
    w = philox4x32(np.stack([b & np.uint64(0xFFFFFFFF), b >> np.uint64(32), np.full_like(b, 1), np.zeros_like(b)], axis=-1), (4, 0))
    w = w[np.arange(tail), e % 4].astype(np.int64)
    cm, xm = OO.state_codes(m, w % 65536, True)
    assert np.array_equal(to_np(s.m[0][-tail:]), cm) and np.array_equal(to_np(s.m_exp[0][-3:]), xm)
    assert not bool(s.m[0][:-tail].any()) and not bool(c[:-tail].any())


def test_refusals_write_nothing(dev):
    c = torch.ones(100, device=dev)
    with pytest.raises(ValueError):
        ff.AdamWSet([])
    with pytest.raises(ValueError):
        ff.AdamWSet([c.double()])
    with pytest.raises(ValueError):
        ff.AdamWSet([c], states="4bit")
    with pytest.raises(ValueError):
        ff.AdamWSet([c], copies=[torch.ones(99, device=dev, dtype=torch.bfloat16)])
    with pytest.raises(ff.FrameFTError):
        ff.AdamWSet([c], weight_decay=-1.0)
    s = ff.AdamWSet([c])
    g = torch.ones(100, device=dev)
    with pytest.raises(ValueError):
        s.step([g, g], 0.1, 1)
    with pytest.raises(ValueError):
        s.step([g.bfloat16()], 0.1, 1)
    with pytest.raises(ValueError):
        s.step(ff.AdamWSet([torch.ones(7, device=dev)]).grads([torch.ones(7, device=dev)]), 0.1, 1)
    with pytest.raises(ff.FrameFTError):
        ff.AdamWSet([c, c])
    with pytest.raises(ValueError):
        s.step([torch.ones(200, device=dev)[::2]], 0.1, 1)
    for kw in (dict(lr=0.1, step=0), dict(lr=-0.1, step=1), dict(lr=float("nan"), step=1), dict(lr=0.1, step=1, grad_scale=float("inf"))):
        with pytest.raises(ff.FrameFTError) as ei:
            s.step([g], **kw)
        assert ei.value.name == "FF_EINVAL"
    for betas, eps in (((1.0, 0.9), 1e-8), ((0.9, -0.1), 1e-8), ((0.9, 0.999), 0.0), ((0.9, 0.999), 1e-60)):
        with pytest.raises(ff.FrameFTError):
            ff.AdamWSet([c], betas=betas, eps=eps).step([g], 0.1, 1)
    torch.cuda.synchronize()
    assert bool((c == 1).all()) and not bool(s.m_all.any())
