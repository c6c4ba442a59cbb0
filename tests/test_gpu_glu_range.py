"""The gated feed-forward's backward where G or U is large: finite inputs give the gradients that they determine.

In bf16, G and U are kept as words that end at 2^26 (1 - 2^-11); larger ones are kept as infinity.  With such a G, f' is 1 or 0 and f is 0
below; with dH = 0 both gradients are 0; what needs the value itself, dH f(G) of a large positive G and dH U f'(G) of a large U,
is infinite.  Without kept words nothing ends: the function's slope is 1 or 0 to the largest numbers.

Bounds, u the type's unit roundoff, v = 2^-24: dG = dH U f'(G) has U's word (2^-10; fp32 exact), two products and the result (u); at |G|
>= 16 the functions' slopes differ from 1 and 0 by less than 2e-6 (SiLU: 17 exp -16)."""
import pytest

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402
from tests.test_gpu_glu import DT, FNS, U, check_products, kept_values  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def large(T, n, F, dtype, dev, seed):
    """A call whose G and U come from what is added: per element G large, U large or neither (all at least 16 in size, so that the
    slope is 1 or 0), of both signs, up to 2^100; dH = 0 here and there."""
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DT[dtype]

    def rand(*s):
        return torch.rand(s, generator=gen, device=dev)
    sign = torch.where(rand(2, T, F) < 0.5, -1.0, 1.0)
    size = torch.exp2(26.5 + 73 * rand(2, T, F))
    kind = (3 * rand(T, F)).int()
    Ag = sign[0] * torch.where(kind == 1, size[0], 16 + 100 * rand(T, F))
    Au = sign[1] * torch.where(kind == 2, size[1], 1 + 100 * rand(T, F))
    # (a large U with a slope of 1, so that its gradient is as large)
    Ag = torch.where(kind == 2, Ag.abs(), Ag)
    dH = torch.where(rand(T, F) < 0.2, 0.0, torch.where(rand(T, F) < 0.5, -1.0, 1.0) * (0.5 + rand(T, F)))
    X = torch.zeros((T, n), device=dev)
    Wg, Wu = (torch.randn((F, n), generator=gen, device=dev) / n ** 0.5 for _ in range(2))
    return dict(X=X.to(dt), Wg=Wg.to(dt), Wu=Wu.to(dt), Ag=Ag.to(dt), Au=Au.to(dt), dH=dH.to(dt)), kind


def near(got, want, u, what):
    err = (got.double() - want).abs()
    assert bool((err <= u * want.abs()).all()), (what, float((err / want.abs().clamp(min=1e-30)).max()))


@pytest.mark.parametrize("fn", FNS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n,F", [(5, 64, 64), (300, 128, 1000), (700, 1032, 1544)])
def test_large_g_and_u(dev, T, n, F, dtype, fn):
    d, kind = large(T, n, F, dtype, dev, T + n)
    g, p, x = (d[k].double() for k in ("Ag", "Au", "dH"))
    slope = (g > 0).double()
    want_g, want_u = x * p * slope, x * g * slope
    _, G, P = ff.glu_fwd(d["X"], d["Wg"], d["Wu"], fn, d["Ag"], d["Au"], save=True)
    made = ff.glu_bwd(d["dH"], d["X"], d["Wg"], d["Wu"], fn, Ag=d["Ag"], Au=d["Au"], want_dx=False)
    kept = ff.glu_bwd(d["dH"], d["X"], d["Wg"], d["Wu"], fn, G=G, U=P, want_dx=False)
    torch.cuda.synchronize()
    u = U[DT[dtype]] + 4e-6
    below = g < 0
    near(made[0][~below], want_g[~below], u, "dG")
    near(made[1][~below], want_u[~below], u, "dU")
    # below -16 what is left of f and f' is under 2e-6 of dH U and dH G, and nothing at all far below
    assert bool((made[0][below].abs() <= 2e-6 * (x * p)[below].abs()).all() and (made[1][below].abs() <= 2e-6 * (x * g)[below].abs()).all())
    far = below & (kind == 1)
    assert not bool(made[0][far].any()) and not bool(made[1][far].any())
    words = kept_values(G).isinf(), kept_values(P).isinf()
    assert torch.equal(words[0], kind == 1) == (dtype == "bf16") and torch.equal(words[1], kind == 2) == (dtype == "bf16")
    for got, want, lost, name in ((kept[0], want_g, words[1], "dG"), (kept[1], want_u, words[0] & ~below, "dU")):
        some = x != 0
        near(got[~lost & ~below], want[~lost & ~below], u + 2.0 ** -10, name)
        assert not bool(got[~some].any()) and not bool(got[far].any()), name
        assert torch.equal(got[lost & some].double(), want[lost & some].sign() * float("inf")), name
        assert bool(got[~lost].isfinite().all()), name


@pytest.mark.parametrize("fn", FNS)
def test_rows_without_gradient_reach_nothing(dev, fn):
    """Padding rows, dH = 0, whose G and U are kept as infinities: dX and both weights' gradients are the other rows'."""
    T, n, F = 130, 256, 512
    d, _ = large(T, n, F, "bf16", dev, 3)
    gen = torch.Generator(device=dev).manual_seed(4)
    d["X"] = torch.randn((T, n), generator=gen, device=dev).to(torch.bfloat16)
    d["dH"] = torch.randn((T, F), generator=gen, device=dev).to(torch.bfloat16)
    pad = torch.arange(T, device=dev) % 3 == 1
    d["dH"][pad] = 0
    for k in ("Ag", "Au"):
        d[k][~pad] = torch.randn((int((~pad).sum()), F), generator=gen, device=dev).to(torch.bfloat16)
    _, G, P = ff.glu_fwd(d["X"], d["Wg"], d["Wu"], fn, d["Ag"], d["Au"], save=True)
    out = ff.glu_bwd(d["dH"], d["X"], d["Wg"], d["Wu"], fn, G=G, U=P, want_dw=True)
    torch.cuda.synchronize()
    assert bool(kept_values(G)[pad].isinf().any()) and bool(kept_values(P)[pad].isinf().any())
    assert all(bool(t.isfinite().all()) for t in out) and not bool(out[0][pad].any()) and not bool(out[2][pad].any())
    check_products(d, *out)


def test_nan_stays_seen(dev):
    """A NaN that was added to G is kept as infinity: dU is not finite there, whatever the function."""
    d, _ = large(40, 64, 64, "bf16", dev, 5)
    d["Ag"] = torch.full_like(d["Ag"], float("nan"))
    d["dH"] = torch.ones_like(d["dH"])
    for fn in FNS:
        H, G, P = ff.glu_fwd(d["X"], d["Wg"], d["Wu"], fn, d["Ag"], None, save=True)
        dU = ff.glu_bwd(d["dH"], d["X"], d["Wg"], d["Wu"], fn, G=G, U=P, want_dx=False)[1]
        torch.cuda.synchronize()
        assert bool(H.isnan().all()) and not bool(dU.isfinite().any()), fn


def test_where_words_become_infinite(dev):
    """The largest word is 2^26 (1 - 2^-10); half a step above it, at 2^26 (1 - 2^-11), rounding goes to infinity, of either sign."""
    n = 64
    top, half = 2.0 ** 26 * (1 - 2.0 ** -10), 2.0 ** 26 * (1 - 2.0 ** -11)
    want = torch.tensor([0.0, top, 2.0 ** 26 * (1 - 2.0 ** -9), half - 256, half, half + 256, 2.0 ** 26, 2.0 ** 100], device=dev).repeat(n // 8)
    want = torch.stack((want, -want))
    # G in two parts that bf16 holds: what W = 1 makes of X, and what is added
    x = want.to(torch.bfloat16)
    rest = (want - x.float()).to(torch.bfloat16)
    assert torch.equal(x.float() + rest.float(), want)
    eye = torch.eye(n, device=dev, dtype=torch.bfloat16)
    _, G, P = ff.glu_fwd(x, eye, eye, "silu", rest, rest, save=True)
    torch.cuda.synchronize()
    kept = torch.tensor([0.0, top, 2.0 ** 26 * (1 - 2.0 ** -9), top, float("inf"), float("inf"), float("inf"), float("inf")],
                        device=dev, dtype=torch.float64).repeat(n // 8)
    kept = torch.stack((kept, -kept))
    assert torch.equal(kept_values(G), kept) and torch.equal(kept_values(P), kept)


def test_gradients_over_what_they_are_made_of(dev):
    """dG and dU over G and U, over U and G, dG or dU over dH, with infinite words among the others: as in memory of their own."""
    bf = torch.bfloat16
    d, _ = large(70, 64, 200, "bf16", dev, 6)
    args = d["X"], d["Wg"], d["Wu"], "gelu_tanh"
    _, G, P = ff.glu_fwd(*args, d["Ag"], d["Au"], save=True)
    want = ff.glu_bwd(d["dH"], *args, G=G, U=P, want_dx=False)[:2]
    got = []
    for place in ("words", "words crossed", "dG over dH", "dU over dH"):
        x, g, p = d["dH"].clone(), G.clone(), P.clone()
        own = {"words": (g.view(bf), p.view(bf)), "words crossed": (p.view(bf), g.view(bf)), "dG over dH": (x, None), "dU over dH": (None, x)}[place]
        got.append(ff.glu_bwd(x, *args, G=g, U=p, dG=own[0], dU=own[1], want_dx=False)[:2])
    torch.cuda.synchronize()
    # (an infinity's sign counts, a zero's does not)
    assert all(torch.equal(a, b) for pair in got for a, b in zip(pair, want))
