"""The join of two blocks (ff_resnorm_fwd, ff_resnorm_bwd) against the fp64 reference.

Bounds per element, u the activations' unit roundoff, v = 2^-24, propagated to first order from the inputs on.  A normalised
value h = (x - mean) q of a row whose x is off by e_x is off by q (e_x + mean e_x) + |h| q rms(e_x), and by the norm's own
arithmetic, 128 v (|h| + q (|x| + mean|x|)) as for the layer norm: sums of at most 32 terms a thread and 10 levels.  A sum over T
rows adds (T + 64) v of its absolute terms.  Results in the activations' type add u of themselves."""
import numpy as np
import pytest

from oracle import train_oracle as TO
from paper_2608_26430_amd import inputs
from tests.parity_util import to_np, torch_act

torch = pytest.importorskip("torch")
import paper_2608_26430_amd as ff  # noqa: E402

pytestmark = pytest.mark.gpu
V = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
RES, BLOCK, EPS = 0.875, 1.25, 1e-5


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    torch.cuda.set_device(0)
    return torch.device("cuda:0")


def _mean(a):
    return a.mean(axis=1, keepdims=True)


def _norm_error(kind, x, h, q, ex):
    """Errors of h and, relative, of q."""
    own = 128 * V * (np.abs(h) + q * (np.abs(x) + _mean(np.abs(x))))
    eh = q * (ex + _mean(ex)) + np.abs(h) * q * np.sqrt(_mean(ex ** 2)) + own
    return eh, eh.max(axis=1, keepdims=True)


def _grad_error(h, q, eh, rel, a, ea):
    """Error of q (a - mean a - h mean(a h))."""
    A, H = np.abs(a), np.abs(h)
    return q * (ea + _mean(ea) + H * _mean(ea * H) + (64 * V + rel) * (A + _mean(A) + H * _mean(A * H)) + eh * _mean(A * H)
                + H * _mean(A * eh))


def bounds(o, c, post, norm, u):
    """Error bounds of every result of the oracle's o."""
    r, b, dx, dy = (np.asarray(c[k], dtype=np.float64) if c.get(k) is not None else None for k in ("r", "b", "dx", "dy"))
    T, n = r.shape
    B, zero = {}, np.zeros_like(r)
    ehp, relp = (_norm_error(post, b, o["hp"], o["rp"], zero) if post != "none" else (zero, 0.0))
    ep = np.abs(o["pw"]) * ehp + 4 * V * (np.abs(o["pw"] * o["hp"]) + np.abs(o["pb"])) if post != "none" else zero
    sg = np.abs(BLOCK * o["G"])
    ex = sg * ep + 4 * V * (sg * np.abs(o["p"]) + np.abs(RES * r))
    B["x"] = u * np.abs(o["x"]) + ex
    if norm != "none":
        eh, rel = _norm_error(norm, o["x"], o["h"], o["q"], ex)
        B["y"] = u * np.abs(o["y"]) + np.abs(o["w"]) * eh + 4 * V * (np.abs(o["w"] * o["h"]) + np.abs(o["bias"]))
    if "D" not in o:
        return B
    eD = 4 * V * np.abs(o["D"])
    if norm != "none":
        a = dy * o["w"]
        eD = eD + 4 * V * (np.abs(dx) if dx is not None else 0.0) + _grad_error(o["h"], o["q"], eh, rel, a, V * np.abs(a))
        B["dw"] = (np.abs(dy) * eh).sum(axis=0) + (T + 64) * V * np.abs(dy * o["h"]).sum(axis=0)
        B["dbias"] = (T + 64) * V * np.abs(dy).sum(axis=0)
    B["dr"] = u * np.abs(o["dr"]) + RES * eD
    ee = sg * eD + 3 * V * np.abs(o["e"])
    rows = T // o["dgate"].shape[0]
    B["dgate"] = (BLOCK * (eD * np.abs(o["p"]) + np.abs(o["D"]) * ep + (rows + 64) * V * np.abs(o["D"] * o["p"]))
                  ).reshape(-1, rows, n).sum(axis=1)
    B["db"] = u * np.abs(o["db"]) + ee
    if post != "none":
        f = o["e"] * o["pw"]
        B["db"] = u * np.abs(o["db"]) + _grad_error(o["hp"], o["rp"], ehp, relp, f, np.abs(o["pw"]) * ee + V * np.abs(f))
        B["dpw"] = (ee * np.abs(o["hp"]) + np.abs(o["e"]) * ehp + (T + 64) * V * np.abs(o["e"] * o["hp"])).sum(axis=0)
        B["dpb"] = (ee + (T + 64) * V * np.abs(o["e"])).sum(axis=0)
    return B


def close(got, want, bound, what):
    bad = ~(np.abs(to_np(got).reshape(want.shape) - want) <= bound * 1.05 + 1e-30)
    assert not bad.any(), (what, int(bad.sum()), float((np.abs(to_np(got).reshape(want.shape) - want) / (bound + 1e-30)).max()))


def case(T, n, dtype, post, norm, gate, seed, bias=True):
    g = inputs.rng(seed)
    x = inputs.gaussian(g, (T, n), dtype="f32") * 1.3 + 0.5
    c = dict(r=inputs.bf16_round(x) if dtype == "bf16" else x.astype(np.float32), b=inputs.gaussian(g, (T, n), dtype=dtype),
             dx=inputs.gaussian(g, (T, n), dtype=dtype), dy=inputs.gaussian(g, (T, n), dtype=dtype) if norm != "none" else None)
    c["pw"] = inputs.gaussian(g, (n,), std=0.3) + 1 if post != "none" else None
    c["pb"] = inputs.gaussian(g, (n,)) if post != "none" and bias else None
    c["w"] = inputs.gaussian(g, (n,), std=0.3) + 1 if norm != "none" else None
    c["bias"] = inputs.gaussian(g, (n,)) if norm != "none" and bias else None
    c["gate"] = {0: None, 1: inputs.gaussian(g, (n,)) + 1}.get(gate) if gate < 2 else inputs.gaussian(g, (gate, n), dtype=dtype)
    return c


def device_args(c, dtype, dev, gate_dtype=None):
    def vec(a):
        return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev)
    gate = c["gate"]
    if gate is not None:
        gate = vec(gate) if gate.ndim == 1 else torch_act(gate, dtype, dev)
    return dict(gate=gate, post_weight=vec(c["pw"]), post_bias=vec(c["pb"]), weight=vec(c["w"]), bias=vec(c["bias"]))


def reference(c, post, norm):
    return TO.resnorm(c["r"], c["b"], c["gate"], post, c["pw"], c["pb"], norm, c["w"], c["bias"], RES, BLOCK, EPS, c["dx"], c["dy"])


OUT = ("dr", "db", "dgate", "dpw", "dpb", "dw", "dbias")


def run(c, dtype, dev, post, norm, **kw):
    act = {k: None if c[k] is None else torch_act(c[k], dtype, dev) for k in ("r", "b", "dx", "dy")}
    how = dict(post=post, norm=norm, res_scale=RES, block_scale=BLOCK, eps=EPS, **device_args(c, dtype, dev))
    X, Y, stats = ff.resnorm_fwd(act["r"], act["b"], **how)
    return X, Y, stats, ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, **how, **kw), act, how


def check(c, dtype, post, norm, X, Y, stats, grads):
    o = reference(c, post, norm)
    B = bounds(o, c, post, norm, U[dtype])
    close(X, o["x"], B["x"], "x")
    if norm != "none":
        close(Y, o["y"], B["y"], "y")
    else:
        assert Y is None
    want = np.concatenate([o["mp"], o["rp"], o["m"], o["q"]], axis=1)
    assert np.allclose(to_np(stats), want, rtol=1e-4, atol=1e-5)
    for name, g in zip(OUT, grads):
        has = {"dgate": c["gate"], "dpw": c["pw"], "dpb": c["pb"], "dw": c["w"], "dbias": c["bias"]}
        if name in has and has[name] is None:
            assert g is None, name
        else:
            close(g, o[name], B[name], name)


# one row to many; widths of every instance (one, four and eight waves, 4 to 16 elements a lane), odd ones, and
# ones that are read several times
SIZES = [(1, 1), (3, 2), (7, 64), (66, 509), (513, 768), (130, 1000), (40, 1021), (5, 2048), (9, 2056), (700, 1024), (17, 4096),
         (33, 8192), (3, 5001), (20, 8191), (2, 28672), (3, 9001), (600, 15), (600, 509)]
KINDS = [("rms", "rms"), ("layer", "layer"), ("none", "rms"), ("none", "layer"), ("layer", "none"), ("none", "none"), ("layer", "rms")]


@pytest.mark.parametrize("T,n", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes(dev, T, n, dtype):
    """Every kind of norms at every width, the gate's kind changing with them; equal calls give equal bits."""
    for i, (post, norm) in enumerate(KINDS):
        gate = (0, 1, T if T > 1 and T < 50 else 1)[(i + n) % 3]
        c = case(T, n, dtype, post, norm, gate, 100 * T + n + i, bias=i != 0)
        X, Y, stats, grads, act, how = run(c, dtype, dev, post, norm)
        again = ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, **how)
        torch.cuda.synchronize()
        check(c, dtype, post, norm, X, Y, stats, grads)
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("T,groups", [(6, 6), (1200, 2), (1200, 3), (1199, 11), (1400, 700), (2100, 300), (5, 5)])
@pytest.mark.parametrize("n", [500, 4096, 9001])
def test_gates_by_groups(dev, T, groups, n):
    """More and fewer groups than workgroups; groups of one row; shares that no number of workgroups divides."""
    if n > 4096 and T > 1000:
        T, groups = T // groups * 2 if groups > 100 else T // groups, 2 if groups > 100 else 1
    c = case(T, n, "bf16", "layer", "layer", groups if groups > 1 else 1, T + n)
    X, Y, stats, grads, _, _ = run(c, "bf16", dev, "layer", "layer")
    torch.cuda.synchronize()
    check(c, "bf16", "layer", "layer", X, Y, stats, grads)


def _strided(a, dtype, dev, ld, at):
    """Tensor of a's values inside rows of ld elements, `at` elements into the buffer, NaN around."""
    T, n = a.shape
    buf = torch.full((T * ld + at + 8,), float("nan"), device=dev, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    t = torch.as_strided(buf, (T, n), (ld, 1), at)
    t.copy_(torch_act(a, dtype, dev))
    return t, buf


@pytest.mark.parametrize("post,norm", [("rms", "rms"), ("none", "layer"), ("layer", "none"), ("none", "none")])
@pytest.mark.parametrize("n,ld,at", [(1000, 1003, 1), (768, 776, 0), (768, 768, 3), (1021, 1027, 1), (4097, 4097, 0), (8189, 8192, 2), (9000, 9002, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_places_and_outputs_over_inputs(dev, n, ld, at, dtype, post, norm):
    """Rows inside wider ones, off 16-byte alignment; x over r, dr over dx, db over dy or b; gradients added to what is there;
    nothing outside the rows is written or used."""
    T = 37
    c = case(T, n, dtype, post, norm, 1, n + ld)
    t = {k: _strided(c[k], dtype, dev, ld, at) for k in ("r", "b", "dx", "dy") if c[k] is not None}
    how = dict(post=post, norm=norm, res_scale=RES, block_scale=BLOCK, eps=EPS, **device_args(c, dtype, dev))
    r2, _ = _strided(c["r"], dtype, dev, ld, at)
    X, Y, stats = ff.resnorm_fwd(r2, t["b"][0], X=r2, Y=_strided(c["b"] * 0, dtype, dev, ld, at)[0] if norm != "none" else None, **how)
    old = {k: np.float32(i + 1) for i, k in enumerate(OUT)}
    give = {k2: torch.full((n,), float(old[k]), device=dev) for k, k2, v in
            (("dgate", "dgate", c["gate"]), ("dpw", "dpost_weight", c["pw"]), ("dpb", "dpost_bias", c["pb"]), ("dw", "dweight", c["w"]),
             ("dbias", "dbias", c["bias"])) if v is not None}
    over = t["dy"][0] if norm != "none" else t["b"][0]
    grads = ff.resnorm_bwd(t["r"][0], t["b"][0], t["dx"][0], t["dy"][0] if norm != "none" else None, stats, dR=t["dx"][0], dB=over,
                           accumulate=True, **give, **how)
    torch.cuda.synchronize()
    grads = [g if g is None or i < 2 else g - float(old[k]) for i, (k, g) in enumerate(zip(OUT, grads))]
    o = reference(c, post, norm)
    B = bounds(o, c, post, norm, U[dtype])
    close(X, o["x"], B["x"], "x")
    if norm != "none":
        close(Y, o["y"], B["y"], "y")
    for k, g in zip(OUT, grads):
        if g is not None:
            # adding to what is there and taking it off again: a rounding each
            close(g, o[k], B[k] + (0 if k in ("dr", "db") else 2 * V * (np.abs(o[k]) + old[k])), k)
    for name, (_, buf) in t.items():
        out = np.ones(buf.numel(), dtype=bool)
        out[(np.arange(T)[:, None] * ld + at + np.arange(n)[None, :]).ravel()] = False
        assert np.isnan(to_np(buf)[out]).all(), name


def test_offsets_past_32_bits(dev):
    """Rows 65,600 elements apart, 65,600 of them: bits equal to those of packed rows."""
    T, ld, n = 65600, 65600, 40
    if torch.cuda.mem_get_info()[0] < 12 * 2 ** 30:
        pytest.skip("needs 12 GiB")
    buf = torch.empty(T * ld, device=dev, dtype=torch.bfloat16).view(T, ld)
    gen = torch.Generator(device=dev).manual_seed(3)
    far = [buf[:, 48 * i:48 * i + n] for i in range(8)]
    near = [torch.randn((T, n), device=dev, generator=gen).bfloat16() for _ in range(4)] + [None] * 4
    for a, b in zip(far[:4], near[:4]):
        a.copy_(b)
    w = torch.randn((2, n), device=dev, generator=gen)
    how = dict(gate=torch.randn((41, n), device=dev, generator=gen), post="layer", post_weight=w[0], norm="rms", weight=w[1])
    got = []
    for R, B, dX, dY, X, Y, dR, dB in (near, far):
        X, Y, stats = ff.resnorm_fwd(R, B, X=X, Y=Y, **how)
        got.append((X, Y, stats, *ff.resnorm_bwd(R, B, dX, dY, stats, dR=dR, dB=dB, **how)))
    torch.cuda.synchronize()
    assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(*got))
    assert bool(got[0][1].isfinite().all()) and bool((got[0][4] != 0).any(dim=1).all())


def test_some_gradients_only(dev):
    """No dx, no dr, no db, no vectors, one vector: what is asked for is as in the whole call."""
    c = case(90, 1024, "bf16", "rms", "layer", 3, 5)
    X, Y, stats, grads, act, how = run(c, "bf16", dev, "rms", "layer")
    z = dict(c, dx=None)
    got = ff.resnorm_bwd(act["r"], act["b"], None, act["dy"], stats, want_dr=False, **how)
    torch.cuda.synchronize()
    o = reference(z, "rms", "layer")
    B = bounds(o, z, "rms", "layer", U["bf16"])
    assert got[0] is None
    for k, g in list(zip(OUT, got))[1:]:
        close(g, o[k], B[k], k)
    got = ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, want_vectors=False, want_db=False, **how)
    torch.cuda.synchronize()
    assert torch.equal(got[0], grads[0]) and all(g is None for g in got[1:])
    dw = torch.empty(1024, device=dev)
    got = ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, want_vectors=False, dweight=dw, **how)
    torch.cuda.synchronize()
    assert torch.equal(got[5], grads[5]) and torch.equal(got[1], grads[1]) and got[2] is None and got[6] is None


def test_no_rows(dev):
    e = torch.empty((0, 64), device=dev)
    w = torch.ones(64, device=dev)
    X, Y, stats = ff.resnorm_fwd(e, e, weight=w, gate=w)
    out = ff.resnorm_bwd(e, e, e, e, stats, weight=w, gate=w)
    torch.cuda.synchronize()
    assert X.shape == (0, 64) and not bool(out[2].any()) and not bool(out[5].any())
    keep = torch.full((64,), 3.0, device=dev)
    ff.resnorm_bwd(e, e, e, e, stats, weight=w, dweight=keep, accumulate=True)
    torch.cuda.synchronize()
    assert bool((keep == 3).all())


def test_vectors_and_gates_in_bf16(dev):
    c = case(70, 1536, "f32", "layer", "layer", 7, 8)
    for k in ("pw", "pb", "w", "bias", "gate"):
        c[k] = inputs.bf16_round(c[k])
    act = {k: torch_act(c[k], "f32", dev) for k in ("r", "b", "dx", "dy")}
    v = {k: torch_act(a, "bf16", dev) for k, a in (("gate", c["gate"]), ("post_weight", c["pw"]), ("post_bias", c["pb"]),
                                                   ("weight", c["w"]), ("bias", c["bias"]))}
    wide = torch.full((7, 2000), float("nan"), device=dev, dtype=torch.bfloat16)
    wide[:, :1536] = v["gate"]
    v["gate"] = wide[:, :1536]
    how = dict(post="layer", norm="layer", res_scale=RES, block_scale=BLOCK, eps=EPS, **v)
    X, Y, stats = ff.resnorm_fwd(act["r"], act["b"], **how)
    grads = ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, **how)
    torch.cuda.synchronize()
    check(c, "f32", "layer", "layer", X, Y, stats, grads)


def test_refusals(dev):
    R = torch.ones((6, 64), device=dev)
    B, w, half = R * 2, torch.ones(64, device=dev), torch.ones(64, device=dev, dtype=torch.bfloat16)
    X, Y, stats = ff.resnorm_fwd(R, B, weight=w)
    bad = [lambda: ff.resnorm_fwd(R, B[0]), lambda: ff.resnorm_fwd(R[0], B[0]), lambda: ff.resnorm_fwd(R, B.bfloat16()),
           lambda: ff.resnorm_fwd(R, B[:5]), lambda: ff.resnorm_fwd(R, B.t()), lambda: ff.resnorm_fwd(R, B.cpu()),
           lambda: ff.resnorm_fwd(R, B, norm="batch"), lambda: ff.resnorm_fwd(R, B, weight=w[:63]),
           lambda: ff.resnorm_fwd(R, B, weight=w.double()), lambda: ff.resnorm_fwd(R, B, weight=w, bias=half),
           lambda: ff.resnorm_fwd(R, B, weight=torch.ones(128, device=dev)[::2]), lambda: ff.resnorm_fwd(R, B, post_weight=w),
           lambda: ff.resnorm_fwd(R, B, norm="none", bias=w), lambda: ff.resnorm_fwd(R, B, gate=w[:32]),
           lambda: ff.resnorm_fwd(R, B, gate=torch.ones((4, 64), device=dev)), lambda: ff.resnorm_fwd(R, B, gate=w.double()),
           lambda: ff.resnorm_fwd(R, B, gate=torch.ones((), device=dev)), lambda: ff.resnorm_fwd(R, B, X=torch.ones((6, 65), device=dev)),
           lambda: ff.resnorm_fwd(R, B, stats=torch.ones((6, 3), device=dev)), lambda: ff.resnorm_bwd(R, B, X, None, stats, weight=w),
           lambda: ff.resnorm_bwd(R, B, X, Y, stats[:5], weight=w), lambda: ff.resnorm_bwd(R, B, X, Y, stats, weight=w, dR=Y[0]),
           lambda: ff.resnorm_bwd(R, B, X, Y, stats, weight=w, accumulate=True), lambda: ff.resnorm_bwd(R, B, X, Y, stats, dgate=w)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", i)
    for call in (lambda: ff.resnorm_fwd(R, B, eps=-1.0), lambda: ff.resnorm_fwd(R, B, X=Y, Y=Y),
                 lambda: ff.resnorm_bwd(R, B, X, Y, stats, dR=X, dB=X), lambda: ff.resnorm_bwd(R, B, X, Y, stats, dweight=w, weight=w,
                                                                                              workspace=torch.empty(16, dtype=torch.uint8, device=dev))):
        with pytest.raises(ff.FrameFTError) as ei:
            call()
        assert ei.value.name == "FF_EINVAL"


def test_rows_of_nothing_and_of_one_value(dev):
    """Rows of zeros (rstd = 1 / sqrt(eps)) and constant rows of a layer norm give finite results and gradients."""
    n = 1000
    r = torch.zeros((4, n), device=dev)
    b = torch.zeros((4, n), device=dev)
    b[1] = 3.0
    r[2] = -2.0
    g = torch.ones((4, n), device=dev)
    for kind in ("rms", "layer"):
        X, Y, stats = ff.resnorm_fwd(r, b, post=kind, norm=kind)
        grads = ff.resnorm_bwd(r, b, g, g, stats, post=kind, norm=kind)
        torch.cuda.synchronize()
        assert torch.isfinite(Y).all() and torch.isfinite(grads[0]).all() and torch.isfinite(grads[1]).all()
        assert not bool(Y[0].any())


def test_captured_and_replayed_on_another_stream(dev):
    """Forward and backward captured once, replayed with new values between eager calls on the default stream: every replay
    equals the eager call."""
    post, norm = "rms", "rms"
    cs = [case(600, 2048, "bf16", post, norm, 6, s, bias=False) for s in range(3)]
    c = cs[0]
    act = {k: torch_act(c[k], "bf16", dev) for k in ("r", "b", "dx", "dy")}
    how = dict(post=post, norm=norm, res_scale=RES, block_scale=BLOCK, eps=EPS, **device_args(c, "bf16", dev))
    ws, ws2 = ff.resnorm_workspace(600, 2048, 6), ff.resnorm_workspace(600, 2048, 6)

    def step(ws, stream=None):
        X, Y, stats = ff.resnorm_fwd(act["r"], act["b"], stream=stream, **how)
        return (X, Y, *ff.resnorm_bwd(act["r"], act["b"], act["dx"], act["dy"], stats, workspace=ws, stream=stream, **how))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(ws)
    for c in cs:
        for k in act:
            act[k].copy_(torch_act(c[k], "bf16", dev))
        graph.replay()
        eager = step(ws2)
        torch.cuda.synchronize()
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(out, eager))
        other = step(ws2, side)
        torch.cuda.synchronize()
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(other, eager))
