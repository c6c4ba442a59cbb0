"""Performance cases of the operators of a block's step: gated feed-forward, the join of two blocks, AdamW over a
set of tensors.

`listed()` are the standing cases, `draw(rng)` further ones of the same ranges.  `prepare(case, seed)` makes what a
program holds before the call (inputs on the GPU, and with `own` the workspace or the set that it keeps), `run(state)`
is one pass: with `own` the package's public calls, otherwise the operators in plain torch operations in fp32 (fp64 where
a state of 8 bits is rounded), rounded once at the end.  `work(case)` is the bytes and operations that the pass cannot
do without, `exact(case, seed)` its results from the definitions in float64.

Kinds of case:
  glu         H = f(X Wg^T [+ Ag]) * (X Wu^T [+ Au]): a gated feed-forward block up to its down projection; Ag and Au
              are what adapters on the two projections add.
  glu_step    its training step: forward, then backward from dH with the gradients of both projections' results (which
              the adapters' backwards take), dX, and with `dw` those of the weights.  keep: G and U are kept for the
              backward; otherwise it makes them again.
  join        x = a r + s gate * post(b), y = norm(x): what stands between two blocks.
  join_step   the same and its backward: gradients of the stream, the block's output, the gate and the norms' vectors.
  adamw       one AdamW step over a set of tensors, states in fp32 or in 8 bits (whose values are then read).
"""
import math

import torch

own = False


def listed():
    def glu(name, kind, T, n, F, dtype="bf16", fn="silu", adapters=False, dw=False, keep=True):
        return dict(name=name, kind=kind, tokens=T, n=n, hidden=F, dtype=dtype, fn=fn, adapters=adapters, dw=dw, keep=keep)

    def join(name, kind, T, n, dtype="bf16", post="none", norm="rms", gate="none", groups=1):
        return dict(name=name, kind=kind, tokens=T, n=n, dtype=dtype, post=post, norm=norm, gate=gate, groups=groups)

    def adamw(name, count, length, states, vectors=0, width=0, grads="f32", copies=False):
        return dict(name=name, kind="adamw", count=count, length=length, vectors=vectors, width=width, states=states,
                    grads=grads, copies=copies)

    return [
        # one token of a 4096-wide model with 11008 hidden units: reads both weights once
        glu("glu_decode", "glu", 1, 4096, 11008),
        # evaluation of a 1024-wide model with adapters on both projections, an odd number of tokens
        glu("glu_eval", "glu", 2003, 1024, 4096, fn="gelu", adapters=True),
        # fine-tuning of a 4096-wide model, 4096 tokens, weights frozen, adapters on both projections
        glu("glu_frozen_step", "glu_step", 4096, 4096, 11008, adapters=True),
        # a small model trained whole, ragged sizes, nothing kept between forward and backward
        glu("glu_full_step", "glu_step", 1003, 768, 2304, fn="gelu_tanh", dw=True, keep=False),
        # fp32 training of a small model
        glu("glu_f32_step", "glu_step", 500, 768, 2048, "f32", dw=True),
        # between two blocks of a 4096-wide model in decoding, norms on both sides of a block: latency
        join("join_decode", "join", 16, 4096, post="rms"),
        # ViT-B/16 in training, 64 images x 197 tokens, a learned scale for each channel of the block's output
        join("join_vit_step", "join_step", 64 * 197, 768, norm="layer", gate="vector"),
        # the widest model in training, 8192 tokens, norms on both sides
        join("join_wide_step", "join_step", 8192, 8192, post="rms"),
        # fp32, a gate computed for each of 7 samples, a width that is no multiple of the wave's
        join("join_f32_step", "join_step", 7 * 143, 1000, "f32", post="layer", norm="layer", gate="rows", groups=7),
        # one adapter of a 256-wide layer with the vectors of its norm: latency
        adamw("adamw_small", 1, 1000, "f32", 2, 256),
        # the adapters of a 32-layer model, seven projections each, of different lengths, and the norms' vectors
        adamw("adamw_stack", 224, 20000, "f32", 65, 4096),
        # three feed-forward weights of 4096 x 11008 trained in mixed precision, states in 8 bits
        adamw("adamw_ffn_8bit", 3, 4096 * 11008, "8bit", 2, 4096, "bf16", True),
    ]


# -------------------------------------------------------------------------------------- draws

_MAX_GLU = 8 * 4096 * 4096 * 11008      # operations of the largest listed step


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["glu", "glu_step", "glu_step", "join", "join_step", "join_step", "adamw", "adamw"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind.startswith("glu"):
        T, n, F = _log_int(rng, 1, 4096), 8 * _log_int(rng, 16, 512), 8 * _log_int(rng, 16, 1376)
        if rng.random() < 0.6:              # most widths are multiples of 128
            n, F = max(128, n // 128 * 128), max(128, F // 128 * 128)
        if dtype == "f32":                  # the fp32 models are the smaller ones
            T, n, F = min(T, 2048), min(n, 1024), min(F, 4096)
        step = kind == "glu_step"
        dw, keep = step and rng.random() < 0.4, not step or rng.random() < 0.7
        T = max(1, min(T, _MAX_GLU // (n * F * (4 + 4 * step + 4 * dw + 4 * (not keep)))))
        return dict(kind=kind, tokens=T, n=n, hidden=F, dtype=dtype, fn=rng.choice(["silu", "gelu", "gelu_tanh"]),
                    adapters=rng.random() < 0.5, dw=dw, keep=keep)
    if kind.startswith("join"):
        n = _log_int(rng, 64, 8192)
        if rng.random() < 0.7:
            n = max(64, n // 64 * 64)
        gate = rng.choice(["none", "vector", "rows"])
        groups = _log_int(rng, 1, 64) if gate == "rows" else 1
        T = max(1, _log_int(rng, 1, 8192) // groups) * groups
        post, norm = rng.choice([("none", "rms"), ("none", "layer"), ("rms", "rms"), ("layer", "layer"), ("layer", "none")])
        return dict(kind=kind, tokens=T, n=n, dtype=dtype, post=post, norm=norm, gate=gate, groups=groups)
    count = _log_int(rng, 1, 256)
    length = min(_log_int(rng, 100, 1 << 25), (1 << 26) // count)
    return dict(kind="adamw", count=count, length=length, vectors=rng.randrange(0, 65), width=_log_int(rng, 64, 8192),
                states=rng.choice(["f32", "8bit"]), grads=rng.choice(["f32", "bf16"]), copies=rng.random() < 0.5)


# -------------------------------------------------------------------------------------- inputs

_HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=40, scale=0.5)
_DECAY = 0.01
_RES, _BLOCK, _EPS = 0.875, 1.25, 1e-5      # scales of the stream and the block, the norms' eps


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _lengths(case):
    """Lengths of a set's tensors: the largest first, the others spread over a third to the whole of it."""
    n, L = case["count"], case["length"]
    return [max(1, int(L * (1.0 - 0.65 * ((i * 0.6180339887) % 1.0)))) for i in range(n)] + [case["width"]] * case["vectors"]


def _flat(case, dtype):
    """One array for all tensors of a set, each at the next multiple of 256 elements, and the tensors as views of it."""
    lengths = _lengths(case)
    at = [0]
    for n in lengths:
        at.append(at[-1] + (n + 255) // 256 * 256)
    flat = torch.zeros((at[-1],), dtype=dtype, device="cuda")
    return flat, [flat[a:a + n] for a, n in zip(at, lengths)]


def _glu_data(case, seed):
    T, n, F, dt = case["tokens"], case["n"], case["hidden"], _dtype(case)
    gen = _generator(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    d = dict(X=randn(T, n).to(dt), Wg=(randn(F, n) * (1.5 / math.sqrt(n))).to(dt), Wu=(randn(F, n) / math.sqrt(n)).to(dt),
             Ag=None, Au=None)
    if case["adapters"]:
        d["Ag"], d["Au"] = (0.2 * randn(T, F)).to(dt), (0.2 * randn(T, F)).to(dt)
    if case["kind"] == "glu_step":
        d["dH"] = randn(T, F).to(dt)
    return d


def _join_data(case, seed):
    """The stream has a mean and a spread for each column, as streams of trained models have."""
    T, n, dt = case["tokens"], case["n"], _dtype(case)
    gen = _generator(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def vectors(norm):
        if norm == "none":
            return None, None
        return 1.0 + 0.1 * randn(n), 0.1 * randn(n) if norm == "layer" else None

    d = dict(R=(randn(T, n) * (1.0 + 0.3 * randn(n)) + 0.5 * randn(n)).to(dt), B=(0.7 * randn(T, n) + 0.1 * randn(n)).to(dt))
    d["pw"], d["pb"] = vectors(case["post"])
    d["w"], d["b"] = vectors(case["norm"])
    d["gate"] = {"none": lambda: None, "vector": lambda: 0.5 + 0.2 * randn(n),
                 "rows": lambda: (0.5 + 0.5 * randn(case["groups"], n)).to(dt)}[case["gate"]]()
    if case["kind"] == "join_step":
        d["dX"] = randn(T, n).to(dt)
        d["dY"] = randn(T, n).to(dt) if case["norm"] != "none" else None
    return d


def _adamw_data(case, seed):
    """Tensors in the middle of a training run: gradients of another size for each tensor, moments that fit them."""
    gen = _generator(seed)
    gdt = torch.bfloat16 if case["grads"] == "bf16" else torch.float32
    eight = case["states"] == "8bit"
    d = dict(g=[], mx=[], vx=[], seed=0x9E3779B97F4A7C15 ^ (seed * 0x2545F4914F6CDD1D & (1 << 62) - 1))
    d["c_all"], d["c"] = _flat(case, torch.float32)
    d["w_all"], d["w"] = _flat(case, torch.bfloat16) if case["copies"] else (None, None)
    d["m_all"], d["m"] = _flat(case, torch.uint8 if eight else torch.float32)
    d["v_all"], d["v"] = _flat(case, torch.uint8 if eight else torch.float32)
    for i, n in enumerate(_lengths(case)):
        size = 1e-3 * 10.0 ** (i % 4 - 2)

        def randn():
            return torch.randn((n,), generator=gen, device="cuda")

        d["c"][i].copy_(0.02 * randn())
        d["g"].append((2 * size * randn()).to(gdt))
        m, v = 0.3 * size * randn(), size * size * (0.05 + randn().square_())
        if eight:
            for x, codes, exps, top in ((m, "m", "mx", 14), (v, "v", "vx", 30)):
                k = _unit(_blocks(x), top)
                d[codes][i].copy_(_encode(_blocks(x).double(), k, 0.5, top).view(-1)[:n])
                d[exps].append((k + 120).to(torch.uint8))
        else:
            d["m"][i].copy_(m)
            d["v"][i].copy_(v)
    d["decay"] = [_DECAY] * case["count"] + [0.0] * case["vectors"]
    return d


def prepare(case, seed):
    kind = case["kind"]
    st = dict(case=case)
    if kind == "adamw":
        st.update(_adamw_data(case, seed))
        if own:
            import paper_2608_26430_amd as ff
            s = ff.AdamWSet(st["c"], weight_decay=st["decay"], states=case["states"], copies=st["w"],
                            grad_dtype=st["g"][0].dtype, betas=(_HYPER["beta1"], _HYPER["beta2"]), eps=_HYPER["eps"],
                            seed=st["seed"])
            for i in range(len(st["c"])):
                s.m[i].copy_(st["m"][i])
                s.v[i].copy_(st["v"][i])
                if case["states"] == "8bit":
                    s.m_exp[i].copy_(st["mx"][i])
                    s.v_exp[i].copy_(st["vx"][i])
            st["set"], st["grads"] = s, s.grads(st["g"])
            for k in ("m_all", "m", "mx", "v_all", "v", "vx"):
                del st[k]
        return st
    st.update(_glu_data(case, seed) if kind.startswith("glu") else _join_data(case, seed))
    if own:
        import paper_2608_26430_amd as ff
        if kind == "glu_step":
            st["ws"] = ff.glu_workspace(case["tokens"], case["n"], case["hidden"], _dtype(case), want_dx=True,
                                        want_dw=case["dw"])
        elif kind == "join_step":
            st["ws"] = ff.resnorm_workspace(case["tokens"], case["n"], case["groups"])
    return st


# -------------------------------------------------------------------------------------- one pass

def _run_own(st):
    import paper_2608_26430_amd as ff
    case = st["case"]
    kind = case["kind"]
    if kind == "adamw":
        h, s = _HYPER, st["set"]
        s.step(st["grads"], h["lr"], h["step"], grad_scale=h["scale"])
        m, v = s.read()
        return [t for t in (st["c_all"], st["w_all"], m, v) if t is not None]
    if kind == "glu":
        return ff.glu_fwd(st["X"], st["Wg"], st["Wu"], case["fn"], st["Ag"], st["Au"])
    if kind == "glu_step":
        X, Wg, Wu, fn, Ag, Au = st["X"], st["Wg"], st["Wu"], case["fn"], st["Ag"], st["Au"]
        if case["keep"]:
            H, G, U = ff.glu_fwd(X, Wg, Wu, fn, Ag, Au, save=True)
            out = ff.glu_bwd(st["dH"], X, Wg, Wu, fn, G=G, U=U, want_dw=case["dw"], workspace=st["ws"])
        else:
            H = ff.glu_fwd(X, Wg, Wu, fn, Ag, Au)
            out = ff.glu_bwd(st["dH"], X, Wg, Wu, fn, Ag=Ag, Au=Au, want_dw=case["dw"], workspace=st["ws"])
        return (H,) + (out if case["dw"] else out[:3])
    how = dict(gate=st["gate"], post=case["post"], post_weight=st["pw"], post_bias=st["pb"], norm=case["norm"],
               weight=st["w"], bias=st["b"], res_scale=_RES, block_scale=_BLOCK, eps=_EPS)
    X, Y, stats = ff.resnorm_fwd(st["R"], st["B"], **how)
    if kind == "join":
        return [t for t in (X, Y, stats) if t is not None]
    grads = ff.resnorm_bwd(st["R"], st["B"], st["dX"], st["dY"], stats, workspace=st["ws"], **how)
    return [t for t in (X, Y, *grads) if t is not None]


def _gated(fn, g):
    """f(g) and f'(g) in g's type."""
    if fn == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if fn == "gelu":
        cdf = 0.5 * torch.erfc(g * -math.sqrt(0.5))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    c = math.sqrt(2.0 / math.pi)
    s = 1.0 / (1.0 + torch.exp(-2.0 * c * (g + 0.044715 * g * g * g)))
    return g * s, s + g * s * (1.0 - s) * 2.0 * c * (1.0 + 3 * 0.044715 * g * g)


def _run_glu(st):
    case, dt = st["case"], st["X"].dtype
    X, Wg, Wu = st["X"].float(), st["Wg"].float(), st["Wu"].float()
    G, U = X @ Wg.t(), X @ Wu.t()
    if st["Ag"] is not None:
        G += st["Ag"].float()
        U += st["Au"].float()
    f, df = _gated(case["fn"], G)
    H = (f * U).to(dt)
    if case["kind"] == "glu":
        return H
    dH = st["dH"].float()
    dG, dU = dH * U * df, dH * f
    dX = dG @ Wg + dU @ Wu
    out = (H, dG.to(dt), dU.to(dt), dX.to(dt))
    return out + ((dG.t() @ X).to(dt), (dU.t() @ X).to(dt)) if case["dw"] else out


def _normed(kind, x, eps):
    """Normalised rows, their mean and 1 / deviation."""
    mean = x.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    xc = x - mean
    rstd = 1.0 / torch.sqrt((xc * xc).mean(dim=1, keepdim=True) + eps)
    return xc * rstd, mean, rstd


def _normed_back(kind, h, rstd, a):
    """Gradient of the row from a, that of its normalised values h."""
    d = a - h * (a * h).mean(dim=1, keepdim=True)
    return rstd * (d - a.mean(dim=1, keepdim=True) if kind == "layer" else d)


def _run_join(st):
    case, dt = st["case"], st["R"].dtype
    T, n = case["tokens"], case["n"]
    r, b = st["R"].float(), st["B"].float()
    zero = torch.zeros((T, 1), device="cuda")
    p, pm, pr, hp = b, zero, zero, None
    if case["post"] != "none":
        hp, pm, pr = _normed(case["post"], b, _EPS)
        p = hp * st["pw"] + (st["pb"] if st["pb"] is not None else 0.0)
    gate = _BLOCK
    if case["gate"] == "vector":
        gate = _BLOCK * st["gate"]
    elif case["gate"] == "rows":
        gate = _BLOCK * st["gate"].float().repeat_interleave(T // case["groups"], dim=0)
    x = _RES * r + gate * p
    m, s, h, y = zero, zero, None, None
    if case["norm"] != "none":
        h, m, s = _normed(case["norm"], x, _EPS)
        y = h * st["w"] + (st["b"] if st["b"] is not None else 0.0)
    out = [x.to(dt)] + ([y.to(dt)] if y is not None else [])
    if case["kind"] == "join":
        return out + [torch.cat((pm, pr, m, s), dim=1)]
    dx, grads = st["dX"].float(), [None] * 4
    if y is not None:
        dy = st["dY"].float()
        grads[2] = (dy * h).sum(dim=0)
        grads[3] = dy.sum(dim=0) if st["b"] is not None else None
        dx = dx + _normed_back(case["norm"], h, s, dy * st["w"])
    dgate = None
    if case["gate"] != "none":
        dgate = (_BLOCK * dx * p).view(case["groups"], -1, n).sum(dim=1)
        dgate = dgate[0] if case["gate"] == "vector" else dgate
    db = gate * dx
    if hp is not None:
        grads[0] = (db * hp).sum(dim=0)
        grads[1] = db.sum(dim=0) if st["pb"] is not None else None
        db = _normed_back(case["post"], hp, pr, db * st["pw"])
    return out + [t for t in ((_RES * dx).to(dt), db.to(dt), dgate, *grads) if t is not None]


# States of 8 bits: blocks of 256 values share a unit 2^k; a code c stands for c units below 16 and (8 + c % 8) 2^(c / 8 - 1)
# from there on.  m has a sign in bit 7 and 7 bits of code (up to 15 x 2^14 units), v 8 bits (up to 15 x 2^30).  k is the
# least that holds the block's largest value, at least -120.  Values are rounded up where a random fraction (16 bits and a
# half) carries theirs over the next code; a positive v has a code of 1 at least; where a moment is not finite, both have the code 0.
# (The half: moments of short gradients and codes often lie on multiples of 2^-16 of a step, where the last bit of the
# 64 would decide.)

def _blocks(x):
    """x as rows of 256, zero behind its end."""
    return torch.nn.functional.pad(x, (0, -x.numel() % 256)).view(-1, 256)


def _two(k):
    """2^k (float64) for an integer tensor."""
    return (k.long() + 1023 << 52).view(torch.float64)


def _unit(x, top):
    """Exponents k of the blocks' units."""
    big = x.abs().amax(dim=1).float()
    frac, e = torch.frexp(big)                  # big = frac 2^e, frac in [0.5, 1)
    k = e - (top + 4) + (frac > 0.9375).to(e.dtype)
    return torch.where(big > 0, k, torch.full_like(k, -120)).clamp(-120, 135)


def _encode(x, k, r, top):
    """Codes of the blocks x (float64) in units 2^k, r in [0, 1) the random fractions."""
    y = x.abs() * _two(-k)[:, None]
    t = (torch.frexp(y)[1] - 4).clamp(min=0)    # step between codes 2^t units
    q = torch.floor(y * _two(-t) + r).to(torch.int64)
    code = (8 * t + q).clamp(max=8 * top + 15)
    if top == 30:
        return torch.where(x > 0, code.clamp(min=1), code)
    return code + 128 * (x < 0)


def _decode(codes, k, top):
    """Values of codes (int64 blocks) in units 2^k, float64."""
    a = codes if top == 30 else codes & 127
    e = (a >> 3).clamp(min=1) - 1
    y = (a - 8 * e).double() * _two(e + k[:, None])
    return y if top == 30 else torch.where(codes >= 128, -y, y)


def _philox(block, step, number, seed):
    """Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): four
    32-bit words, as int64 tensors, of counter (block, step, number) under key seed."""
    m32 = 0xFFFFFFFF
    c0, c1 = block & m32, block >> 32
    c2, c3 = torch.full_like(block, step & m32), torch.full_like(block, number & m32)
    k0, k1 = seed & m32, seed >> 32 & m32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57         # modulo 2^64: every bit of the product
        c0, c1, c2, c3 = (b >> 32 & m32) ^ c1 ^ k0, b & m32, (a >> 32 & m32) ^ c3 ^ k1, a & m32
        k0, k1 = k0 + 0x9E3779B9 & m32, k1 + 0xBB67AE85 & m32
    return c0, c1, c2, c3


def _run_adamw(st):
    case, h = st["case"], _HYPER
    b1, b2 = h["beta1"], h["beta2"]
    bc1, bc2 = 1.0 - b1 ** h["step"], 1.0 - b2 ** h["step"]
    eight = case["states"] == "8bit"
    m_all, v_all = st["m_all"], st["v_all"]
    if eight:
        (m_all, ms), (v_all, vs) = _flat(case, torch.bfloat16), _flat(case, torch.bfloat16)
    for i, c in enumerate(st["c"]):
        n = c.numel()
        g = st["g"][i].double() * h["scale"] if eight else st["g"][i].float() * h["scale"]
        m, v = st["m"][i], st["v"][i]
        if eight:
            mk, vk = st["mx"][i].int() - 120, st["vx"][i].int() - 120
            m = _decode(_blocks(m).long(), mk, 14).view(-1)[:n]
            v = _decode(_blocks(v).long(), vk, 30).view(-1)[:n]
        m = b1 * m + (1.0 - b1) * g
        v = b2 * v + (1.0 - b2) * (g * g)
        m32, v32 = m.float(), v.float()
        c.mul_(1.0 - h["lr"] * st["decay"][i])
        c.sub_(h["lr"] * (m32 / bc1) / (torch.sqrt(v32 / bc2) + h["eps"]))
        if st["w"] is not None:
            st["w"][i].copy_(c)
        if eight:
            words = torch.stack(_philox(torch.arange((n + 3) // 4, device="cuda"), h["step"], i, st["seed"]), dim=1).view(-1)[:n]
            for x, codes, exps, top, shift, values in ((m, "m", "mx", 14, 0, ms), (v, "v", "vx", 30, 16, vs)):
                xb = _blocks(torch.where(m32.isfinite() & v32.isfinite(), x, torch.zeros_like(x)))
                k = _unit(xb, top)
                code = _encode(xb, k, _blocks(((words >> shift & 0xFFFF).double() + 0.5) / 65536.0), top)
                st[codes][i].copy_(code.view(-1)[:n])
                st[exps][i].copy_(k + 120)
                values[i].copy_(_decode(code, k, top).view(-1)[:n])
        else:
            st["m"][i].copy_(m)
            st["v"][i].copy_(v)
    return [t for t in (st["c_all"], st["w_all"], m_all, v_all) if t is not None]


def run(st):
    if own:
        return _run_own(st)
    kind = st["case"]["kind"]
    if kind == "adamw":
        return _run_adamw(st)
    return _run_glu(st) if kind.startswith("glu") else _run_join(st)


# -------------------------------------------------------------------------------------- bounds

def work(case):
    kind = case["kind"]
    if kind == "adamw":
        N = float(sum(_lengths(case)))
        # parameters both ways, gradients; the states both ways, and where they are codes, their values
        each = 8 + (2 if case["grads"] == "bf16" else 4) + (2 if case["copies"] else 0)
        each += 16 if case["states"] == "f32" else 2 * 2 * (1 + 1 / 256) + 4
        return {"bytes": N * each, "flops": 15.0 * N}
    T, n = case["tokens"], case["n"]
    e = 2 if case["dtype"] == "bf16" else 4
    if kind.startswith("join"):
        ops = 4 if kind == "join" else 10       # r, b -> x, y; then r, b, dx, dy -> dr, db
        if case["norm"] == "none":
            ops -= 1 if kind == "join" else 2
        return {"bytes": float(ops) * T * n * e + 40.0 * n, "flops": (14.0 if kind == "join" else 50.0) * T * n}
    F, step = case["hidden"], kind == "glu_step"
    data = T * n + 2 * F * n + T * F + (2 * T * F if case["adapters"] else 0)
    products = 2
    if step:
        # dH -> dG, dU; G and U both ways or made again; dX, the weights' gradients
        data += 3 * T * F + (4 * T * F if case["keep"] else 0) + T * n + (2 * F * n if case["dw"] else 0)
        products += 2 + (2 if case["dw"] else 0) + (0 if case["keep"] else 2)
    return {"bytes": float(data) * e, "flops": 2.0 * products * T * n * F}


# -------------------------------------------------------------------------------------- float64

def _exact_glu(case, seed):
    d = _glu_data(case, seed)
    X, Wg, Wu = d["X"].double(), d["Wg"].double(), d["Wu"].double()
    G, U = torch.nn.functional.linear(X, Wg), torch.nn.functional.linear(X, Wu)
    if case["adapters"]:
        G, U = G + d["Ag"].double(), U + d["Au"].double()
    G.requires_grad_()
    f = (torch.nn.functional.silu(G) if case["fn"] == "silu" else
         torch.nn.functional.gelu(G, approximate="tanh" if case["fn"] == "gelu_tanh" else "none"))
    H = f.detach() * U
    if case["kind"] == "glu":
        return H
    dH = d["dH"].double()
    dG, = torch.autograd.grad(f, G, dH * U)
    dU = dH * f.detach()
    dX = torch.cat((dG, dU), dim=1) @ torch.cat((Wg, Wu), dim=0)
    return (H, dG, dU, dX, dG.t() @ X, dU.t() @ X) if case["dw"] else (H, dG, dU, dX)


def _exact_join(case, seed):
    d = _join_data(case, seed)
    T, n = case["tokens"], case["n"]
    step = case["kind"] == "join_step"
    names = [k for k in ("R", "B", "gate", "pw", "pb", "w", "b") if d[k] is not None]
    q = {k: d[k].double().requires_grad_(step) for k in names}

    def norm(kind, x, w, b):
        mu = x.sum(1, keepdim=True) / n if kind == "layer" else torch.zeros_like(x[:, :1])
        r = (((x - mu) ** 2).sum(1, keepdim=True) / n + _EPS) ** -0.5
        y = (x - mu) * r * w
        return y if b is None else y + b, mu, r

    none = torch.zeros((T, 1), dtype=torch.float64, device="cuda")
    p, stats = q["B"], [none] * 4
    if case["post"] != "none":
        p, *stats[:2] = norm(case["post"], p, q["pw"], q.get("pb"))
    p = _BLOCK * p
    if case["gate"] != "none":
        p = (p.view(case["groups"], -1, n) * q["gate"].view(case["groups"], 1, n)).view(T, n)
    x = p + _RES * q["R"]
    out, up = [x], [d["dX"].double()] if step else None
    if case["norm"] != "none":
        y, *stats[2:] = norm(case["norm"], x, q["w"], q.get("b"))
        out.append(y)
        if step:
            up.append(d["dY"].double())
    if not step:
        return out + [torch.cat(stats, dim=1)]
    grads = torch.autograd.grad(out, [q[k] for k in names], up)
    return [t.detach() for t in out] + list(grads)


def _mul_hi_lo(a, m):
    """High and low 32 bits of a m for a < 2^32 (int64 tensor) and a constant m < 2^32, by 16-bit limbs."""
    m1, m0 = m >> 16, m & 0xFFFF
    a1, a0 = a >> 16, a & 0xFFFF
    mid = a1 * m0 + ((a0 * m0) >> 16)
    mid2 = a0 * m1 + (mid & 0xFFFF)
    return a1 * m1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) + ((a0 * m0) & 0xFFFF)


def _values(top):
    """The value of every code without its sign, in units."""
    return torch.tensor([float(a if a < 16 else (8 + a % 8) << (a // 8 - 1)) for a in range(8 * top + 16)],
                        dtype=torch.float64, device="cuda")


def _powers(k):
    """2^k (float64) for a tensor of whole numbers from -250 to 250, from a table."""
    return torch.tensor([2.0 ** i for i in range(-250, 251)], dtype=torch.float64, device="cuda")[k.long() + 250]


def _exact_state(x, finite, draws, top):
    """The values that a moment x (float64) has after its rounding to 8 bits; draws: 16 random bits for each."""
    n, grid = x.numel(), _values(top)
    rows = -(-n // 256)
    full = torch.zeros((rows * 256,), dtype=torch.float64, device="cuda")
    full[:n] = torch.where(finite, x, torch.zeros_like(x))
    full = full.view(rows, 256)
    # the least power of two for which the block's largest value, in fp32, is one of the codes' values or below
    big = full.abs().max(dim=1).values.float().double()
    k = torch.ceil(torch.log2((big / grid[-1]).clamp(min=2.0 ** -130)))
    k = torch.where(big > grid[-1] * _powers(k), k + 1, k)
    k = torch.where(big <= grid[-1] * _powers(k - 1), k - 1, k).clamp(min=-120.0)
    y = full.abs() / _powers(k)[:, None]
    at = (torch.searchsorted(grid, y, right=True) - 1).clamp(max=len(grid) - 2)
    low, high = grid[at], grid[at + 1]
    r = torch.zeros((rows * 256,), dtype=torch.float64, device="cuda")
    r[:n] = draws.double() + 0.5
    up = ((y - low) / (high - low) + r.view(rows, 256) / 65536.0) >= 1.0
    z = torch.where(up, high, low)
    if top == 30:
        z = torch.where((full > 0) & (z == 0), torch.ones_like(z), z)
    return (torch.sign(full) * z * _powers(k)[:, None]).view(-1)[:n]


def _exact_adamw(case, seed):
    d, h = _adamw_data(case, seed), _HYPER
    eight = case["states"] == "8bit"
    (c_all, cs), (m_all, ms), (v_all, vs) = (_flat(case, torch.float64) for _ in range(3))
    for i, c in enumerate(d["c"]):
        n = c.numel()
        g = d["g"][i].double() * h["scale"]
        if eight:
            mc, vc = d["m"][i].long(), d["v"][i].long()
            m = _values(14)[mc % 128] * (1 - 2 * (mc // 128)) * _powers(d["mx"][i].long() - 120).repeat_interleave(256)[:n]
            v = _values(30)[vc] * _powers(d["vx"][i].long() - 120).repeat_interleave(256)[:n]
        else:
            m, v = d["m"][i].double(), d["v"][i].double()
        m = m + (1.0 - h["beta1"]) * (g - m)
        v = v + (1.0 - h["beta2"]) * (g * g - v)
        x = c.double()
        x = x - h["lr"] * d["decay"][i] * x
        x = x - h["lr"] * (m / (1.0 - h["beta1"] ** h["step"])) / ((v / (1.0 - h["beta2"] ** h["step"])) ** 0.5 + h["eps"])
        cs[i].copy_(x)
        if eight:
            e = torch.arange(n, device="cuda")
            blk = e // 4
            q = [blk % 2 ** 32, blk // 2 ** 32, torch.zeros_like(blk) + h["step"], torch.zeros_like(blk) + i]
            key = [d["seed"] % 2 ** 32, d["seed"] // 2 ** 32]
            for r in range(10):
                hi0, lo0 = _mul_hi_lo(q[0], 0xD2511F53)
                hi1, lo1 = _mul_hi_lo(q[2], 0xCD9E8D57)
                q = [hi1 ^ q[1] ^ (key[0] + r * 0x9E3779B9) % 2 ** 32, lo1,
                     hi0 ^ q[3] ^ (key[1] + r * 0xBB67AE85) % 2 ** 32, lo0]
            word = torch.where(e % 4 < 2, torch.where(e % 2 == 0, q[0], q[1]), torch.where(e % 2 == 0, q[2], q[3]))
            finite = (m.abs() <= torch.finfo(torch.float32).max) & (v <= torch.finfo(torch.float32).max)
            m, v = _exact_state(m, finite, word % 65536, 14), _exact_state(v, finite, word // 65536, 30)
        ms[i].copy_(m)
        vs[i].copy_(v)
    return [c_all] + ([c_all.clone()] if case["copies"] else []) + [m_all, v_all]


def exact(case, seed):
    if case["kind"] == "adamw":
        return _exact_adamw(case, seed)
    return _exact_glu(case, seed) if case["kind"].startswith("glu") else _exact_join(case, seed)
