"""The Peri-LN residual update and its gradients against the formulas in 64 bits.

Tolerances.  An fp32 output is off by its roundings: the row sums (d terms each, added in
a tree or in short runs: below 32 * 2^-24 of the summed magnitudes) and a dozen
operations, so 1e-5 of the row's largest magnitude, plus 1e-5 of the value; where a
row's deviation is far below its mean (f = 1 + small), the subtraction of the mean costs what it
costs in the inputs, which the tests do not go to.  bf16 outputs add 2^-8 of the value.  Sums over
rows: 1e-5 of the sum of magnitudes.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2510_05361_gb300 as P
    P.load()
    return P


def inputs(rows, d, stream, branch, weights="f32", bias=False, gate=0, gate_kind="f32", extra=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def draw(shape, kind, scale=1.0, at=0.0):
        return (torch.randn(shape, device="cuda", generator=gen) * scale + at).to(KINDS[kind])

    def wide(kind, scale):
        return draw((rows, d + extra), kind, scale)[:, :d]
    s = {"x": wide(stream, 1.0), "f": wide(branch, 0.5), "post_weight": draw((d,), weights, 0.3, 1.0),
         "pre_weight": draw((d,), weights, 0.3, 1.0), "dy": wide(stream, 0.1), "dh": wide(branch, 0.1)}
    if bias:
        s |= {"post_bias": draw((d,), weights, 0.2), "pre_bias": draw((d,), weights, 0.2)}
    if gate:
        s["gate"] = draw((gate, d), gate_kind, 0.4, 0.5)
    return s


def definition(s, norm, a, with_y=None):
    """y, h, the statistics and all gradients, with torch's autograd on CPU doubles."""
    leaf = {k: v.double().cpu().requires_grad_() for k, v in s.items() if k not in ("dy", "dh")}

    def normed(z):
        if norm == "layer":
            z = z - z.mean(1, keepdim=True)
        return z / torch.sqrt((z * z).mean(1, keepdim=True) + EPS)
    z = normed(leaf["f"]) * leaf["post_weight"]
    if "post_bias" in leaf:
        z = z + leaf["post_bias"]
    if "gate" in leaf:
        z = z * leaf["gate"].repeat_interleave(z.shape[0] // leaf["gate"].shape[0], 0)
    y = a * leaf["x"] + z
    h = normed(y) * leaf["pre_weight"]
    if "pre_bias" in leaf:
        h = h + leaf["pre_bias"]
    loss = (h * s["dh"].double().cpu()).sum()
    if s["dy"] is not None:
        loss = loss + (y * s["dy"].double().cpu()).sum()
    names = list(leaf)
    grads = dict(zip(names, torch.autograd.grad(loss, [leaf[k] for k in names])))
    return y.detach(), h.detach(), grads


def near(got, want, what, scale=None):
    got, want = got.double().cpu(), want.double()
    if not want.numel():
        return
    scale = want.abs().amax(-1, keepdim=True) if scale is None else scale
    tol = 1e-5 * scale + 1e-5 * want.abs()
    if what[1] == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    worst = ((got - want).abs() - tol).max()
    assert worst <= 0, (what, float(worst), float((got - want).abs().max()))


CASES = [  # rows, d, norm, stream, branch, weights, bias, gate rows, gate kind, extra
    (1, 1, "rms", "f32", "f32", "f32", False, 0, "f32", 0),
    (1, 1, "layer", "f32", "f32", "f32", True, 1, "f32", 0),
    (3, 2, "layer", "bf16", "bf16", "f32", True, 3, "bf16", 0),
    (5, 7, "rms", "f32", "bf16", "bf16", False, 1, "bf16", 1),
    (4, 64, "layer", "bf16", "bf16", "bf16", True, 2, "bf16", 0),
    (17, 129, "rms", "f32", "f32", "f32", False, 17, "f32", 3),
    (33, 256, "layer", "f32", "f32", "f32", False, 0, "f32", 0),
    (64, 513, "layer", "bf16", "bf16", "f32", True, 4, "f32", 0),
    (6, 768, "layer", "bf16", "bf16", "f32", True, 0, "f32", 8),
    (700, 768, "rms", "f32", "bf16", "f32", False, 7, "bf16", 0),
    (1000, 1001, "layer", "f32", "f32", "f32", True, 8, "f32", 3),
    (300, 1024, "rms", "bf16", "bf16", "bf16", False, 1, "bf16", 0),
    (41, 2048, "rms", "bf16", "bf16", "f32", False, 41, "bf16", 0),
    (41, 2048, "layer", "bf16", "bf16", "f32", True, 1, "f32", 8),
    (7, 4096, "layer", "f32", "bf16", "f32", True, 7, "bf16", 0),
    (5, 8192, "rms", "f32", "f32", "f32", False, 1, "f32", 0),
    (2, 8193, "layer", "bf16", "bf16", "f32", True, 2, "f32", 0),
    (3, 16384, "layer", "f32", "f32", "f32", True, 1, "f32", 0),
    (9, 5120, "rms", "bf16", "bf16", "bf16", False, 9, "bf16", 0),
    (400, 5120, "layer", "f32", "bf16", "f32", True, 5, "f32", 0),
    (300, 6144, "layer", "f32", "f32", "f32", True, 1, "f32", 8),
    (160, 8192, "rms", "bf16", "bf16", "f32", False, 0, "f32", 0),
    (160, 8200, "layer", "bf16", "bf16", "f32", True, 160, "bf16", 0),
    (90, 16384, "layer", "f32", "bf16", "bf16", True, 3, "f32", 0),
    (700, 768, "layer", "f32", "bf16", "f32", True, 7, "f32", 0),
    (1300, 1536, "layer", "f32", "f32", "f32", False, 13, "f32", 0),
    (1000, 257, "rms", "bf16", "bf16", "f32", False, 8, "f32", 3),
    (650, 1777, "layer", "f32", "bf16", "f32", True, 13, "bf16", 1),
    (400, 3001, "layer", "bf16", "bf16", "bf16", True, 1, "bf16", 0),
    (2000, 40, "layer", "f32", "bf16", "f32", True, 20, "f32", 0),
    (5000, 96, "rms", "bf16", "bf16", "f32", False, 0, "f32", 0),
    (0, 64, "rms", "bf16", "bf16", "f32", False, 0, "f32", 0),
]


@pytest.mark.parametrize("rows,d,norm,stream,branch,weights,bias,gate,gate_kind,extra", CASES)
def test_forward_and_backward(P, rows, d, norm, stream, branch, weights, bias, gate, gate_kind, extra):
    s = inputs(rows, d, stream, branch, weights, bias, gate, gate_kind, extra, seed=rows + d)
    a = 0.875
    rest = {k: s.get(k) for k in ("post_bias", "pre_bias", "gate")}
    y, h, stats = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"], **rest, residual_scale=a,
                                      eps=EPS, norm=norm, save=True)
    if rows == 0:
        assert y.shape == h.shape == (0, d)
    want_y, want_h, _ = definition(s, norm, a)
    near(y, want_y, ("y", y.dtype))
    # a row of few columns may have a deviation far below its values: what y's own rounding leaves is divided by it
    spread = want_y - (want_y.mean(1, keepdim=True) if norm == "layer" else 0)
    lost = want_y.abs().amax(1, keepdim=True) / torch.sqrt((spread ** 2).mean(1, keepdim=True) + EPS) if rows else 1.0
    near(h, want_h, ("h", h.dtype), scale=(want_h.abs().amax(1, keepdim=True) + lost) if rows else None)
    for dy in (s["dy"], None):
        got = P.peri_norm_backward(s["dh"], dy, y, s["f"], stats, s["post_weight"], s["pre_weight"], **rest,
                                   residual_scale=a, norm=norm)
        check_gradients(got, {**s, "dy": dy}, y, stats, norm, a)


def check_gradients(got, s, y, stats, norm, a):
    """Against the formulas in 64 bits, on what backward is given (y as stored, stats)."""
    dbl = lambda t: t.double().cpu()  # noqa: E731
    rows, d = s["f"].shape
    st = dbl(stats)
    (mf, rf), (my, ry) = ((k[:, :1], k[:, 1:]) for k in st)
    dh, f, yy = dbl(s["dh"]), dbl(s["f"]), dbl(y)
    dy = torch.zeros_like(yy) if s["dy"] is None else dbl(s["dy"])
    n_y, n_f = (yy - my) * ry, (f - mf) * rf
    gate = dbl(s["gate"]).repeat_interleave(rows // s["gate"].shape[0], 0) if "gate" in s else torch.ones_like(f)
    layer = norm == "layer"

    def through(q, n, r):
        back = q - n * (q * n).mean(1, keepdim=True) - (q.mean(1, keepdim=True) if layer else 0.0)
        return back * r, q.abs().amax(1, keepdim=True) * r * (1 + n.abs().amax(1, keepdim=True) ** 2) if rows else q
    back, size = through(dh * dbl(s["pre_weight"]), n_y, ry)
    total = dy + back
    size = size + dy.abs().amax(1, keepdim=True) if rows else size
    near(got["x"], a * total, ("x", got["x"].dtype), scale=size)
    dz = total * gate
    df, dsize = through(dz * dbl(s["post_weight"]), n_f, rf)
    if rows:
        reach = (gate.abs() * dbl(s["post_weight"]).abs()).amax(1, keepdim=True)
        dsize = size * reach * rf * (1 + n_f.abs().amax(1, keepdim=True) ** 2)
    near(got["f"], df, ("f", got["f"].dtype), scale=dsize)
    sums = {"pre_weight": dh * n_y, "post_weight": dz * n_f}
    mags = {"pre_weight": dh.abs() * n_y.abs(), "post_weight": size * gate.abs() * n_f.abs()}
    if "post_bias" in s:
        sums |= {"pre_bias": dh, "post_bias": dz}
        mags |= {"pre_bias": dh.abs(), "post_bias": size * gate.abs()}
    for k, t in sums.items():
        near(got[k], t.sum(0), (k, got[k].dtype), scale=mags[k].sum(0) if rows else None)
    if "gate" in s:
        z = n_f * dbl(s["post_weight"]) + (dbl(s["post_bias"]) if "post_bias" in s else 0.0)
        groups = s["gate"].shape[0]
        each = lambda t: t.view(groups, rows // groups, d).sum(1)  # noqa: E731
        near(got["gate"], each(total * z), ("gate", got["gate"].dtype), scale=each(size * z.abs()))
    assert set(got) == {"x", "f", "post_weight", "pre_weight"} | ({"post_bias", "pre_bias"} if "post_bias" in s else set()) \
        | ({"gate"} if "gate" in s else set())


@pytest.mark.parametrize("norm,bias,gate", [("rms", False, 0), ("layer", True, 1), ("layer", False, 4), ("rms", False, 12)])
def test_autograd(P, norm, bias, gate):
    """peri_norm under autograd against the definition differentiated by torch on the
    CPU in 64 bits, three-dimensional inputs."""
    s = inputs(12, 160, "f32", "f32", "f32", bias, gate, seed=3)
    leaf = {k: v.clone().requires_grad_() for k, v in s.items() if k not in ("dy", "dh")}
    shape = (3, 4, 160)
    y, h = P.peri_norm(leaf["x"].view(shape), leaf["f"].view(shape), leaf["post_weight"], leaf["pre_weight"],
                       post_bias=leaf.get("post_bias"), pre_bias=leaf.get("pre_bias"), gate=leaf.get("gate"),
                       residual_scale=0.5, eps=EPS, norm=norm)
    assert y.shape == h.shape == shape
    ((y * s["dy"].view(shape)).sum() + (h * s["dh"].view(shape)).sum()).backward()
    _, _, want = definition(s, norm, 0.5)
    for k, g in want.items():
        near(leaf[k].grad, g, (k, torch.float32), scale=g.abs().max() * 10)


def test_gradients_against_differences(P):
    """Directional central differences of the forward pass in fp32: with a step of 1e-2 and outputs of
    size 1 the difference carries 2^-24 / 1e-2 * sqrt(n) of rounding and 1e-4 of curvature: 2e-3 of the
    directional derivative's scale."""
    s = inputs(6, 200, "f32", "f32", "f32", True, 2, seed=5)
    names = [k for k in s if k not in ("dy", "dh")]

    def loss(v):
        y, h, _ = P.peri_norm_forward(v["x"], v["f"], v["post_weight"], v["pre_weight"], post_bias=v["post_bias"],
                                      pre_bias=v["pre_bias"], gate=v["gate"], residual_scale=0.75, eps=EPS, norm="layer")
        return float((y.double() * s["dy"].double()).sum() + (h.double() * s["dh"].double()).sum())
    y, h, stats = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"], post_bias=s["post_bias"],
                                      pre_bias=s["pre_bias"], gate=s["gate"], residual_scale=0.75, eps=EPS, norm="layer", save=True)
    g = P.peri_norm_backward(s["dh"], s["dy"], y, s["f"], stats, s["post_weight"], s["pre_weight"], post_bias=s["post_bias"],
                             pre_bias=s["pre_bias"], gate=s["gate"], residual_scale=0.75, norm="layer")
    gen = torch.Generator(device="cuda").manual_seed(1)
    for k in names:
        along = torch.randn(s[k].shape, device="cuda", generator=gen)
        step = 1e-2
        ends = [loss({**s, k: s[k] + sign * step * along}) for sign in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * step)
        want = float((g[k].double() * along.double()).sum())
        scale = float(g[k].double().norm() * along.double().norm()) / np.sqrt(along.numel())
        assert abs(slope - want) <= 2e-3 * scale * 5, (k, slope, want, scale)


def test_rows_that_are_not_finite_stay_apart(P):
    """A NaN or an infinity in one row reaches that row's outputs only."""
    s = inputs(9, 300, "f32", "f32", seed=2)
    clean = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"])
    s["f"][3, 5], s["x"][6, 7] = float("nan"), float("inf")
    y, h, _ = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"])
    keep = [i for i in range(9) if i not in (3, 6)]
    assert torch.equal(y[keep], clean[0][keep]) and torch.equal(h[keep], clean[1][keep])
    assert torch.isnan(y[3]).all() and torch.isnan(h[3]).all()
    assert torch.isinf(y[6, 7]) and torch.isnan(h[6, 7])


def test_zero_rows_of_input(P):
    """An all-zero f (a masked token): its norm is 0, the gradients finite."""
    s = inputs(4, 128, "bf16", "bf16", "f32", seed=4)
    s["f"].zero_(), s["x"][1].zero_()
    y, h, stats = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"], save=True)
    assert torch.equal(y, s["x"]) and not h[1].any() and torch.isfinite(h).all()
    g = P.peri_norm_backward(s["dh"], s["dy"], y, s["f"], stats, s["post_weight"], s["pre_weight"])
    assert all(torch.isfinite(t).all() for t in g.values())


def test_equal_calls_give_equal_bits(P):
    s = inputs(3001, 520, "bf16", "bf16", "f32", True, 1, seed=6)
    args = dict(post_bias=s["post_bias"], pre_bias=s["pre_bias"], gate=s["gate"], norm="layer")
    y, h, stats = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"], **args, save=True)
    one, two = (P.peri_norm_backward(s["dh"], s["dy"], y, s["f"], stats, s["post_weight"], s["pre_weight"], **args)
                for _ in range(2))
    assert all(torch.equal(one[k], two[k]) for k in one)


def test_another_stream(P):
    side = torch.cuda.Stream()
    s = inputs(2048, 768, "bf16", "bf16", seed=7)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = s["x"] * 2
        y, h, _ = P.peri_norm_forward(x, s["f"], s["post_weight"], s["pre_weight"])
    side.synchronize()
    want, _, _ = definition({**s, "x": s["x"] * 2}, "rms", 1.0)
    near(y, want, ("y", y.dtype))


def test_refusals(P):
    s = inputs(4, 64, "bf16", "bf16", "f32", True, 2, seed=1)
    x, f, w, q = s["x"], s["f"], s["post_weight"], s["pre_weight"]
    y, h, stats = P.peri_norm_forward(x, f, w, q, save=True)
    for bad in (dict(gate=s["gate"][:, :63].contiguous()), dict(gate=torch.ones(3, 64, device="cuda")), dict(norm="batch"),
                dict(post_bias=s["post_bias"].double(), pre_bias=s["pre_bias"]), dict(gate=s["gate"].double())):
        with pytest.raises(ValueError):
            P.peri_norm_forward(x, f, w, q, **bad)
    for bad in (dict(post_bias=s["post_bias"]), dict(eps=-1.0), dict(residual_scale=float("nan"))):
        with pytest.raises(P.MTDAOError) as e:
            P.peri_norm_forward(x, f, w, q, **bad)
        assert e.value.code == P.ERR_INVALID
    for args in ((x[:3], f, w, q), (x, f.half(), w, q), (x.cpu(), f.cpu(), w, q), (x, f, w[:60], q), (x, f, w.bfloat16(), q),
                 (x.t().contiguous().t(), f, w, q)):
        with pytest.raises(ValueError):
            P.peri_norm_forward(*args)
    with pytest.raises(P.MTDAOError):                   # a bf16 stream with an fp32 branch
        P.peri_norm_forward(x, f.float(), w, q)
    wide = torch.zeros(2, P.PERI_NORM_MAX_D + 1, device="cuda")
    with pytest.raises(P.MTDAOError):
        P.peri_norm_forward(wide, wide, wide[0], wide[0])
    for args in ((s["dh"].float(), s["dy"], y, f, stats), (s["dh"], s["dy"][:2], y, f, stats), (s["dh"], None, y, f, stats[:1])):
        with pytest.raises(ValueError):
            P.peri_norm_backward(*args, w, q)
    shape = P.mtdao_peri_norm(4, 64, 0, 1, 1, 0, 0, 0, 1e-5, 1.0, *([64] * 8))
    a = [t.data_ptr() for t in (s["dh"], s["dy"], y, f, stats, w)]
    need = P.mtdao_peri_norm_workspace(shape)
    if need:
        with pytest.raises(P.MTDAOError):
            P.mtdao_peri_norm_backward(shape, *a, None, q.data_ptr(), None, x.data_ptr(), h.data_ptr(), w.data_ptr(), None,
                                       q.data_ptr(), None, None, stats.data_ptr(), need - 1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("d", [8, 72, 136, 257, 264, 520, 776, 1001, 1032, 1777, 1544, 2056, 4104, 5120, 6152, 8200])
@pytest.mark.parametrize("stream,branch", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
def test_columns_past_the_end_hold_nothing(P, d, stream, branch):
    """Threads past a row's last column: NaN that longer rows left in their place on chip does not reach a result."""
    whole = 1 << (d - 1).bit_length()
    for norm, bias, gate in (("layer", True, 304), ("rms", False, 304), ("rms", False, 4)):
        s = inputs(304, d, stream, branch, "f32", bias, gate, "bf16", seed=d)
        bad = inputs(304, whole, stream, branch, "f32", bias, gate, "bf16", seed=d)
        bad = {k: torch.full_like(v, float("nan")) for k, v in bad.items()}
        results = []
        for use in (s, bad, s):
            rest = {k: use.get(k) for k in ("post_bias", "pre_bias", "gate")}
            y, h, stats = P.peri_norm_forward(use["x"], use["f"], use["post_weight"], use["pre_weight"], **rest, norm=norm,
                                              save=True)
            g = P.peri_norm_backward(use["dh"], use["dy"], y, use["f"], stats, use["post_weight"], use["pre_weight"], **rest,
                                     norm=norm)
            results.append({"y": y, "h": h, "stats": stats, **g})
        for k, v in results[0].items():
            assert torch.isfinite(v).all(), (norm, k)
            assert torch.equal(v, results[2][k]), (norm, k)


@pytest.mark.parametrize("rows,d,stream,branch", [(400, 3001, "bf16", "bf16"), (300, 1024, "f32", "bf16"), (65, 6144, "f32", "f32")])
def test_gate_of_every_element_with_biases(P, rows, d, stream, branch):
    """The gate's gradient dY (post_weight n_f + post_bias) where the two terms may cancel: the bound goes by their magnitudes."""
    s = inputs(rows, d, stream, branch, branch, True, rows, branch, seed=rows + d)
    rest = {k: s[k] for k in ("post_bias", "pre_bias", "gate")}
    y, _, stats = P.peri_norm_forward(s["x"], s["f"], s["post_weight"], s["pre_weight"], **rest, norm="layer", save=True)
    got = P.peri_norm_backward(s["dh"], s["dy"], y, s["f"], stats, s["post_weight"], s["pre_weight"], **rest, norm="layer")["gate"]
    dbl = lambda t: t.double().cpu()  # noqa: E731
    (mf, rf), (my, ry) = ((k[:, :1], k[:, 1:]) for k in dbl(stats))
    n_y, n_f = (dbl(y) - my) * ry, (dbl(s["f"]) - mf) * rf
    u = dbl(s["dh"]) * dbl(s["pre_weight"])
    total = dbl(s["dy"]) + (u - n_y * (u * n_y).mean(1, keepdim=True) - u.mean(1, keepdim=True)) * ry
    size = u.abs().amax(1, keepdim=True) * ry * (1 + n_y.abs().amax(1, keepdim=True) ** 2) + dbl(s["dy"]).abs().amax(1, keepdim=True)
    term, bias = n_f * dbl(s["post_weight"]), dbl(s["post_bias"])
    near(got, total * (term + bias), ("gate", got.dtype), scale=size * (term.abs() + bias.abs()))
