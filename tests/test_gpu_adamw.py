"""AdamW on tensor lists (m and v in 32 or 8 bits) against its formulas in numpy.

Tolerances.  8-bit states: m and v before they are held are one fp32 rounding
after each operation of the formula, so the codes and scales of the reference
have to be met bit for bit (with clipping, where the factor's last bit may
differ, one code step apart at most).  32-bit states: four roundings of
2^-24.  Parameters: p' = p keep - u with |u| = lr |m^| / (v^ + eps): the
product, the sum and p's own rounding leave 3 * 2^-24 of |p| + |u|, the square
root, the quotient and the scalars 8 * 2^-23 of |u|; bf16 adds one step
(2^-7 of the value: rounding up or down is random), checked on its mean too.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import adamw_reference as R

pytestmark = pytest.mark.gpu

BETAS, EPS, SEED = (0.9, 0.999), 1e-8, 77
LISTS = {"one": [1], "few": [3, 8, 0, 5], "blocks": [255, 256, 257, 2048, 2049], "long": [70001, 4096, 1, 513]}


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2510_05361_gb300 as P
    P.load()
    return P


def cut(flat, numels, shift):
    """Tensors of the given sizes from one vector, each ``shift`` elements off alignment."""
    out, at = [], 0
    for k in numels:
        out.append(flat[at + shift:at + shift + k])
        at += -(-(k + shift) // 64) * 64
    return out


def make(numels, M, pdt, gdt, shift=0, seed=0, sigma=1e-2):
    """M lists of parameters and of gradients; dtypes alternate for "mixed"."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    total = sum(-(-(k + shift) // 64) * 64 for k in numels) + 64

    def lists(kind, scale):
        kinds = [{"f32": torch.float32, "bf16": torch.bfloat16}[kind] if kind != "mixed"
                 else (torch.float32, torch.bfloat16)[i % 2] for i in range(len(numels))]
        rows = []
        for _ in range(M):
            pools = {k: torch.randn(total, device="cuda", generator=gen).mul_(scale).to(k) for k in set(kinds)}
            parts = {k: cut(pools[k], numels, shift) for k in pools}
            rows.append([parts[k][i] for i, k in enumerate(kinds)])
        return rows
    return lists(pdt, 0.02), lists(gdt, sigma)


def padded(row, numels):
    offs, n = R.state_offsets(numels)
    out = np.zeros(n)
    for at, k, t in zip(offs, numels, row):
        out[at:at + k] = t.detach().double().cpu().numpy().reshape(-1)
    return out


def inside(numels):
    offs, n = R.state_offsets(numels)
    mask = np.zeros(n, bool)
    for at, k in zip(offs, numels):
        mask[at:at + k] = True
    return mask


def held(opt, name):
    """(values, codes' values, scales) of a state as fp64 arrays [M][...]."""
    s = opt.state(name)
    if opt.state_bits == 32:
        return s.double().cpu().numpy(), None, None
    codes, scales = s["codes"].double().cpu().numpy(), s["scales"].double().cpu().numpy()
    return codes * np.repeat(scales, R.BLOCK, axis=1), codes, scales


def check_params(got, want, p0, keep, mask, bf16):
    u = np.abs(p0 * keep - want)
    tol = 3 * 2.0 ** -24 * (np.abs(p0) + u) + 8 * 2.0 ** -23 * u
    if bf16 is not None:
        tol = tol + np.where(bf16, 2.0 ** -7 * (np.abs(want) + tol), 0.0)
    bad = mask & ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.flatnonzero(bad)[:5], got[bad][:5], want[bad][:5])


def per_tensor(numels, values):
    offs, n = R.state_offsets(numels)
    out = np.zeros(n, type(values[0]) if values else float)
    for at, k, x in zip(offs, numels, values):
        out[at:at + -(-k // R.BLOCK) * R.BLOCK] = x
    return out


@pytest.mark.parametrize("shape", list(LISTS))
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("pdt,gdt,M,shift,clip", [
    ("f32", "f32", 1, 0, None), ("bf16", "bf16", 3, 0, 0.1), ("f32", "bf16", 2, 1, 1e6),
    ("bf16", "f32", 1, 3, 0.1), ("mixed", "mixed", 2, 8, None)])
def test_steps_match_the_formulas(P, shape, bits, pdt, gdt, M, shift, clip):
    numels = LISTS[shape]
    params, grads = make(numels, M, pdt, gdt, shift, seed=len(numels) + M)
    decay = [float(i % 2) for i in range(len(numels))]
    opt = P.AdamW(params, grads, betas=BETAS, eps=EPS, state_bits=bits, decay=decay, seed=SEED)
    mask, lr, wd = inside(numels), 1e-3, 0.1
    dec = per_tensor(numels, decay)
    bf16 = per_tensor(numels, [t.dtype == torch.bfloat16 for t in params[0]]).astype(bool)
    for step in range(3):
        for row in grads:
            for t in row:
                t.mul_(-0.7)
        p0 = [padded(r, numels) for r in params]
        g0 = [padded(r, numels) for r in grads]
        m0, v0 = held(opt, "m")[0], held(opt, "v")[0]
        opt.step(lr, weight_decay=wd, max_norm=clip)
        torch.cuda.synchronize()
        m1, v1 = held(opt, "m"), held(opt, "v")
        for r in range(M):
            s = 1.0 if clip is None else min(1.0, clip / (np.sqrt(np.sum(g0[r] ** 2)) + 1e-6))
            g = g0[r] * s
            keep = 1 - lr * wd * dec
            want, m64, v64 = R.update64(p0[r], g, m0[r], v0[r], step, lr, wd * dec, BETAS, EPS)
            check_params(padded(params[r], numels), want, p0[r], keep, mask, bf16)
            if bits == 32:
                for got, w64, old, new in ((m1[0][r], m64, m0[r], g), (v1[0][r], v64, v0[r], g * g)):
                    assert np.all(np.abs(got - w64) <= 4 * 2.0 ** -24 * (np.abs(old) + np.abs(new)))
                continue
            g32 = (g0[r].astype(np.float32) * np.float32(s))
            low, high = R.words(SEED, step, r, mask.size)
            for name, old, target, word, got in (("m", m0[r], g32, low, m1), ("v", v0[r], g32 * g32, high, v1)):
                codes, scales = R.hold(R.ema32(BETAS[name == "v"], old.astype(np.float32), target), name, word)
                if clip is None or s == 1.0:
                    assert np.array_equal(got[2][r], scales), name
                    assert np.array_equal(got[1][r], codes), name
                else:                      # one step either way: the next code up is at most 1/8 (m), 1/4 (v) larger
                    assert np.allclose(got[2][r], scales, rtol=1e-5), name
                    near = 0.125 if name == "m" else 0.25
                    assert np.all(np.abs(got[1][r] - codes) <= near * np.maximum(np.abs(codes), np.abs(got[1][r]))
                                  + R.FORMATS[name][0][1])
                    assert np.mean(got[1][r] != codes) < 0.01
    assert opt.t == 3
    opt.close()


def test_stochastic_rounding_keeps_the_mean(P):
    """v decays by 0.1 % a step when gradients stop, m by 0.1 % too with beta = 0.999:
    to nearest, neither would ever leave its code.  Over n elements and T steps the mean
    moves by (1 - 1e-3)^T; a step's rounding adds at most half a code's distance (1/8 of a value for
    m, 1/4 for v), independent between elements, so the mean of n is off by
    at most 0.25 sqrt(T / n) of the values' size at one standard deviation."""
    n, T = 1 << 16, 100
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, device="cuda")
    opt = P.AdamW([p], [g], betas=(0.999, 0.999), state_bits=8, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(1)
    g.copy_(torch.rand(n, device="cuda", generator=gen) + 0.5)
    opt.step(0.0)
    before = [held(opt, k)[0].mean() for k in "mv"]
    g.zero_()
    for _ in range(T):
        opt.step(0.0)
    torch.cuda.synchronize()
    for k, b in zip("mv", before):
        ratio = held(opt, k)[0].mean() / b
        assert abs(ratio - 0.999 ** T) < 5 * 0.25 * np.sqrt(T / n), (k, ratio)
    opt.close()


def test_bf16_parameters_move_by_less_than_a_step(P):
    """An update of 1e-4 on weights of 1 (bf16 step 2^-8 below, 2^-7 above): the mean follows it.
    The mean of n roundings, each at most 2^-7 off, is within 5 * 2^-7 * sqrt(T / n)."""
    n, T = 1 << 16, 20
    p = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    g = torch.full((n,), 0.3, device="cuda")
    opt = P.AdamW([p], [g], state_bits=32, seed=9)
    for _ in range(T):
        opt.step(1e-4)
    torch.cuda.synchronize()
    assert abs(float(p.double().mean()) - (1 - T * 1e-4)) < 5 * 2.0 ** -7 * np.sqrt(T / n)
    opt.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_zero_tiny_and_nonfinite_gradients(P, bits):
    """A list of three blocks: all zero; 1e-20 (v = 1e-43, below what 8 bits
    hold: zero); one NaN or infinity among ordinary values, which in 8 bits
    makes its whole block NaN and in 32 its element."""
    p = [torch.ones(256, device="cuda") for _ in range(4)]
    g = [torch.zeros(256, device="cuda"), torch.full((256,), 1e-20, device="cuda"),
         torch.full((256,), 0.5, device="cuda"), torch.full((256,), 0.5, device="cuda")]
    g[2][7] = float("nan")
    g[3][9] = float("inf")
    opt = P.AdamW(p, g, state_bits=bits, seed=1)
    for _ in range(2):
        opt.step(1e-3)
    torch.cuda.synchronize()
    m, v = held(opt, "m")[0].reshape(4, 256), held(opt, "v")[0].reshape(4, 256)
    assert torch.equal(p[0], torch.ones_like(p[0])) and not m[0].any() and not v[0].any()
    assert torch.isfinite(p[1]).all() and (p[1] == 1.0).all()          # eps outweighs 1e-20
    for k, at in ((2, 7), (3, 9)):
        odd = ~np.isfinite(m[k]) | ~np.isfinite(v[k])
        if bits == 8:
            assert odd.all()
        else:
            assert odd[at] and odd.sum() == 1
            rest = torch.cat([p[k][:at], p[k][at + 1:]])
            assert torch.isfinite(rest).all()
    assert not torch.isfinite(p[2][7])
    opt.close()


@pytest.mark.parametrize("gdt", ["f32", "bf16"])
def test_gradient_norm(P, gdt):
    """Sums over several tensors, of gradients whose squares fp32 does not hold among them:
    2^-20 relative is far above the compensated sums' error."""
    numels = [5000, 1, 0, 2049]
    params, grads = make(numels, 3, "f32", gdt, 1, seed=4, sigma=3.0)
    for scale in (1.0, 1e25, 1e-25):
        for row in grads:
            for t in row:
                t.mul_(scale)
        opt = P.AdamW(params, grads)
        got = opt.grad_sqnorm().cpu().numpy()
        want = np.array([sum(float(t.double().square().sum()) for t in row) for row in grads])
        assert np.all(np.abs(got - want) <= 2.0 ** -20 * want), (got, want)
        opt.close()
        for row in grads:
            for t in row:
                t.div_(scale)


def test_clip_of_zero_and_huge_gradients(P):
    p, g = [torch.ones(300, device="cuda")], [torch.zeros(300, device="cuda")]
    opt = P.AdamW(p, g, state_bits=8)
    opt.step(1e-3, max_norm=1.0)
    assert (p[0] == 1.0).all()
    g[0].fill_(1e30)                              # norm 1.7e31: clipped to 1
    opt.step(1e-3, max_norm=1.0)
    m = held(opt, "m")[0][0, :300]
    assert np.all(np.abs(m - 0.1 / np.sqrt(300)) <= 0.125 * 0.1 / np.sqrt(300))
    opt.close()


@pytest.mark.parametrize("M", [2, 3, 5, 8, 17])
@pytest.mark.parametrize("bits,pdt", [(8, "bf16"), (8, "f32"), (32, "f32"), (32, "bf16"), (8, "mixed")])
def test_average(P, M, bits, pdt):
    """Means of all quantities, and of some; the 8-bit result is the mean's
    nearest code (the mean of a few codes is exact in fp32 or off by an ulp)."""
    numels = [700, 3, 2100, 0, 256]
    params, grads = make(numels, M, pdt, "f32", 1, seed=M)
    opt = P.AdamW(params, grads, state_bits=bits, seed=3)
    for _ in range(2):
        opt.step(1e-2)
    mask = inside(numels)
    p0 = np.stack([padded(r, numels) for r in params])
    before = {k: held(opt, k)[0] for k in "mv"}
    opt.average(P.adamw.PARAMS | P.adamw.V_STATE)
    assert np.array_equal(held(opt, "m")[0], before["m"])
    opt.average(P.adamw.M_STATE)
    torch.cuda.synchronize()
    bf16 = per_tensor(numels, [t.dtype == torch.bfloat16 for t in params[0]]).astype(bool)
    want = p0.mean(0)
    size = np.abs(p0).max(0)
    for r in range(M):
        got = padded(params[r], numels)
        tol = 4 * 2.0 ** -24 * size + np.where(bf16, 2.0 ** -8 * 1.001 * np.abs(want), 0.0)
        assert np.all(np.abs(got - want)[mask] <= tol[mask])
    for k in "mv":
        got, codes, scales = held(opt, k)
        assert np.array_equal(got, np.broadcast_to(got[:1], got.shape))
        w = before[k].mean(0)
        if bits == 32:
            assert np.all(np.abs(got[0] - w) <= 4 * 2.0 ** -24 * np.abs(before[k]).max(0))
            continue
        table, top, _ = R.FORMATS[k]
        scale = R.block_scales(w * (1 + 1e-7) if k == "v" else w, top)
        ok = np.isclose(scales[0], scale) | np.isclose(scales[0], R.block_scales(w * (1 - 1e-6), top)) \
            | np.isclose(scales[0], R.block_scales(w * (1 + 1e-6), top))
        assert ok.all()
        per = np.repeat(scales[0], R.BLOCK)
        y = np.divide(w, per, out=np.zeros_like(w), where=per > 0)
        if k == "v":
            y = np.where(per > 0, np.maximum(y, 2.0 ** -16), y)
        a, b = R.nearest(y * (1 - 1e-6), table), R.nearest(y * (1 + 1e-6), table)
        assert np.all((codes[0] == a) | (codes[0] == b))
    opt.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_average_of_equal_replicas_changes_nothing(P, bits):
    numels, M = [700, 2049], 3
    params, grads = make(numels, 1, "bf16", "f32", 0, seed=8)
    params = [[t.clone() for t in params[0]] for _ in range(M)]
    grads = [grads[0]] * M                               # gradients may be shared
    opt = P.AdamW(params, grads, state_bits=bits, seed=3)
    opt.step(1e-2)
    for name in "mv":                                     # the replicas' random numbers differ: make the states equal
        s = opt.state(name)
        for t in (s.values() if bits == 8 else [s]):
            t[1:].copy_(t[:1].expand_as(t[1:]))
    for r in range(1, M):
        for a, b in zip(params[r], params[0]):
            a.copy_(b)
    before = [held(opt, k)[0] for k in "mv"]
    p0 = [t.clone() for t in params[0]]
    opt.average()
    torch.cuda.synchronize()
    assert all(np.array_equal(held(opt, k)[0], b) for k, b in zip("mv", before))
    assert all(torch.equal(a, b) for r in range(M) for a, b in zip(params[r], p0))
    opt.close()


def test_equal_calls_give_equal_bits_and_resume(P):
    numels = [5000, 33]

    def run(resume):
        params, grads = make(numels, 2, "bf16", "bf16", 0, seed=6)
        opt = P.AdamW(params, grads, state_bits=8, seed=11)
        for t in range(4):
            if resume and t == 2:
                saved = [{k: x.clone() for k, x in opt.state(n).items()} for n in "mv"]
                opt.close()
                opt = P.AdamW(params, grads, state_bits=8, seed=11)
                for n, s in zip("mv", saved):
                    for k, x in opt.state(n).items():
                        x.view(torch.uint8).copy_(s[k].view(torch.uint8))
                opt.t = 2
            opt.step(1e-3, max_norm=0.5)
        torch.cuda.synchronize()
        out = [padded(r, numels) for r in params] + [held(opt, k)[0] for k in "mv"]
        opt.close()
        return out
    first = run(False)
    for other in (run(False), run(True)):
        assert all(np.array_equal(a, b) for a, b in zip(first, other))


def test_another_stream(P):
    numels = [300000]
    params, grads = make(numels, 1, "f32", "f32", 0, seed=2)
    side = torch.cuda.Stream()
    opt = P.AdamW(params, grads, state_bits=8, stream=side.cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        grads[0][0].mul_(3.0)                 # ordered before the step on the same stream
        g0, p0 = padded(grads[0], numels), padded(params[0], numels)
        opt.step(1e-3, max_norm=1.0)
    side.synchronize()
    s = 1.0 / (np.sqrt(np.sum(g0 ** 2)) + 1e-6)
    want, _, _ = R.update64(p0, g0 * min(1.0, s), 0 * p0, 0 * p0, 0, 1e-3, 0.0, BETAS, EPS)
    check_params(padded(params[0], numels), want, p0, 1.0, inside(numels), None)
    opt.close()


def test_new_gradients_are_bound(P):
    p, g = [torch.zeros(100, device="cuda")], [torch.ones(100, device="cuda")]
    opt = P.AdamW(p, g)
    opt.step(1e-3)
    opt.bind_grads([torch.full((100,), -1.0, device="cuda", dtype=torch.bfloat16)])
    opt.step(1e-3)
    torch.cuda.synchronize()
    m = opt.state("m")[0, :100]
    assert torch.allclose(m, torch.full_like(m, 0.9 * 0.1 - 0.1), atol=1e-8)
    opt.close()


def test_refusals(P):
    dev = {"device": "cuda"}
    p, g = [torch.zeros(64, **dev)], [torch.zeros(64, **dev)]
    for bad in ({"betas": (1.0, 0.9)}, {"betas": (0.9, -0.1)}, {"eps": 0.0}, {"eps": float("nan")}, {"state_bits": 16},
                {"decay": [float("inf")]}):
        with pytest.raises(P.MTDAOError) as e:
            P.AdamW(p, g, **bad)
        assert e.value.code == P.ERR_INVALID
    with pytest.raises(ValueError):
        P.AdamW(p, g, decay=[1.0, 1.0])
    for bad in ([torch.zeros(64)], [torch.zeros(64, dtype=torch.float16, **dev)], [torch.zeros((8, 16), **dev).t()],
                [torch.zeros(64, device="cuda"), torch.zeros(3)], []):
        with pytest.raises(ValueError):
            P.AdamW(bad)
    for bad in ([torch.zeros(63, **dev)], [torch.zeros(64)], [], [torch.zeros(128, **dev)[::2]]):
        with pytest.raises(ValueError):
            P.AdamW(p, bad)
    whole = torch.zeros(100, **dev)
    with pytest.raises(P.MTDAOError) as e:
        P.AdamW([whole[:60], whole[59:]])
    assert e.value.code == P.ERR_INVALID
    with pytest.raises(P.MTDAOError) as e:
        P.AdamW([whole[:60]], [whole[40:]])
    assert e.value.code == P.ERR_INVALID
    with pytest.raises(P.MTDAOError):
        P.AdamW([torch.zeros(0, **dev)])
    opt = P.AdamW(p)
    with pytest.raises(P.MTDAOError) as e:
        opt.step(1e-3)
    assert e.value.code == P.ERR_STATE
    opt.bind_grads(g)
    for bad in ((float("nan"), 0.0, None), (1e-3, -1.0, None), (1e-3, 0.0, float("inf"))):
        with pytest.raises(P.MTDAOError) as e:
            opt.step(bad[0], weight_decay=bad[1], max_norm=bad[2])
        assert e.value.code == P.ERR_INVALID
    with pytest.raises(ValueError):
        opt.step(1e-3, max_norm=0.0)
    with pytest.raises(P.MTDAOError):
        opt.average(8)
    with pytest.raises(P.MTDAOError):
        opt.t = -1
    assert opt.t == 0
    opt.close()
    with pytest.raises(P.MTDAOError):
        opt.step(1e-3)
