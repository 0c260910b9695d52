"""AdamW on lists long enough for the records that are streamed four blocks at a
time, in every pair of types and alignment, and averages over more replicas than
a warp has lanes.  The reference and its tolerances are those of
test_gpu_adamw.py: 8-bit codes bit for bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import adamw_reference as R
from test_gpu_adamw import BETAS, EPS, SEED, check_params, held, inside, make, padded, per_tensor

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2510_05361_gb300 as P
    P.load()
    return P


NUMELS = [10000019, 8192 * 3, 513, 255, 4096 + 7]


@pytest.mark.parametrize("pdt,gdt,shift", [("bf16", "bf16", 0), ("bf16", "bf16", 1), ("bf16", "bf16", 4), ("f32", "f32", 0),
                                           ("f32", "f32", 4), ("f32", "bf16", 3), ("bf16", "f32", 2), ("mixed", "mixed", 0),
                                           ("mixed", "bf16", 7)])
def test_a_step_of_a_long_list(P, pdt, gdt, shift):
    params, grads = make(NUMELS, 1, pdt, gdt, shift, seed=shift)
    opt = P.AdamW(params, grads, betas=BETAS, eps=EPS, state_bits=8, seed=SEED)
    opt.step(1e-3)                                   # states that are not zero
    mask = inside(NUMELS)
    bf16 = per_tensor(NUMELS, [t.dtype == torch.bfloat16 for t in params[0]]).astype(bool)
    p0, g0 = padded(params[0], NUMELS), padded(grads[0], NUMELS)
    m0, v0 = held(opt, "m")[0][0], held(opt, "v")[0][0]
    opt.step(1e-3, weight_decay=0.1)
    torch.cuda.synchronize()
    want, _, _ = R.update64(p0, g0, m0, v0, 1, 1e-3, 0.1, BETAS, EPS)
    check_params(padded(params[0], NUMELS), want, p0, 1 - 1e-4, mask, bf16)
    low, high = R.words(SEED, 1, 0, mask.size)
    g32 = g0.astype(np.float32)
    for name, old, target, word in (("m", m0, g32, low), ("v", v0, g32 * g32, high)):
        codes, scales = R.hold(R.ema32(BETAS[name == "v"], old.astype(np.float32), target), name, word)
        _, got, got_scales = held(opt, name)
        assert np.array_equal(got_scales[0], scales) and np.array_equal(got[0], codes), name
    opt.close()


def test_a_clipped_step_of_a_long_list_follows_the_norm(P):
    params, grads = make(NUMELS, 1, "bf16", "bf16", 0, seed=5)
    norm = np.sqrt(sum(float(t.double().square().sum()) for t in grads[0]))
    opt = P.AdamW(params, grads, state_bits=8, seed=SEED)
    opt.step(1e-3, max_norm=0.01 * norm)
    torch.cuda.synchronize()
    m, g = held(opt, "m")[0][0], padded(grads[0], NUMELS)
    want = 0.1 * 0.01 * g
    blocks = np.abs(want).reshape(-1, 256).max(1).repeat(256)
    # a code is at most 1/8 of the value off, or one step of the smallest codes (2^-9 of a scale, 2^-7 to 2^-8 of the block's largest)
    assert np.all(np.abs(m - want) <= 0.126 * np.abs(want) + 2.0 ** -16 * blocks)
    assert abs(m.sum() - want.sum()) <= 5 * 0.125 * np.sqrt((want ** 2).sum())
    opt.close()


@pytest.mark.parametrize("M,pdt,numels,shift", [(3, "bf16", [3500003, 700], 1), (3, "f32", [3500003, 700], 4), (40, "bf16", [300001], 0),
                                                (40, "f32", [300001, 17], 1), (2, "mixed", [5300000, 300000], 0)])
def test_average_of_long_lists_and_many_replicas(P, M, pdt, numels, shift):
    params, grads = make(numels, M, pdt, "f32", shift, seed=M)
    opt = P.AdamW(params, grads, state_bits=8, seed=3)
    opt.step(1e-2)
    p0 = np.stack([padded(r, numels) for r in params])
    before = {k: held(opt, k)[0] for k in "mv"}
    opt.average()
    torch.cuda.synchronize()
    mask = inside(numels)
    bf16 = per_tensor(numels, [t.dtype == torch.bfloat16 for t in params[0]]).astype(bool)
    want, size = p0.mean(0), np.abs(p0).max(0)
    tol = 4 * 2.0 ** -24 * size + np.where(bf16, 2.0 ** -8 * 1.001 * np.abs(want), 0.0)
    for r in (0, 1, M - 1):
        assert np.all((np.abs(padded(params[r], numels) - want) <= tol)[mask])
    for k in "mv":
        got, codes, scales = held(opt, k)
        assert np.array_equal(got, np.broadcast_to(got[:1], got.shape))
        w = before[k].mean(0)
        table, top, _ = R.FORMATS[k]
        both = [R.block_scales(w * (1 + d), top) for d in (-1e-6, 0.0, 1e-6)]
        assert np.all((scales[0] == both[0]) | (scales[0] == both[1]) | (scales[0] == both[2]))
        per = np.repeat(scales[0], R.BLOCK)
        y = np.divide(w, per, out=np.zeros_like(w), where=per > 0)
        if k == "v":
            y = np.where(per > 0, np.maximum(y, 2.0 ** -16), y)
        assert np.all((codes[0] == R.nearest(y * (1 - 1e-6), table)) | (codes[0] == R.nearest(y * (1 + 1e-6), table)))
    opt.close()


def test_average_with_values_that_are_not_finite(P):
    """A parameter's infinity in one replica makes the mean infinite, infinities of both
    signs or a NaN make it NaN, as the sum of the values does; neighbours are not touched."""
    M, n = 3, 4000
    params = [[torch.full((n,), 1.0 + r, device="cuda")] for r in range(M)]
    params[1][0][5] = float("inf")
    params[0][0][6], params[2][0][6] = float("inf"), float("-inf")
    params[2][0][7] = float("nan")
    params[0][0][8], params[1][0][8], params[2][0][8] = 3e38, -3e38, 3e38
    opt = P.AdamW(params, state_bits=8)
    opt.average(P.adamw.PARAMS)
    torch.cuda.synchronize()
    for r in range(M):
        p = params[r][0]
        assert p[5] == float("inf") and torch.isnan(p[6]) and torch.isnan(p[7]) and torch.isfinite(p[8])
        rest = torch.cat([p[:5], p[9:]])
        assert (rest == 2.0).all()
    opt.close()


def test_average_of_bf16_parameters_that_are_not_finite(P):
    M, n = 3, 4000
    params = [[torch.full((n,), 1.0 + r, device="cuda", dtype=torch.bfloat16)] for r in range(M)]
    params[1][0][5] = float("inf")
    params[0][0][6], params[2][0][6] = float("inf"), float("-inf")
    params[2][0][7] = float("nan")
    opt = P.AdamW(params, state_bits=8)
    opt.average(P.adamw.PARAMS)
    torch.cuda.synchronize()
    for r in range(M):
        p = params[r][0]
        assert p[5] == float("inf") and torch.isnan(p[6]) and torch.isnan(p[7])
        assert (p[:5] == 2.0).all() and (p[8:] == 2.0).all()
    opt.close()
