"""The example that trains a small Peri-LN network with the operators together:
the loss falls, the workers agree bit for bit after an average, the padding of
their state vectors holds nothing, 8-bit states train about as well as 32-bit
ones."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "local_adamw.py")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("local_adamw_example", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_workers_train_and_agree(example, dtype):
    steps = 160                                   # a multiple of the period: the last step is averaged
    ends = {}
    for bits in (8, 32):
        before, after, params, opt = example.train(workers=3, steps=steps, period=16, state_bits=bits, dtype=dtype)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for row in params[1:] for a, b in zip(row, params[0]))
        assert after < 0.7 * before, (bits, before, after)
        ends[bits] = after
        m = opt.state("m")
        codes = (m["codes"].float() if bits == 8 else m)
        at = 0
        for k in opt.numels:
            pad = -k % 256
            assert not codes[:, at + k:at + k + pad].any()
            at += k + pad
        opt.close()
    assert abs(ends[8] - ends[32]) < 0.1 * ends[32], ends


def test_the_same_run_gives_the_same_bits(example):
    one = example.train(workers=2, steps=20, period=8)
    two = example.train(workers=2, steps=20, period=8)
    assert all(torch.equal(a, b) for r, s in zip(one[2], two[2]) for a, b in zip(r, s))
    assert one[:2] == two[:2]
