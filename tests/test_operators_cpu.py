"""AdamW and the Peri-LN update without a GPU: the checks that the library makes
before it touches a device, and the sizes that it states."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def P():
    from paper_2510_05361_gb300 import build
    build.build()
    import paper_2510_05361_gb300 as P
    P.load()
    return P


def config(P, beta1=0.9, beta2=0.999, eps=1e-8, bits=8, seed=0):
    return P.mtdao_adamw_config(beta1, beta2, eps, bits, seed)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("numels,M", [([1], 1), ([0, 5, 256, 257], 3), ([70000, 1], 8), ([123570432], 4)])
def test_memory_holds_the_states(P, bits, numels, M):
    """Two states of a byte or four an element, rounded up to blocks of 256 of one
    tensor, 4 bytes of scale a block and state in 8 bits; tables add under 2 % and some kilobytes."""
    blocks = sum(-(-k // P.ADAMW_BLOCK) for k in numels) * M
    held = blocks * (2 * 256 + 2 * 4 if bits == 8 else 2 * 256 * 4)
    got = P.mtdao_adamw_memory(config(P, bits=bits), M, numels)
    assert held <= got <= 1.02 * held + 65536 + 256 * M


@pytest.mark.parametrize("bad", [{"beta1": 1.0}, {"beta2": -0.1}, {"beta1": float("nan")}, {"eps": 0.0},
                                 {"eps": 1e-16}, {"bits": 4}])
def test_configurations_that_are_refused(P, bad):
    with pytest.raises(P.MTDAOError) as e:
        P.mtdao_adamw_memory(config(P, **bad), 2, [10])
    assert e.value.code == P.ERR_INVALID and P.mtdao_last_error(None)


@pytest.mark.parametrize("numels,M", [([], 1), ([0, 0], 1), ([-1], 1), ([1 << 41], 1), ([10], 0), ([10], 1025),
                                      ([1 << 39, 1 << 39, 1 << 39], 1), ([1 << 36], 1), ([1 << 34], 1024)])
def test_lists_that_are_refused(P, numels, M):
    with pytest.raises(P.MTDAOError) as e:
        P.mtdao_adamw_memory(config(P), M, numels)
    assert e.value.code == P.ERR_INVALID


def test_create_checks_before_it_touches_a_device(P):
    h = ctypes.c_void_p(7)
    one = (ctypes.c_int64 * 1)(10)
    cfg = config(P)
    assert P.lib.mtdao_adamw_create(None, 1, one, None, 1, None, None, ctypes.byref(h)) == P.ERR_INVALID
    assert not h.value
    assert P.lib.mtdao_adamw_create(ctypes.byref(cfg), 1, None, None, 1, None, None, ctypes.byref(h)) == P.ERR_INVALID
    assert P.lib.mtdao_adamw_create(ctypes.byref(cfg), 1, one, None, 1, None, None, None) == P.ERR_INVALID
    assert P.lib.mtdao_adamw_create(ctypes.byref(cfg), 1, one, None, 1, 0x1008, None, ctypes.byref(h)) == P.ERR_ALIGN
    bad = (ctypes.c_float * 1)(float("nan"))
    assert P.lib.mtdao_adamw_create(ctypes.byref(cfg), 1, one, bad, 1, None, None, ctypes.byref(h)) == P.ERR_INVALID


def test_null_handles_are_safe(P):
    lib = P.lib
    lib.mtdao_adamw_destroy(None)
    assert lib.mtdao_adamw_get_step(None) == -1
    for call in (lambda: lib.mtdao_adamw_step(None, 0.1, 0.0, 0.0), lambda: lib.mtdao_adamw_average(None, 7),
                 lambda: lib.mtdao_adamw_set_step(None, 0), lambda: lib.mtdao_adamw_set_stream(None, None),
                 lambda: lib.mtdao_adamw_bind_params(None, None, None), lambda: lib.mtdao_adamw_bind_grads(None, None, None),
                 lambda: lib.mtdao_adamw_grad_sqnorm(None, None), lambda: lib.mtdao_adamw_state(None, 0, None, None, None)):
        assert call() == P.ERR_INVALID


def shape(P, rows=8, d=64, norm=0, stream=1, branch=1, weight=0, gate=0, gate_rows=0, eps=1e-5, scale=1.0, ld=None):
    ld = [d] * 8 if ld is None else ld
    return P.mtdao_peri_norm(rows, d, norm, stream, branch, weight, gate, gate_rows, eps, scale, *ld)


@pytest.mark.parametrize("bad", [{"rows": -1}, {"d": 0}, {"d": 16385}, {"norm": 2}, {"stream": 2}, {"branch": -1}, {"weight": 5},
                                 {"stream": 1, "branch": 0}, {"eps": -1.0}, {"eps": float("inf")}, {"scale": float("nan")},
                                 {"gate_rows": 3}, {"gate_rows": -1}, {"gate_rows": 2, "gate": 9}, {"ld": [63] * 8}])
def test_peri_norm_descriptions_that_are_refused(P, bad):
    s = shape(P, **bad)
    with pytest.raises(P.MTDAOError) as e:
        P.mtdao_peri_norm_workspace(s)
    assert e.value.code == P.ERR_INVALID
    with pytest.raises(P.MTDAOError):
        P.mtdao_peri_norm_forward(s, *([0x10000] * 10))


def test_peri_norm_arguments_that_are_refused(P):
    s, a = shape(P), 0x10000                       # stand-ins for addresses, never read
    for args in ((a, a, a, a, a, None, None, a, a, None),      # one bias without the other
                 (a, a, a, None, a, None, a, a, a, None),      # a gate that the description lacks
                 (a, None, a, None, a, None, None, a, a, None)):
        with pytest.raises(P.MTDAOError) as e:
            P.mtdao_peri_norm_forward(s, *args)
        assert e.value.code == P.ERR_INVALID
    with pytest.raises(P.MTDAOError) as e:
        P.mtdao_peri_norm_forward(s, a + 1, a, a, None, a, None, None, a, a, None)
    assert e.value.code == P.ERR_ALIGN
    with pytest.raises(P.MTDAOError) as e:        # no workspace
        P.mtdao_peri_norm_backward(s, a, a, a, a, a, a, None, a, None, a, a, a, None, a, None, None, a, 0)
    assert e.value.code == P.ERR_INVALID
    P.mtdao_peri_norm_forward(shape(P, rows=0), *([None] * 10))           # no rows, nothing to do


@pytest.mark.parametrize("d", [1, 64, 100, 768, 1001, 2048, 4096, 8192, 16384])
@pytest.mark.parametrize("rows,gate_rows", [(1, 0), (7, 7), (4096, 1), (4096, 32), (65536, 16384)])
def test_workspace_is_small(P, d, rows, gate_rows):
    """Four vectors for each of the kernel's row sets and gate rows, at most: some thousands."""
    n = P.mtdao_peri_norm_workspace(shape(P, rows=rows, d=d, gate_rows=gate_rows))
    assert 0 < n <= 4 * 4 * d * (152 * 64 + min(gate_rows, 4 * 152 * 64))
