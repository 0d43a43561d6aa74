"""Products with 4-bit weights refuse bad arguments before touching the GPU (no
GPU needed): the C ABI's own checks, and the binding's checks of tensors."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2305_06942_amd as ebag
    return ebag.load()


@pytest.mark.parametrize("kw,msg", [
    (dict(M=0), "M="), (dict(M=1 << 31), "M="), (dict(K=0), "K="), (dict(K=1 << 31), "K="), (dict(M=1 << 22, K=1 << 20), "2^40"),
    (dict(group=0), "group"), (dict(group=16), "group"), (dict(group=48), "group"), (dict(group=-32), "group"),
    (dict(dtype=3), "dtype"), (dict(experts=0), "experts"), (dict(experts=513), "experts"), (dict(glu=2), "glu"),
    (dict(M=15, glu=1), "even M")])
def test_create_refuses(lib, kw, msg):
    import paper_2305_06942_amd as ebag
    a = dict(M=16, K=64, group=32, dtype=0, experts=1, glu=0)
    a.update(kw)
    h = ctypes.c_void_p()
    assert lib.gemv_ar_q4_create(ctypes.byref(h), *a.values()) == ebag.abi.EBAG_EINVAL
    assert msg in ebag.last_error() and not h.value


def test_null_plan_is_refused(lib):
    import paper_2305_06942_amd as ebag
    bad = ebag.abi.EBAG_EINVAL
    assert lib.gemv_ar_q4_create(None, 16, 64, 32, 0, 1, 0) == bad
    assert lib.gemv_ar_q4_quantize(None, None, None, None, None, None) == bad
    assert lib.gemv_ar_q4_forward(None, None, None, None, None, 64, 1, None, 16, 0, None) == bad
    assert lib.gemv_ar_q4_experts(None, None, None, None, None, 64, 1, None, None, 1, 1, None, 16, 0, None) == bad
    lib.gemv_ar_q4_destroy(None)


class _NoCalls:
    def __getattr__(self, name):
        def call(*a):
            raise AssertionError(f"{name} was called")
        return call


class _On:
    """A CPU tensor that says it is on the GPU."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def _plan(M=6, K=40, group=32, dtype=1, experts=3, glu=0):
    import paper_2305_06942_amd as ebag
    p = object.__new__(ebag.Q4Gemv)
    p._h, p._lib = None, _NoCalls()
    p._shape(M, K, group, dtype, experts, glu)
    return p


def _args(**kw):
    import torch
    a = dict(codes=torch.zeros(3, 6, 20, dtype=torch.uint8), scales=torch.zeros(3, 6, 2).half(),
             zeros=torch.zeros(3, 6, 2, dtype=torch.uint8), x=torch.zeros(5, 40).half(),
             offsets=torch.zeros(4, dtype=torch.int32), y=torch.zeros(5, 6).half(), src=None)
    a.update(kw)
    return a


def test_binding_refuses(lib):
    import torch
    p = _plan()
    u8 = dict(dtype=torch.uint8)
    a = _args()
    with pytest.raises(ValueError, match="codes must be a GPU tensor"):
        p.forward(a["codes"], a["scales"], a["zeros"], a["x"], a["y"], stream=0)
    for kw, msg in [(dict(codes=torch.zeros(3, 6, 19, **u8)), "codes holds"), (dict(codes=torch.zeros(3, 6, 20, dtype=torch.int8)), "codes must be uint8"),
                    (dict(codes=torch.zeros(3, 6, 40, **u8)[..., ::2]), "codes must be contiguous"),
                    (dict(scales=torch.zeros(3, 6, 1).half()), "scales holds"), (dict(scales=torch.zeros(3, 6, 2)), "scales must be float16"),
                    (dict(zeros=torch.zeros(3, 6, 1, **u8)), "zeros holds"), (dict(x=torch.zeros(5, 40)), "x must be float16"),
                    (dict(x=torch.zeros(5, 41).half()), "x must be"), (dict(x=torch.zeros(40, 5).half().t()), "contiguous rows"),
                    (dict(y=torch.zeros(4, 6).half()), "y must be"), (dict(y=torch.zeros(5, 7).half()), "y must be"),
                    (dict(y=torch.zeros(5, 6).bfloat16()), "y must be float16"), (dict(y=torch.zeros(6, 5).half().t()), "contiguous rows")]:
        a = {n: None if t is None else _On(t) for n, t in _args(**kw).items()}
        with pytest.raises(ValueError, match=msg):
            p.forward(a["codes"], a["scales"], a["zeros"], a["x"], a["y"], stream=0)
        with pytest.raises(ValueError, match=msg):
            p.experts(a["codes"], a["scales"], a["zeros"], a["x"], a["offsets"], a["y"], stream=0)
    for kw, msg in [(dict(offsets=torch.zeros(3, dtype=torch.int32)), "offsets holds"), (dict(offsets=torch.zeros(4, dtype=torch.int64)), "offsets must be int32"),
                    (dict(src=torch.zeros(10, dtype=torch.int64)), "src must be int32"), (dict(src=torch.zeros(10, dtype=torch.int32)), "y must be")]:
        a = {n: None if t is None else _On(t) for n, t in _args(**kw).items()}
        with pytest.raises(ValueError, match=msg):
            p.experts(a["codes"], a["scales"], a["zeros"], a["x"], a["offsets"], a["y"], src=a["src"], k=2, stream=0)
    a = {n: None if t is None else _On(t) for n, t in _args().items()}
    for w, msg in [(torch.zeros(3, 6, 39).half(), "w holds"), (torch.zeros(3, 6, 40), "w must be float16")]:
        with pytest.raises(ValueError, match=msg):
            p.quantize(_On(w), a["codes"], a["scales"], a["zeros"], stream=0)
