"""Products in 8-bit integers refuse bad arguments before touching the GPU (no
GPU needed): the C ABI's own checks, and the binding's checks of tensors."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2305_06942_amd as ebag
    return ebag.load()


@pytest.mark.parametrize("kw,msg", [
    (dict(M=0), "M="), (dict(M=1 << 31), "M="), (dict(K=0), "K="), (dict(K=(1 << 17) + 1), "K="), (dict(dtype=3), "dtype"),
    (dict(dtype=-1), "dtype"), (dict(experts=0), "experts"), (dict(experts=513), "experts"), (dict(glu=2), "glu"),
    (dict(M=15, glu=1), "even M")])
def test_create_refuses(lib, kw, msg):
    import paper_2305_06942_amd as ebag
    a = dict(M=16, K=64, dtype=0, experts=1, glu=0)
    a.update(kw)
    h = ctypes.c_void_p()
    assert lib.gemv_ar_q8_create(ctypes.byref(h), *a.values()) == ebag.abi.EBAG_EINVAL
    assert msg in ebag.last_error() and not h.value


def test_null_plan_is_refused(lib):
    import paper_2305_06942_amd as ebag
    bad = ebag.abi.EBAG_EINVAL
    assert lib.gemv_ar_q8_create(None, 16, 64, 0, 1, 0) == bad
    assert lib.gemv_ar_q8_pitch(None) == 0
    assert lib.gemv_ar_q8_quantize(None, None, None, None, None) == bad
    assert lib.gemv_ar_q8_round(None, None, 64, 1, None, None, None) == bad
    assert lib.gemv_ar_q8_forward(None, None, None, None, 64, 1, None, None, None, 16, 0, None) == bad
    assert lib.gemv_ar_q8_experts(None, None, None, None, 64, 1, None, None, None, None, 1, 1, None, 16, 0, None) == bad
    lib.gemv_ar_q8_destroy(None)


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


def _plan(M=6, K=140, dtype=1, experts=3, glu=0):
    import paper_2305_06942_amd as ebag
    p = object.__new__(ebag.Q8Gemv)
    p._h, p._lib = None, _NoCalls()
    p._shape(M, K, dtype, experts, glu)
    return p


def _args(**kw):
    import torch
    a = dict(codes=torch.zeros(3, 6, 256, dtype=torch.int8), scales=torch.zeros(3, 6), x=torch.zeros(5, 140).half(),
             y=torch.zeros(5, 6).half(), xq=torch.zeros(5, 256, dtype=torch.int8), xs=torch.zeros(5),
             offsets=torch.zeros(4, dtype=torch.int32), src=None)
    a.update(kw)
    return a


def _on(a):
    return {n: None if t is None else _On(t) for n, t in a.items()}


def test_binding_refuses(lib):
    import torch
    p = _plan()
    assert p.pitch == 256
    i8 = dict(dtype=torch.int8)
    a = _args()
    with pytest.raises(ValueError, match="codes must be a GPU tensor"):
        p.forward(a["codes"], a["scales"], a["x"], a["y"], a["xq"], a["xs"], stream=0)
    for kw, msg in [(dict(codes=torch.zeros(3, 6, 255, **i8)), "codes holds"), (dict(codes=torch.zeros(3, 6, 256, dtype=torch.uint8)), "codes must be int8"),
                    (dict(codes=torch.zeros(3, 6, 512, **i8)[..., ::2]), "codes must be contiguous"), (dict(scales=torch.zeros(3, 5)), "scales holds"),
                    (dict(scales=torch.zeros(3, 6).half()), "scales must be float32"), (dict(x=torch.zeros(5, 140)), "x must be float16"),
                    (dict(x=torch.zeros(5, 256).half()), "x must be"), (dict(x=torch.zeros(140, 5).half().t()), "contiguous rows"),
                    (dict(xq=torch.zeros(5, 140, **i8)), "xq holds"), (dict(xq=torch.zeros(5, 256).half()), "xq must be int8"),
                    (dict(xs=torch.zeros(4)), "xs holds"), (dict(xs=torch.zeros(5).half()), "xs must be float32"),
                    (dict(y=torch.zeros(4, 6).half()), "y must be"), (dict(y=torch.zeros(5, 7).half()), "y must be"),
                    (dict(y=torch.zeros(5, 6).bfloat16()), "y must be float16"), (dict(y=torch.zeros(6, 5).half().t()), "contiguous rows")]:
        a = _on(_args(**kw))
        with pytest.raises(ValueError, match=msg):
            p.forward(a["codes"], a["scales"], a["x"], a["y"], a["xq"], a["xs"], stream=0)
        with pytest.raises(ValueError, match=msg):
            p.experts(a["codes"], a["scales"], a["x"], a["offsets"], a["y"], a["xq"], a["xs"], stream=0)
    for kw, msg in [(dict(offsets=torch.zeros(3, dtype=torch.int32)), "offsets holds"), (dict(offsets=torch.zeros(4, dtype=torch.int64)), "offsets must be int32"),
                    (dict(src=torch.zeros(10, dtype=torch.int64)), "src must be int32"), (dict(src=torch.zeros(10, dtype=torch.int32)), "y must be")]:
        a = _on(_args(**kw))
        with pytest.raises(ValueError, match=msg):
            p.experts(a["codes"], a["scales"], a["x"], a["offsets"], a["y"], a["xq"], a["xs"], src=a["src"], k=2, stream=0)
    a = _on(_args())
    for w, msg in [(torch.zeros(3, 6, 139).half(), "w holds"), (torch.zeros(3, 6, 140), "w must be float16")]:
        with pytest.raises(ValueError, match=msg):
            p.quantize(_On(w), a["codes"], a["scales"], stream=0)
    for kw, msg in [(dict(xq=torch.zeros(4, 256, **i8)), "xq holds"), (dict(x=torch.zeros(5, 139).half()), "x must be")]:
        a = _on(_args(**kw))
        with pytest.raises(ValueError, match=msg):
            p.round(a["x"], a["xq"], a["xs"], stream=0)
