"""The tokens-by-expert calls refuse bad arguments before touching the GPU (no
GPU needed): the C ABI's own checks, and the binding's checks of tensors."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2305_06942_amd as ebag
    return ebag.load()


@pytest.mark.parametrize("args,msg", [
    ((10, 0, 4), "choices"), ((10, 65, 4), "choices"), ((10, 2, 0), "experts"), ((10, 2, 513), "experts"),
    ((-1, 2, 4), "max_tokens"), ((1 << 30, 2, 4), "max_tokens"), ((1 << 62, 1, 4), "max_tokens")])
def test_create_refuses(lib, args, msg):
    import paper_2305_06942_amd as ebag
    h = ctypes.c_void_p()
    assert lib.ebag_a2a_moe_create(ctypes.byref(h), *args) == ebag.abi.EBAG_EINVAL
    assert msg in ebag.last_error() and not h.value


def test_null_plan_is_refused(lib):
    import paper_2305_06942_amd as ebag
    bad = ebag.abi.EBAG_EINVAL
    assert lib.ebag_a2a_moe_create(None, 1, 1, 1) == bad
    assert lib.ebag_a2a_moe_sort(None, None, 1, None, None, None, None) == bad
    assert lib.ebag_a2a_moe_dispatch(None, None, 8, 8, 0, 1, None, None, None, 8, None) == bad
    assert lib.ebag_a2a_moe_dispatch_backward(None, None, 8, 8, 0, 1, None, None, None, 8, None) == bad
    assert lib.ebag_a2a_moe_combine(None, None, 8, 8, 0, 1, None, None, None, None, 8, None) == bad
    assert lib.ebag_a2a_moe_combine_backward(None, None, 8, None, 8, 8, 0, 1, None, None, None, None, 8, None, None) == bad
    lib.ebag_a2a_moe_destroy(None)


class _NoCalls:
    def __getattr__(self, name):
        def call(*a):
            raise AssertionError(f"{name} was called")
        return call


def _plan(choices=2, experts=4):
    import paper_2305_06942_amd as ebag
    p = object.__new__(ebag.MoePerm)
    p._h, p._lib = None, _NoCalls()
    p._shape(choices, experts)
    return p


def _args(N=3, k=2, E=4, D=8):
    import torch
    return dict(x=torch.zeros(N, D), xs=torch.zeros(N * k, D), offsets=torch.zeros(E + 1, dtype=torch.int32),
                pos=torch.zeros(N, k, dtype=torch.int32), src=torch.zeros(N * k, dtype=torch.int32),
                w=torch.zeros(N, k), ids=torch.zeros(N, k, dtype=torch.int32))


def _with(**kw):
    a = _args()
    a.update(kw)
    return a


def test_binding_refuses(lib):
    import torch
    p = _plan()
    i32 = dict(dtype=torch.int32)
    # These tensors are on the CPU: each is refused for what is wrong with it first, and a right one for its device.
    for a, msg in [(_args(), "must be a GPU tensor"), (_with(ids=torch.zeros(3, 2)), "experts_of must be int32"),
                   (_with(offsets=torch.zeros(5, dtype=torch.int64)), "offsets must be int32"),
                   (_with(src=torch.zeros(12, **i32)[::2]), "src must be contiguous")]:
        with pytest.raises(ValueError, match=msg):
            p.sort(a["ids"], a["offsets"], a["pos"], a["src"], stream=0)

    def fields(**kw):
        """With the device check of whole-number tensors out of the way."""
        class On:
            def __init__(self, t):
                self.t = t

            is_cuda = True

            def __getattr__(self, name):
                return getattr(self.t, name)
        return {n: On(t) for n, t in _with(**kw).items()}

    for kw, msg in [(dict(ids=torch.zeros(3, 3, **i32)), "experts_of must be"), (dict(offsets=torch.zeros(4, **i32)), "offsets holds"),
                    (dict(pos=torch.zeros(2, 2, **i32)), "pos holds"), (dict(src=torch.zeros(5, **i32)), "src holds")]:
        a = fields(**kw)
        with pytest.raises(ValueError, match=msg):
            p.sort(a["ids"], a["offsets"], a["pos"], a["src"], stream=0)
    for kw, msg in [(dict(x=torch.zeros(3, 8).double()), "x must be float32 or float16 or bfloat16"),
                    (dict(xs=torch.zeros(6, 8).half()), "xs must be float32"), (dict(xs=torch.zeros(5, 8)), "xs must be"),
                    (dict(x=torch.zeros(8, 3).t()), "contiguous rows"), (dict(x=torch.zeros(3, 1).expand(3, 8)), "contiguous rows"),
                    (dict(x=torch.zeros(1, 8).expand(3, 8)), "contiguous rows"), (dict(xs=torch.zeros(6, 7)), "xs must be")]:
        a = fields(**kw)
        with pytest.raises(ValueError, match=msg):
            p.dispatch(a["x"], a["offsets"], a["pos"], a["xs"], stream=0)
    for kw, msg in [(dict(w=torch.zeros(2, 2)), "weights holds"), (dict(w=torch.zeros(3, 2).half()), "weights must be float32")]:
        a = fields(**kw)
        with pytest.raises(ValueError, match=msg):
            p.combine(a["xs"], a["offsets"], a["pos"], a["w"], a["x"], stream=0)
        with pytest.raises(ValueError, match=msg):
            p.combine_backward(a["x"], a["xs"], a["offsets"], a["pos"], a["w"], a["xs"], a["w"], stream=0)
