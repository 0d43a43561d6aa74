"""The router's calls refuse bad arguments before touching the GPU (no GPU
needed): the C ABI's own checks, and the binding's checks of tensors."""
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2305_06942_amd as ebag
    return ebag.load()


def test_null_plan_is_refused(lib):
    import paper_2305_06942_amd as ebag
    bad = ebag.abi.EBAG_EINVAL
    assert lib.ebag_a2a_moe_choose(None, None, 8, 0, 1, None, None, 1, None, None, None, None, None, None, None) == bad
    assert lib.ebag_a2a_moe_choose_backward(None, None, 8, 0, 1, None, 1, None, None, None, None, None, 8, None) == bad
    assert lib.ebag_a2a_moe_choose_work(None) == 0


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


def _plan(choices=2, experts=4):
    import paper_2305_06942_amd as ebag
    p = object.__new__(ebag.MoePerm)
    p._h, p._lib = None, _NoCalls()
    p._shape(choices, experts)
    return p


def _args(**kw):
    import torch
    i32 = dict(dtype=torch.int32)
    a = dict(logits=torch.zeros(3, 4), ids=torch.zeros(3, 2, **i32), weights=torch.zeros(3, 2), counts=torch.zeros(5, **i32),
             sums=torch.zeros(5), losses=torch.zeros(2), work=torch.zeros(32 + 512 * 5), bias=torch.zeros(4),
             live=torch.zeros(3, dtype=torch.bool))
    a.update(kw)
    return {n: None if t is None else _On(t) for n, t in a.items()}


def test_choose_refuses(lib):
    import torch
    p = _plan()
    i32 = dict(dtype=torch.int32)
    for kw, msg in [(dict(logits=torch.zeros(3, 5)), "logits must be"), (dict(logits=torch.zeros(3, 4).double()), "logits must be float32"),
                    (dict(logits=torch.zeros(4, 3).t()), "contiguous rows"), (dict(logits=torch.zeros(1, 4).expand(3, 4)), "contiguous rows"),
                    (dict(ids=torch.zeros(2, 2, **i32)), "ids holds"), (dict(ids=torch.zeros(3, 2, dtype=torch.int64)), "ids must be int32"),
                    (dict(weights=torch.zeros(2, 2)), "weights holds"), (dict(weights=torch.zeros(3, 2).half()), "weights must be float32"),
                    (dict(weights=torch.zeros(2, 3).t()), "weights must be contiguous"),
                    (dict(bias=torch.zeros(3)), "bias holds"), (dict(bias=torch.zeros(4).half()), "bias must be float32"),
                    (dict(counts=torch.zeros(4, **i32)), "counts holds"), (dict(sums=torch.zeros(4)), "sums holds"),
                    (dict(losses=torch.zeros(1)), "losses holds"), (dict(work=torch.zeros(512)), "work holds"),
                    (dict(counts=None), "go together"), (dict(work=None), "go together"), (dict(losses=None), "go together"),
                    (dict(live=torch.zeros(2, dtype=torch.bool)), "live holds"), (dict(live=torch.zeros(3)), "live must be bool or uint8"),
                    (dict(live=torch.zeros(6, dtype=torch.bool)[::2]), "live must be contiguous")]:
        a = _args(**kw)
        with pytest.raises(ValueError, match=msg):
            p.choose(**a, stream=0)
    a = _args()
    a["ids"] = a["ids"].t
    with pytest.raises(ValueError, match="ids must be a GPU tensor"):
        p.choose(**a, stream=0)


def test_backward_refuses(lib):
    import torch
    p = _plan()
    i32 = dict(dtype=torch.int32)
    good = dict(logits=torch.zeros(3, 4), ids=torch.zeros(3, 2, **i32), dweights=torch.zeros(3, 2), dlogits=torch.zeros(3, 4),
                counts=torch.zeros(5, **i32), dlosses=torch.zeros(2), live=None)
    for kw, msg in [(dict(logits=torch.zeros(3, 5)), "logits must be"), (dict(dlogits=torch.zeros(3, 4).half()), "dlogits must be float32"),
                    (dict(dlogits=torch.zeros(2, 4)), "dlogits must be"), (dict(ids=None), "dweights need ids"),
                    (dict(ids=torch.zeros(2, 2, **i32)), "ids holds"), (dict(dweights=torch.zeros(2, 2)), "dweights holds"),
                    (dict(counts=None), "dlosses need counts"), (dict(counts=torch.zeros(4, **i32)), "counts holds"),
                    (dict(dlosses=torch.zeros(1)), "dlosses holds"), (dict(live=torch.zeros(2, dtype=torch.uint8)), "live holds")]:
        a = {n: None if t is None else _On(t) for n, t in {**good, **kw}.items()}
        with pytest.raises(ValueError, match=msg):
            p.choose_backward(**a, stream=0)
