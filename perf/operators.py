"""Performance cases of the mixture-of-experts operators and of the products
with 4-bit weights.

A case is one operator as a layer calls it:

* ``route``: the tokens' choices sorted by expert, and the tokens' rows laid
  out in that order;
* ``combine``: the experts' rows summed back into the tokens' rows with the
  router's weights;
* ``grad``: the gradients of both: of the experts' rows and the weights, and
  of the tokens' rows;
* ``q4``: a matrix with 4-bit weights and group scales times one or a few
  vectors;
* ``experts``: the same product with every expert's matrix over the rows that
  belong to it, plain or with a gated activation.

Activations and gradients are normal, the router's weights a softmax over the
chosen experts, 4-bit codes uniform with scales of a matrix of unit gain.  A
popularity exponent above zero makes some experts more popular than others
(expert e is chosen as often as (e + 1) to the minus that power).
"""
from __future__ import annotations

import functools
import math

import torch

own = False

DEV = "cuda"
TORCH_TYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ABI_TYPE = {"f32": 0, "f16": 1, "bf16": 2}
ELT = {"f32": 4, "f16": 2, "bf16": 2}


def _moe(name, kind, N, k, E, D, dtype, dropped=0.0, skew=0.0):
    """dropped: the share of choices that no expert takes."""
    return {"name": name, "kind": kind, "N": N, "k": k, "E": E, "D": D, "dtype": dtype, "dropped": dropped, "skew": skew}


def _q4(name, N, M, K, group, dtype, zeros=True, glu=False):
    return {"name": name, "kind": "q4", "N": N, "M": M, "K": K, "group": group, "dtype": dtype, "zeros": zeros, "glu": glu}


def _experts(name, N, k, E, M, K, group, dtype, zeros=True, glu=False, gather=False, dropped=0.0, skew=0.0):
    """gather: rows are read through the sorted order from the tokens' rows,
    which then need no rows of their own per choice."""
    return {"name": name, "kind": "experts", "N": N, "k": k, "E": E, "M": M, "K": K, "group": group, "dtype": dtype,
            "zeros": zeros, "glu": glu, "gather": gather, "dropped": dropped, "skew": skew}


def listed():
    return [
        # One step of a small decoding batch: launch latency decides.
        _moe("route_decode", "route", 32, 8, 128, 4096, "bf16"),
        # A long prompt or a training batch, popular and unpopular experts.
        _moe("route_prefill", "route", 16384, 8, 256, 2048, "bf16", 0.0, 0.5),
        # The same decoding step on its way back, half precision.
        _moe("combine_decode", "combine", 32, 8, 128, 4096, "f16"),
        # A prompt of odd length with rows of odd width, some choices over the experts' capacity and dropped.
        _moe("combine_odd", "combine", 9001, 6, 64, 1999, "bf16", 0.1, 1.0),
        # A small training step in single precision.
        _moe("grad_small_f32", "grad", 500, 2, 8, 512, "f32", 0.05),
        # A training batch of a wide model.
        _moe("grad_wide", "grad", 16384, 4, 64, 4096, "bf16"),
        # A 4096 x 4096 projection, one token: the smallest decoding product.
        _q4("q4_one_token", 1, 4096, 4096, 128, "bf16"),
        # An output projection to 65536 words, one token.
        _q4("q4_wide_f16", 1, 65536, 8192, 128, "f16", False),
        # A batch of twelve on a matrix of odd sides: rows of 2501 bytes, the last group cut short.
        _q4("q4_batch_odd", 12, 10001, 5001, 64, "bf16"),
        # Gate and up projections of one decoding step: few tokens to each expert, none to some.
        _experts("experts_decode", 32, 8, 128, 2048, 2048, 128, "bf16", True, True, True),
        # A short prompt: ragged groups of small experts, short scales' groups, symmetric codes.
        _experts("experts_ragged", 300, 4, 60, 1400, 1000, 32, "f16", False, False, False, 0.05, 0.7),
        # A long prompt: the experts' products are matrix products.
        _experts("experts_prefill", 4096, 8, 64, 4096, 2048, 128, "bf16", True, True, True, 0.0, 0.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row's width: any number, or one of whole 16-byte vectors."""
    step = rng.choice((1, 8, 160))
    return max(step, _log_int(rng, lo, hi) // step * step)


_MOST_ROW_BYTES = 1.0e9   # of the rows by expert
_MOST_WEIGHTS = 0.5e9     # 4-bit weights of a matrix or of all experts
_MOST_FLOPS = 0.5e12


def draw(rng):
    """One more case over the same ranges."""
    kind = rng.choice(("route", "combine", "grad", "q4", "q4", "experts", "experts"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    E = _log_int(rng, 1, 256)
    k = rng.randint(1, min(8, E))
    N = _log_int(rng, 1, 16384)
    dropped = rng.choice((0.0, 0.0, 0.0, 0.05, 0.3))
    skew = rng.choice((0.0, 0.0, 0.5, 1.0))
    if kind in ("route", "combine", "grad"):
        D = _width(rng, 16, 8192)
        while N > 1 and N * k * D * ELT[dtype] > _MOST_ROW_BYTES * (0.5 if kind == "grad" else 1.0):
            N //= 2
        case = _moe("", kind, N, k, E, D, dtype, dropped, skew)
    else:
        group = rng.choice((32, 64, 128, 128, 256))
        zeros, glu = rng.random() < 0.5, rng.random() < 0.4
        K = _width(rng, 64, 12288)
        if kind == "q4":
            N = rng.choice((1, 1, 2, 4)) if rng.random() < 0.5 else _log_int(rng, 1, 64)
            M = _log_int(rng, 32, 65536) // 2 * 2
            while M > 2 and M * K > _MOST_WEIGHTS:
                M = M // 4 * 2
            case = _q4("", N, M, K, group, dtype, zeros, glu)
        else:
            E = min(E, 128)
            k = min(k, E)
            N = _log_int(rng, 1, 4096)
            K = min(K, 4096)
            M = _log_int(rng, 32, 4096) // 2 * 2
            while M > 2 and E * M * K > _MOST_WEIGHTS:
                M = M // 4 * 2
            most = _MOST_FLOPS / 4 if dtype == "f32" else _MOST_FLOPS
            while N > 1 and 2.0 * N * k * M * K > most:
                N //= 2
            case = _experts("", N, k, E, M, K, group, dtype, zeros, glu, rng.random() < 0.5, dropped, skew)
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs

def _choices(case, g):
    """Every token's k different experts, int32 [N, k]; dropped ones are -1."""
    N, k, E = case["N"], case["k"], case["E"]
    log_p = -case["skew"] * torch.log(torch.arange(1, E + 1, device=DEV, dtype=torch.float32))
    u = torch.rand((N, E), generator=g, device=DEV).clamp_(1e-9, 1 - 1e-7)
    ids = (log_p - torch.log(-torch.log(u))).topk(k, dim=1).indices.int()
    if case["dropped"]:
        ids[torch.rand((N, k), generator=g, device=DEV) < case["dropped"]] = -1
    return ids


def _sorted_by_expert(ids, E):
    """(offsets int32 [E + 1], pos int32 [N, k], src int32 [N k]) of the
    choices: by expert, then in their own order; dropped ones last."""
    key = torch.where((ids >= 0) & (ids < E), ids, E).reshape(-1)
    src = torch.argsort(key, stable=True)
    pos = torch.empty_like(src)
    pos[src] = torch.arange(src.numel(), device=ids.device)
    offsets = torch.searchsorted(key[src], torch.arange(E + 1, device=ids.device, dtype=key.dtype))
    return offsets.int(), pos.int().view(ids.shape), src.int()


def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(TORCH_TYPE[dtype])


def _codes(case, experts, g):
    """4-bit weights of `experts` matrices: codes [.., M, ceil(K / 2)] (even
    columns in the low bits), scales and zero points [.., M, ceil(K / group)]."""
    M, K = case["M"], case["K"]
    groups = -(-K // case["group"])
    codes = torch.randint(0, 256, (experts, M, -(-K // 2)), generator=g, device=DEV, dtype=torch.uint8)
    scales = ((0.75 + 0.5 * torch.rand((experts, M, groups), generator=g, device=DEV)) / (4.6 * math.sqrt(K)))
    zeros = None
    if case["zeros"]:
        zeros = torch.randint(5, 11, (experts, M, groups), generator=g, device=DEV, dtype=torch.uint8)
    return codes, scales.to(TORCH_TYPE[case["dtype"]]), zeros


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    kind, dtype = case["kind"], TORCH_TYPE[case["dtype"]]
    if kind == "q4":
        s["codes"], s["scales"], s["zeros"] = _codes(case, 1, g)
        s["x"] = _normal((case["N"], case["K"]), case["dtype"], g)
        s["y"] = torch.empty((case["N"], case["M"] // (2 if case["glu"] else 1)), dtype=dtype, device=DEV)
        return s
    N, k, E = case["N"], case["k"], case["E"]
    ids = _choices(case, g)
    if kind == "route":
        s["ids"] = ids
        s["x"] = _normal((N, case["D"]), case["dtype"], g)
        s["offsets"] = torch.empty(E + 1, dtype=torch.int32, device=DEV)
        s["pos"] = torch.empty((N, k), dtype=torch.int32, device=DEV)
        s["src"] = torch.empty(N * k, dtype=torch.int32, device=DEV)
        s["xs"] = torch.empty((N * k, case["D"]), dtype=dtype, device=DEV)
        return s
    s["offsets"], s["pos"], s["src"] = _sorted_by_expert(ids, E)
    if kind == "experts":
        s["codes"], s["scales"], s["zeros"] = _codes(case, E, g)
        s["x"] = _normal((N if case["gather"] else N * k, case["K"]), case["dtype"], g)
        s["y"] = torch.empty((N * k, case["M"] // (2 if case["glu"] else 1)), dtype=dtype, device=DEV)
        # The most rows of an expert, for padding them to one length.
        s["most"] = max(1, int((s["offsets"][1:] - s["offsets"][:-1]).max()))
        return s
    s["weights"] = torch.softmax(torch.randn((N, k), generator=g, device=DEV), dim=1)
    s["ys"] = _normal((N * k, case["D"]), case["dtype"], g)
    if kind == "combine":
        s["out"] = torch.empty((N, case["D"]), dtype=dtype, device=DEV)
        return s
    s["dout"] = _normal((N, case["D"]), case["dtype"], g)
    s["dxs"] = _normal((N * k, case["D"]), case["dtype"], g)
    s["dys"] = torch.empty_like(s["ys"])
    s["dweights"] = torch.empty_like(s["weights"])
    s["dx"] = torch.empty_like(s["dout"])
    return s


# -------------------------------------------------------------- plain forms

def _kept_rows(rows, s):
    """The rows of every token's choices, float32 [N, k, D]; zeros for dropped ones."""
    pos = s["pos"].long()
    return torch.where((pos < s["offsets"][-1])[..., None], rows[pos].float(), 0.0)


def _plain_route(s):
    offsets, pos, src = _sorted_by_expert(s["ids"], s["case"]["E"])
    kept = torch.arange(src.numel(), device=DEV) < offsets[-1]
    xs = torch.where(kept[:, None], s["x"][src.long() // s["case"]["k"]], 0.0)
    return {"offsets": offsets, "pos": pos, "src": src, "xs": xs}


def _plain_combine(s):
    out = (_kept_rows(s["ys"], s) * s["weights"][..., None]).sum(1)
    return {"out": out.to(s["ys"].dtype)}


def _plain_grad(s):
    kept = s["pos"] < s["offsets"][-1]
    dout = s["dout"].float()
    dweights = (_kept_rows(s["ys"], s) * dout[:, None, :]).sum(2)
    scaled = torch.where(kept, s["weights"], 0.0)[..., None] * dout[:, None, :]
    dys = scaled.to(s["ys"].dtype).reshape(s["ys"].shape)[s["src"].long()]
    dx = _kept_rows(s["dxs"], s).sum(1)
    return {"dys": dys, "dweights": dweights, "dx": dx.to(s["dxs"].dtype)}


def _plain_weights(s):
    """float32 [experts, M, K]."""
    case, codes = s["case"], s["codes"]
    q = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)[..., :case["K"]].float()
    column = torch.arange(case["K"], device=DEV) // case["group"]
    z = s["zeros"].float()[..., column] if s["zeros"] is not None else 8.0
    return (q - z) * s["scales"].float()[..., column]


def _gated(y, case):
    if not case["glu"]:
        return y
    gate, up = y.chunk(2, dim=-1)
    return gate / (1 + torch.exp(-gate)) * up


def _plain_q4(s):
    y = s["x"].float() @ _plain_weights(s)[0].t()
    return {"y": _gated(y, s["case"]).to(s["x"].dtype)}


def _plain_experts(s):
    case = s["case"]
    x = s["x"][s["src"].long() // case["k"]] if case["gather"] else s["x"]
    offsets = s["offsets"].long()
    at = offsets[:-1, None] + torch.arange(s["most"], device=DEV)  # every expert's rows, padded to one length
    rows = torch.where((at < offsets[1:, None])[..., None], x[at.clamp(max=x.shape[0] - 1)].float(), 0.0)
    y = _gated(torch.bmm(rows, _plain_weights(s).transpose(1, 2)), case)
    p = torch.arange(x.shape[0], device=DEV)
    e = (torch.searchsorted(offsets, p, right=True) - 1).clamp(max=case["E"] - 1)
    y = y[e, (p - offsets[e]).clamp(max=s["most"] - 1)]
    return {"y": torch.where((p < offsets[-1])[:, None], y, 0.0).to(s["x"].dtype)}


# ------------------------------------------------------ the framework's calls

@functools.lru_cache(maxsize=None)
def _perm(N, k, E):
    import paper_2305_06942_amd as ebag
    return ebag.MoePerm(N, k, E)


@functools.lru_cache(maxsize=None)
def _product(M, K, group, dtype, experts, glu):
    import paper_2305_06942_amd as ebag
    return ebag.Q4Gemv(M, K, group, ABI_TYPE[dtype], experts=experts, glu=int(glu))


def _own(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "q4":
        q = _product(case["M"], case["K"], case["group"], case["dtype"], 1, case["glu"])
        q.forward(s["codes"], s["scales"], s["zeros"], s["x"], s["y"])
        return {"y": s["y"]}
    if kind == "experts":
        q = _product(case["M"], case["K"], case["group"], case["dtype"], case["E"], case["glu"])
        q.experts(s["codes"], s["scales"], s["zeros"], s["x"], s["offsets"], s["y"],
                  src=s["src"] if case["gather"] else None, k=case["k"])
        return {"y": s["y"]}
    perm = _perm(case["N"], case["k"], case["E"])
    if kind == "route":
        perm.sort(s["ids"], s["offsets"], s["pos"], s["src"])
        perm.dispatch(s["x"], s["offsets"], s["pos"], s["xs"])
        return {n: s[n] for n in ("offsets", "pos", "src", "xs")}
    if kind == "combine":
        perm.combine(s["ys"], s["offsets"], s["pos"], s["weights"], s["out"])
        return {"out": s["out"]}
    perm.combine_backward(s["dout"], s["ys"], s["offsets"], s["pos"], s["weights"], s["dys"], s["dweights"])
    perm.dispatch_backward(s["dxs"], s["offsets"], s["pos"], s["dx"])
    return {n: s[n] for n in ("dys", "dweights", "dx")}


_PLAIN = {"route": _plain_route, "combine": _plain_combine, "grad": _plain_grad, "q4": _plain_q4, "experts": _plain_experts}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------- bounds

def work(case):
    kind, elt = case["kind"], ELT[case["dtype"]]
    if kind in ("route", "combine", "grad"):
        N, D = case["N"], case["D"]
        S = N * case["k"]
        kept = S * (1 - case["dropped"])
        table = 4 * (case["E"] + 1)
        if kind == "route":
            return {"bytes": 12 * S + table + (N + S) * D * elt, "flops": 0}
        if kind == "combine":
            return {"bytes": 8 * S + table + (N + kept) * D * elt, "flops": 2 * kept * D}
        return {"bytes": 12 * S + table + (2 * N + 2 * kept + S) * D * elt, "flops": 4 * kept * D}
    M, K = case["M"], case["K"]
    matrix = M * (-(-K // 2) + -(-K // case["group"]) * (elt + (1 if case["zeros"] else 0)))
    wide = M // (2 if case["glu"] else 1)
    if kind == "q4":
        N = case["N"]
        return {"bytes": matrix + N * (K + wide) * elt, "flops": 2 * N * M * K}
    E, k, N = case["E"], case["k"], case["N"]
    S = N * k
    kept = S * (1 - case["dropped"])
    p = [(e + 1) ** -case["skew"] for e in range(E)]
    used = sum(1 - (1 - min(1.0, k * v / sum(p))) ** N for v in p)  # experts with rows, as expected
    rows = N if case["gather"] else kept
    return {"bytes": used * matrix + rows * K * elt + S * (wide * elt + 4) + 4 * (E + 1), "flops": 2 * kept * M * K}


# ------------------------------------------------------------ exact results

def _exact_order(ids, E):
    """The flat choices in the order of their experts, and where each expert's end."""
    flat = ids.reshape(-1).long()
    per = [torch.nonzero(flat == e)[:, 0] for e in range(E)]
    return torch.cat(per), [t.numel() for t in per]


def _exact_matrix(s, e):
    case = s["case"]
    q = torch.empty((case["M"], 2 * s["codes"].shape[-1]), dtype=torch.float64, device=DEV)
    q[:, 0::2] = s["codes"][e].bitwise_and(0x0F).double()
    q[:, 1::2] = s["codes"][e].bitwise_right_shift(4).double()
    for b in range(s["scales"].shape[-1]):
        part = q[:, b * case["group"]:(b + 1) * case["group"]]
        part -= s["zeros"][e, :, b:b + 1].double() if s["zeros"] is not None else 8
        part *= s["scales"][e, :, b:b + 1].double()
    return q[:, :case["K"]]


def _exact_product(x, matrix, glu):
    y = torch.matmul(x.double(), matrix.t().contiguous())
    if glu:
        half = y.shape[1] // 2
        y = y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "q4":
        return {"y": _exact_product(s["x"], _exact_matrix(s, 0), case["glu"])}
    if kind == "route":
        order, _ = _exact_order(s["ids"], case["E"])
        xs = torch.zeros((case["N"] * case["k"], case["D"]), dtype=torch.float64, device=DEV)
        xs[:order.numel()] = s["x"].double()[torch.div(order, case["k"], rounding_mode="floor")]
        return {"offsets": None, "pos": None, "src": None, "xs": xs}
    if kind == "experts":
        y = torch.zeros(tuple(s["y"].shape), dtype=torch.float64, device=DEV)
        ends = s["offsets"].tolist()
        for e in range(case["E"]):
            lo, hi = ends[e], ends[e + 1]
            if lo < hi:
                token = torch.div(s["src"][lo:hi].long(), case["k"], rounding_mode="floor")
                rows = s["x"][token] if case["gather"] else s["x"][lo:hi]
                y[lo:hi] = _exact_product(rows, _exact_matrix(s, e), case["glu"])
        return {"y": y}
    total = int(s["offsets"][-1])
    sums = torch.zeros((case["N"], case["D"]), dtype=torch.float64, device=DEV)
    if kind == "combine":
        for j in range(case["k"]):
            here = torch.nonzero(s["pos"][:, j] < total)[:, 0]
            sums[here] += s["weights"][here, j, None].double() * s["ys"][s["pos"][here, j].long()].double()
        return {"out": sums}
    dys = torch.zeros(tuple(s["dys"].shape), dtype=torch.float64, device=DEV)
    dweights = torch.zeros((case["N"], case["k"]), dtype=torch.float64, device=DEV)
    for j in range(case["k"]):
        here = torch.nonzero(s["pos"][:, j] < total)[:, 0]
        at = s["pos"][here, j].long()
        dys[at] = s["weights"][here, j, None].double() * s["dout"][here].double()
        dweights[here, j] = (s["dout"][here].double() * s["ys"][at].double()).sum(1)
        sums[here] += s["dxs"][at].double()
    return {"dys": dys, "dweights": dweights, "dx": sums}
