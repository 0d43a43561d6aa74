"""Performance cases of the router of a mixture-of-experts layer, with its
balance loss, and of products in 8-bit integers.

A case is one operator as a layer calls it:

* ``choose``: every token's k experts and their weights from the router's
  logits, and, where a model is trained, the choices and the probabilities of
  each expert over all tokens with the two losses made of them;
* ``choose_grad``: the gradient of the weights and of both losses;
* ``linear8``: rows rounded to 8 bits with a scale each, times a matrix of 8-bit
  weights with a scale for every channel;
* ``experts8``: the same with every expert's matrix over the rows that belong to
  it, plain or with a gated activation.

Logits and activations are normal; tokens of a padded batch hold NaN, and a
token may be kept from some of the experts by logits of minus infinity.  8-bit
weights are uniform with scales of a matrix of unit gain.  A popularity exponent
above zero makes some experts more popular than others (expert e is chosen as
often as (e + 1) to the minus that power).
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


def _choose(name, kind, N, k, E, dtype, normalise=True, totals=False, bias=False, padded=0.0, masked=0.0):
    """totals: with the experts' sums and the losses.  padded: the share of
    tokens that are padding.  masked: the share of experts that a token may not
    choose.  bias: a bias on the choice, not on the weights."""
    return {"name": name, "kind": kind, "N": N, "k": k, "E": E, "dtype": dtype, "normalise": normalise, "totals": totals,
            "bias": bias, "padded": padded, "masked": masked}


def _linear8(name, N, M, K, dtype, glu=False):
    return {"name": name, "kind": "linear8", "N": N, "M": M, "K": K, "dtype": dtype, "glu": glu}


def _experts8(name, N, k, E, M, K, dtype, glu=False, gather=False, dropped=0.0, skew=0.0):
    """gather: rows are read through the sorted order from the tokens' rows,
    which then need no rows of their own per choice.  dropped: the share of
    choices that no expert takes."""
    return {"name": name, "kind": "experts8", "N": N, "k": k, "E": E, "M": M, "K": K, "dtype": dtype, "glu": glu,
            "gather": gather, "dropped": dropped, "skew": skew}


def listed():
    return [
        # One step of a small decoding batch: launch latency decides.
        _choose("choose_decode", "choose", 32, 8, 128, "f32"),
        # A training batch: choices, counts and both losses.
        _choose("choose_train", "choose", 16384, 8, 256, "f32", True, True),
        # A padded batch of odd length, an odd number of experts of which a token may have half, a bias that evens loads out.
        _choose("choose_odd", "choose", 9001, 6, 60, "bf16", False, True, True, 0.2, 0.5),
        # The gradients of both.
        _choose("choose_grad_train", "choose_grad", 16384, 8, 256, "f32", True, True),
        _choose("choose_grad_odd", "choose_grad", 9001, 6, 60, "bf16", False, True, True, 0.2, 0.5),
        # A 4096 x 4096 projection, one token: the smallest decoding product.
        _linear8("linear8_one_token", 1, 4096, 4096, "bf16"),
        # A batch of twelve on a matrix of odd sides.
        _linear8("linear8_batch_odd", 12, 10001, 5001, "f16"),
        # An output projection to 65536 words for a batch of 64.
        _linear8("linear8_wide", 64, 65536, 8192, "bf16"),
        # A long prompt through a square projection: a matrix product.
        _linear8("linear8_prompt", 8192, 8192, 8192, "bf16"),
        # Gate and up projections of one decoding step: few tokens to each expert, none to some.
        _experts8("experts8_decode", 32, 8, 128, 2048, 2048, "bf16", True, True),
        # A short prompt: ragged groups of small experts, some choices over the experts' capacity and dropped.
        _experts8("experts8_ragged", 300, 4, 60, 1400, 1000, "f16", False, False, 0.05, 0.7),
        # A long prompt: the experts' products are matrix products.
        _experts8("experts8_prefill", 4096, 8, 64, 4096, 2048, "bf16", True, True, 0.0, 0.3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A row's width: any number, or one of whole 16-byte vectors or more."""
    step = rng.choice((1, 8, 160))
    return max(step, _log_int(rng, lo, hi) // step * step)


_MOST_LOGITS = 16384 * 256
_MOST_WEIGHTS = 0.5e9     # of a matrix or of all experts
_MOST_FLOPS = 0.5e12


def draw(rng):
    """One more case over the same ranges."""
    kind = rng.choice(("choose", "choose_grad", "linear8", "linear8", "experts8", "experts8"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    if kind in ("choose", "choose_grad"):
        E = _log_int(rng, 2, 512)
        k = rng.randint(1, min(16, E))
        N = _log_int(rng, 1, min(32768, _MOST_LOGITS // E))
        case = _choose("", kind, N, k, E, dtype, rng.random() < 0.5, kind == "choose_grad" or rng.random() < 0.6,
                       rng.random() < 0.4, rng.choice((0.0, 0.0, 0.1, 0.5)), rng.choice((0.0, 0.0, 0.3, 0.75)))
    else:
        K = _width(rng, 64, 12288)
        glu = rng.random() < 0.4
        if kind == "linear8":
            N = rng.choice((1, 1, 2, 4, 16)) if rng.random() < 0.4 else _log_int(rng, 1, 8192)
            M = _log_int(rng, 32, 65536) // 2 * 2
            while M > 2 and (M * K > _MOST_WEIGHTS or 2.0 * N * M * K > _MOST_FLOPS):
                M = M // 4 * 2
            case = _linear8("", N, M, K, dtype, glu)
        else:
            E = _log_int(rng, 1, 128)
            k = rng.randint(1, min(8, E))
            N = _log_int(rng, 1, 4096)
            K = min(K, 4096)
            M = _log_int(rng, 32, 4096) // 2 * 2
            while M > 2 and E * M * K > _MOST_WEIGHTS:
                M = M // 4 * 2
            while N > 1 and 2.0 * N * k * M * K > _MOST_FLOPS:
                N //= 2
            case = _experts8("", N, k, E, M, K, dtype, glu, rng.random() < 0.5, rng.choice((0.0, 0.0, 0.05, 0.3)),
                             rng.choice((0.0, 0.0, 0.5, 1.0)))
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs

def _normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(TORCH_TYPE[dtype])


def _pitch(K):
    """Bytes of a row of 8-bit codes: whole cache lines of 128."""
    return -(-K // 128) * 128


def _expert_choices(case, g):
    """Every token's k different experts, int32 [N, k]; dropped ones are -1."""
    N, k, E = case["N"], case["k"], case["E"]
    log_p = -case["skew"] * torch.log(torch.arange(1, E + 1, device=DEV, dtype=torch.float32))
    u = torch.rand((N, E), generator=g, device=DEV).clamp_(1e-9, 1 - 1e-7)
    ids = (log_p - torch.log(-torch.log(u))).topk(k, dim=1).indices.int()
    if case["dropped"]:
        ids[torch.rand((N, k), generator=g, device=DEV) < case["dropped"]] = -1
    return ids


def _sorted_by_expert(ids, E):
    """(offsets int32 [E + 1], src int32 [N k]) of the choices: by expert, then
    in their own order; dropped ones last."""
    key = torch.where((ids >= 0) & (ids < E), ids, E).reshape(-1)
    src = torch.argsort(key, stable=True)
    offsets = torch.searchsorted(key[src], torch.arange(E + 1, device=ids.device, dtype=key.dtype))
    return offsets.int(), src.int()


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    kind, N = case["kind"], case["N"]
    if kind in ("choose", "choose_grad"):
        k, E = case["k"], case["E"]
        s["logits"] = _normal((N, E), case["dtype"], g)
        if case["masked"]:
            s["logits"][torch.rand((N, E), generator=g, device=DEV) < case["masked"]] = -math.inf
        s["live"] = s["bias"] = None
        if case["padded"]:
            s["live"] = torch.rand(N, generator=g, device=DEV) >= case["padded"]
            s["logits"][~s["live"]] = math.nan
        if case["bias"]:
            s["bias"] = 0.2 * torch.randn(E, generator=g, device=DEV)
        if kind == "choose":
            s["ids"] = torch.empty((N, k), dtype=torch.int32, device=DEV)
            s["weights"] = torch.empty((N, k), device=DEV)
            if case["totals"]:
                s["counts"] = torch.empty(E + 1, dtype=torch.int32, device=DEV)
                s["sums"] = torch.empty(E + 1, device=DEV)
                s["losses"] = torch.empty(2, device=DEV)
                s["work"] = torch.empty(1 << 19, device=DEV)  # more than any plan asks for
            return s
        s["ids"] = _plain_choice(s)[0]
        s["counts"] = _plain_counts(s, s["ids"])
        # The gradient of a mean over the tokens, scaled as it is for training in 16 bits.
        s["dweights"] = torch.randn((N, k), generator=g, device=DEV)
        s["dlosses"] = torch.tensor((0.01 * N, 0.001 * N), device=DEV)
        s["dlogits"] = torch.empty_like(s["logits"])
        return s
    M, K, E = case["M"], case["K"], case.get("E", 1)
    rows = N if kind == "linear8" or case["gather"] else N * case["k"]
    s["codes"] = torch.randint(-127, 128, (E, M, _pitch(K)), generator=g, device=DEV, dtype=torch.int8)
    s["scales"] = (0.75 + 0.5 * torch.rand((E, M), generator=g, device=DEV)) / (73.3 * math.sqrt(K))
    s["x"] = _normal((rows, K), case["dtype"], g)
    s["xq"] = torch.empty((rows, _pitch(K)), dtype=torch.int8, device=DEV)
    s["xs"] = torch.empty(rows, device=DEV)
    wide = M // (2 if case["glu"] else 1)
    if kind == "experts8":
        s["offsets"], s["src"] = _sorted_by_expert(_expert_choices(case, g), E)
        # The most rows of an expert, for padding them to one length.
        s["most"] = max(1, int((s["offsets"][1:] - s["offsets"][:-1]).max()))
    s["y"] = torch.empty((N if kind == "linear8" else N * case["k"], wide), dtype=s["x"].dtype, device=DEV)
    return s


# -------------------------------------------------------------- plain forms

def _counted(s):
    """(logits in 32 bits with 0 in rows that do not count, which rows do)."""
    logits = s["logits"].float()
    rows = (logits > -math.inf).any(1)
    if s["live"] is not None:
        rows = rows & s["live"]
    return torch.where(rows[:, None], logits, 0.0), rows


def _plain_choice(s):
    """(experts int32 [N, k], logits, rows that count): ties go to the lower number."""
    logits, rows = _counted(s)
    score = logits + s["bias"] if s["bias"] is not None else logits + 0.0
    top, ids = torch.sort(score, dim=1, descending=True, stable=True)
    k = s["case"]["k"]
    ids = torch.where((top[:, :k] > -math.inf) & rows[:, None], ids[:, :k], -1)
    return ids.int(), logits, rows


def _plain_counts(s, ids):
    """Choices of each expert, and behind them the tokens that count, int32 [E + 1]."""
    E = s["case"]["E"]
    flat = ids.reshape(-1).long()
    counts = torch.bincount(torch.where(flat < 0, E, flat), minlength=E + 1)
    counts[E] = _counted(s)[1].sum()
    return counts.int()


def _softmax(v):
    """(softmax, log of the sum of exponentials) over the last dimension, one finite number in it at least."""
    top = v.amax(-1, keepdim=True)
    e = torch.exp(v - top)
    total = e.sum(-1, keepdim=True)
    return e / total, (top + torch.log(total))[..., 0]


def _plain_weights(logits, p, ids, normalise):
    at = ids.clamp(min=0).long()
    if not normalise:
        return torch.where(ids >= 0, p.gather(1, at), 0.0)
    chosen = torch.where(ids >= 0, logits.gather(1, at), -math.inf)
    none = ids[:, :1] < 0
    return torch.where(none, 0.0, _softmax(torch.where(none, 0.0, chosen))[0])


def _plain_choose(s):
    case = s["case"]
    ids, logits, rows = _plain_choice(s)
    p, lse = _softmax(logits)
    out = {"ids": ids, "weights": _plain_weights(logits, p, ids, case["normalise"])}
    if not case["totals"]:
        return out
    counts = _plain_counts(s, ids)
    sums = torch.cat((torch.where(rows[:, None], p, 0.0).sum(0), torch.where(rows, lse * lse, 0.0).sum()[None]))
    T = counts[-1].float().clamp(min=1)
    balance = (counts[:-1].float() * sums[:-1]).sum() * case["E"] / (case["k"] * T * T)
    return {**out, "counts": counts, "sums": sums, "losses": torch.stack((balance, sums[-1] / T))}


def _plain_choose_grad(s):
    case = s["case"]
    logits, rows = _counted(s)
    ids, counts = s["ids"], s["counts"].float()
    p, lse = _softmax(logits)
    w = _plain_weights(logits, p, ids, case["normalise"])
    T = counts[-1].clamp(min=1)
    dp = (s["dlosses"][0] * case["E"] / (case["k"] * T * T) * counts[:-1])[None].expand_as(p)
    dw = torch.where(ids >= 0, s["dweights"], 0.0)
    mean = (w * dw).sum(1, keepdim=True)
    direct = w * (dw - mean) if case["normalise"] else w * dw
    grad = p * (dp - (p * dp).sum(1, keepdim=True) + (2 * s["dlosses"][1] / T * lse)[:, None])
    if not case["normalise"]:
        grad = grad - p * mean
    grad = grad.scatter_add(1, ids.clamp(min=0).long(), torch.where(ids >= 0, direct, 0.0))
    return {"dlogits": torch.where(rows[:, None], grad, 0.0).to(s["logits"].dtype)}


def _plain_rounded(x):
    """(8-bit codes of every row as numbers, scales [rows, 1]), float32.  The
    quotients are of 64 bits: those of 32 round some to the middle of two codes."""
    x = x.double()
    scale = (x.abs().amax(1, keepdim=True) / 127.0).float()
    codes = torch.round(x / torch.where(scale > 0, scale, 1.0).double()).clamp(-127, 127)
    return codes.float(), scale


def _gated(y, case):
    if not case["glu"]:
        return y
    gate, up = y.chunk(2, dim=-1)
    return gate / (1 + torch.exp(-gate)) * up


def _plain_linear8(s):
    codes, scale = _plain_rounded(s["x"])
    y = codes @ s["codes"][0, :, :s["case"]["K"]].float().t()
    return {"y": _gated(y * scale * s["scales"][0], s["case"]).to(s["x"].dtype)}


def _plain_experts8(s):
    case = s["case"]
    codes, scale = _plain_rounded(s["x"])
    if case["gather"]:
        token = s["src"].long() // case["k"]
        codes, scale = codes[token], scale[token]
    offsets = s["offsets"].long()
    at = offsets[:-1, None] + torch.arange(s["most"], device=DEV)  # every expert's rows, padded to one length
    real = at < offsets[1:, None]
    at = at.clamp(max=codes.shape[0] - 1)
    rows = torch.where(real[..., None], codes[at], 0.0)
    weights = s["codes"][:, :, :case["K"]].float().transpose(1, 2).contiguous()
    y = torch.bmm(rows, weights) * scale[at] * s["scales"][:, None, :]
    y = _gated(y, case)
    p = torch.arange(codes.shape[0], device=DEV)
    e = (torch.searchsorted(offsets, p, right=True) - 1).clamp(max=case["E"] - 1)
    y = y[e, (p - offsets[e]).clamp(max=s["most"] - 1)]
    return {"y": torch.where((p < offsets[-1])[:, None], y, 0.0).to(s["x"].dtype)}


# ------------------------------------------------------ the framework's calls

@functools.lru_cache(maxsize=None)
def _perm(N, k, E):
    import paper_2305_06942_amd as ebag
    return ebag.MoePerm(N, k, E)


@functools.lru_cache(maxsize=None)
def _product(M, K, dtype, experts, glu):
    import paper_2305_06942_amd as ebag
    return ebag.Q8Gemv(M, K, ABI_TYPE[dtype], experts=experts, glu=int(glu))


def _own(s):
    case = s["case"]
    kind = case["kind"]
    if kind in ("choose", "choose_grad"):
        perm = _perm(case["N"], case["k"], case["E"])
        if kind == "choose_grad":
            perm.choose_backward(s["logits"], s["ids"], s["dweights"], s["dlogits"], counts=s["counts"],
                                 dlosses=s["dlosses"], live=s["live"], normalise=case["normalise"])
            return {"dlogits": s["dlogits"]}
        if not case["totals"]:
            perm.choose(s["logits"], s["ids"], s["weights"], bias=s["bias"], live=s["live"], normalise=case["normalise"])
            return {n: s[n] for n in ("ids", "weights")}
        perm.choose(s["logits"], s["ids"], s["weights"], counts=s["counts"], sums=s["sums"], losses=s["losses"],
                    work=s["work"], bias=s["bias"], live=s["live"], normalise=case["normalise"])
        return {n: s[n] for n in ("ids", "weights", "counts", "sums", "losses")}
    q = _product(case["M"], case["K"], case["dtype"], case.get("E", 1), case["glu"])
    if kind == "linear8":
        q.forward(s["codes"], s["scales"], s["x"], s["y"], s["xq"], s["xs"])
    else:
        q.experts(s["codes"], s["scales"], s["x"], s["offsets"], s["y"], s["xq"], s["xs"],
                  src=s["src"] if case["gather"] else None, k=case["k"])
    return {"y": s["y"]}


_PLAIN = {"choose": _plain_choose, "choose_grad": _plain_choose_grad, "linear8": _plain_linear8, "experts8": _plain_experts8}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------- bounds

def work(case):
    kind, elt, N = case["kind"], ELT[case["dtype"]], case["N"]
    if kind in ("choose", "choose_grad"):
        E, k = case["E"], case["k"]
        read = N * (1 - case["padded"]) * E * elt + (N if case["padded"] else 0)
        if kind == "choose":
            small = (4 * E if case["bias"] else 0) + (8 * (E + 1) + 8 if case["totals"] else 0)
            return {"bytes": read + 8 * N * k + small, "flops": 6 * N * E}
        return {"bytes": read + 8 * N * k + 4 * (E + 1) + 8 + N * E * elt, "flops": 8 * N * E}
    M, K = case["M"], case["K"]
    wide = M // (2 if case["glu"] else 1)
    matrix = M * (K + 4)
    if kind == "linear8":
        return {"bytes": matrix + N * (K + wide) * elt, "flops": 2 * N * M * K}
    E, k = case["E"], case["k"]
    S = N * k
    kept = S * (1 - case["dropped"])
    p = [(e + 1) ** -case["skew"] for e in range(E)]
    used = sum(1 - (1 - min(1.0, k * v / sum(p))) ** N for v in p)  # experts with rows, as expected
    rows = N if case["gather"] else kept
    return {"bytes": used * matrix + rows * K * elt + S * (wide * elt + 4) + 4 * (E + 1), "flops": 2 * kept * M * K}


# ------------------------------------------------------------ exact results

def _exact_places(score):
    """The place of every expert in its token's order: how many come before it."""
    places = []
    E = score.shape[1]
    lower = torch.arange(E, device=DEV)[:, None] < torch.arange(E, device=DEV)[None, :]  # [f, e]: f is the lower number
    step = max(1, (1 << 27) // (E * E))
    for at in range(0, score.shape[0], step):
        part = score[at:at + step]
        f, e = part[:, :, None], part[:, None, :]
        places.append(((f > e) | ((f == e) & lower)).sum(1))
    return torch.cat(places)


def _exact_rows(s):
    """The tokens that count: with an expert to choose, and no padding, which is NaN."""
    logits = s["logits"]
    return torch.nonzero((~torch.isnan(logits) & ~torch.isneginf(logits)).any(1))[:, 0]


def _exact_losses(logits, chosen, counts, k):
    """(probabilities, both losses) of tokens that count, in logits' 64 bits."""
    p = torch.softmax(logits, dim=1)
    T, E = max(1, logits.shape[0]), logits.shape[1]
    balance = E * ((counts / (k * T)) * (p.sum(0) / T)).sum()
    return p, torch.stack((balance, torch.logsumexp(logits, dim=1).square().sum() / T))


def _exact_weights(logits, p, ids, normalise):
    at = ids.clamp(min=0)
    if not normalise:
        return p.gather(1, at) * (ids >= 0)
    e = torch.exp(logits.gather(1, at) - logits.amax(1, keepdim=True).detach()) * (ids >= 0)
    return e / e.sum(1, keepdim=True)


def _exact_choose(s):
    case = s["case"]
    N, k, E = case["N"], case["k"], case["E"]
    here = _exact_rows(s)
    logits = s["logits"][here].double()
    score = s["logits"][here].float() + (0 if s["bias"] is None else s["bias"])
    place = _exact_places(score)
    ids = torch.full((here.numel(), k), -1, dtype=torch.long, device=DEV)
    n, e = torch.nonzero((place < k) & (score > -math.inf), as_tuple=True)
    ids[n, place[n, e]] = e
    counts = torch.stack([(ids == e).sum() for e in range(E)]).double()
    p, losses = _exact_losses(logits, ids, counts, k)
    weights = torch.zeros((N, k), dtype=torch.float64, device=DEV)
    weights[here] = _exact_weights(logits, p, ids, case["normalise"])
    out = {"ids": None, "weights": weights}
    if case["totals"]:
        lse2 = torch.logsumexp(logits, dim=1).square().sum()
        out.update(counts=None, sums=torch.cat((p.sum(0), lse2[None])), losses=losses)
    return out


def _exact_choose_grad(s):
    """By differentiation of what the gradients belong to, in 64 bits."""
    case = s["case"]
    here = _exact_rows(s)
    logits = s["logits"][here].double().requires_grad_()
    ids = s["ids"][here].long()
    p, losses = _exact_losses(logits, ids, s["counts"][:-1].double(), case["k"])
    w = _exact_weights(logits, p, ids, case["normalise"])
    total = (w * s["dweights"][here].double()).sum() + (losses * s["dlosses"].double()).sum()
    total.backward()
    grad = torch.zeros((case["N"], case["E"]), dtype=torch.float64, device=DEV)
    grad[here] = logits.grad
    return {"dlogits": grad}


def _exact_rounded(x):
    """What the rows' 8-bit codes stand for, and the codes' scales: the scale is rounded to 32 bits, the codes to whole numbers."""
    x = x.double()
    scale = (x.abs().max(dim=1).values / 127).float().double()
    codes = torch.where(scale[:, None] > 0, torch.round(x / scale[:, None]), 0.0)
    return codes.clamp(-127, 127) * scale[:, None]


def _exact_product(x, s, e):
    case = s["case"]
    matrix = s["codes"][e, :, :case["K"]].double() * s["scales"][e].double()[:, None]
    y = torch.matmul(_exact_rounded(x), matrix.t().contiguous())
    if case["glu"]:
        half = y.shape[1] // 2
        y = y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "choose":
        return _exact_choose(s)
    if kind == "choose_grad":
        return _exact_choose_grad(s)
    if kind == "linear8":
        return {"y": _exact_product(s["x"], s, 0)}
    y = torch.zeros(tuple(s["y"].shape), dtype=torch.float64, device=DEV)
    ends = s["offsets"].tolist()
    for e in range(case["E"]):
        lo, hi = ends[e], ends[e + 1]
        if lo < hi:
            token = torch.div(s["src"][lo:hi].long(), case["k"], rounding_mode="floor")
            y[lo:hi] = _exact_product(s["x"][token] if case["gather"] else s["x"][lo:hi], s, e)
    return {"y": y}
