"""The measured cases of the operators around the grouped experts and at the end of a training step.

Kinds of case:

  route    router logits to each token's top-k experts and weights, and the tokens sorted by
           expert (offsets and both directions of the permutation); with "grad" also the
           gradient of the logits from that of the weights
  experts  token rows copied to their experts' places and the experts' rows added up per token
           with the weights; with "grad" the backward pass of both: gradients of the experts'
           rows, of the weights and of the token rows
  loss     softmax cross entropy of hidden rows against a frozen vocabulary projection: loss
           and log-sum-exp per token; with "grad" also the gradient of the hidden rows

Shapes are the package's synthetic workloads' (128 experts of width 2048 routed top-8 and of
width 2880 routed top-4, hidden width 4096, batches of up to 16 x 2048 tokens) and generic ones
of the same range.
"""
import math

import torch

own = False


def listed():
    return [
        # a single token of a decoding step through 128 experts: launches and host calls count
        {"name": "route_token", "kind": "route", "T": 1, "E": 128, "k": 8, "bf16": False, "norm": True, "pad": 0.0, "grad": False},
        # one short training example with bf16 logits, which tie often
        {"name": "route_example", "kind": "route", "T": 187, "E": 128, "k": 4, "bf16": True, "norm": True, "pad": 0.1, "grad": True},
        # the full 16 x 2048 batch, some of it padding, weights not renormalised over the chosen experts
        {"name": "route_batch", "kind": "route", "T": 32768, "E": 128, "k": 8, "bf16": False, "norm": False, "pad": 0.06, "grad": True},
        # a single token of a decoding step: four rows out, four rows back
        {"name": "experts_token", "kind": "experts", "T": 1, "E": 128, "k": 4, "D": 2880, "pad": 0.0, "grad": False},
        # one sequence without its padding, forward only (evaluation, prompt of a served model)
        {"name": "experts_seq", "kind": "experts", "T": 1999, "E": 128, "k": 4, "D": 2880, "pad": 0.0, "grad": False},
        # the backward pass of one 2048-token sequence: the usual micro-batch
        {"name": "experts_seq_grad", "kind": "experts", "T": 2048, "E": 128, "k": 8, "D": 2048, "pad": 0.02, "grad": True},
        # the backward pass of the full batch, some of it padding
        {"name": "experts_batch_grad", "kind": "experts", "T": 32768, "E": 128, "k": 8, "D": 2048, "pad": 0.06, "grad": True},
        # the smallest head of the checks, forward and gradient
        {"name": "loss_tiny", "kind": "loss", "T": 64, "D": 512, "V": 8000, "ignored": 0.0, "grad": True},
        # the log-probability of one token (scoring a continuation): the vocabulary projection is read once
        {"name": "loss_token", "kind": "loss", "T": 1, "D": 4096, "V": 128256, "ignored": 0.0, "grad": False},
        # the loss of one sequence without its padding on a held-out set
        {"name": "loss_eval", "kind": "loss", "T": 1999, "D": 2048, "V": 151936, "ignored": 0.0, "grad": False},
        # one 2048-token sequence of a fine-tuning run, every token a target
        {"name": "loss_seq", "kind": "loss", "T": 2048, "D": 4096, "V": 128256, "ignored": 0.0, "grad": True},
        # four sequences of question and answer: only the answers' tokens are targets
        {"name": "loss_batch", "kind": "loss", "T": 8192, "D": 4096, "V": 128256, "ignored": 0.4, "grad": True},
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(("route", "experts", "experts", "loss", "loss"))
    grad = rng.random() < 0.6
    if kind == "route":
        E = rng.choice((8, 16, 60, 64, 128, 256))
        return {"kind": kind, "T": int(_log(rng, 1, 32768.5)), "E": E, "k": rng.choice((1, 2, 4, 6, 8)),
                "bf16": rng.random() < 0.5, "norm": rng.random() < 0.5, "pad": rng.choice((0.0, 0.05, 0.3)), "grad": grad}
    if kind == "experts":
        k, D = rng.choice((1, 2, 4, 6, 8)), 8 * int(_log(rng, 32, 512.5))
        most = min(32768, 32768 * 8 * 2048 // (k * D))
        return {"kind": kind, "T": int(_log(rng, 1, most + 0.5)), "E": rng.choice((8, 16, 60, 64, 128)), "k": k, "D": D,
                "pad": rng.choice((0.0, 0.05, 0.3)), "grad": grad}
    D, V = 8 * int(_log(rng, 32, 512.5)), int(_log(rng, 1000, 151936.5))
    most = min(8192, int(0.6 * 8192 * 4096 * 128256 / (D * V)))
    return {"kind": kind, "T": int(_log(rng, 1, most + 0.5)), "D": D, "V": V, "ignored": rng.choice((0.0, 0.2, 0.6)), "grad": grad}


# ------------------------------------------------------------------ inputs

def _logits(g, T, E, bf16):
    """Router logits with a log-normal spread of the experts' popularity."""
    z = torch.randn(T, E, generator=g, device="cuda") + 0.3 * torch.randn(E, generator=g, device="cuda")
    return z.bfloat16() if bf16 else z


def _valid(g, T, pad):
    """1 for tokens that are routed, 0 for padding (the first token always is one)."""
    v = torch.rand(T, generator=g, device="cuda") >= pad
    v[:1] = True
    return v.to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    T = case["T"]
    dev = "cuda"
    if case["kind"] == "loss":
        D, V = case["D"], case["V"]
        s["W"] = (torch.randn(V, D, generator=g, device=dev) * (2.0 / math.sqrt(D))).bfloat16()
        labels = torch.randint(V, (T,), generator=g, device=dev)
        # hidden rows of unit size that lean towards their label's row, some more than others: losses
        # from about 1 to above log(V), as of the tokens of one batch
        lean = torch.rand(T, 1, generator=g, device=dev) * (0.25 * math.log(V))
        X = torch.randn(T, D, generator=g, device=dev) + lean * s["W"][labels].float()
        s["X"] = X.bfloat16()
        ignored = torch.rand(T, generator=g, device=dev) < case["ignored"]
        ignored[:1] = False
        s["labels"] = torch.where(ignored, -100, labels)
        # the mean over the labelled tokens, the sequences weighted unequally
        weight = torch.rand(T, generator=g, device=dev) + 0.5
        s["dloss"] = torch.where(ignored, 0.0, weight / (~ignored).sum())
        s["loss"], s["lse"] = torch.empty(T, device=dev), torch.empty(T, device=dev)
        s["dX"] = torch.empty(T, D, dtype=torch.bfloat16, device=dev)
        return s
    E, k = case["E"], case["k"]
    valid = _valid(g, T, case["pad"])
    if case["kind"] == "route":
        s["logits"], s["valid"] = _logits(g, T, E, case["bf16"]), valid
        s["dweights"] = torch.randn(T, k, generator=g, device=dev) * 1e-3
        s["experts"] = torch.empty(T, k, dtype=torch.int32, device=dev)
        s["weights"] = torch.empty(T, k, device=dev)
        s["offsets"] = torch.empty(E + 1, dtype=torch.int64, device=dev)
        s["row_of"], s["slot_of"] = torch.empty_like(s["experts"]), torch.empty(T * k, dtype=torch.int32, device=dev)
        s["dlogits"] = torch.empty_like(s["logits"])
        return s
    D = case["D"]
    experts, s["weights"] = _route(_logits(g, T, E, False), valid, k, True)
    _, s["row_of"], s["slot_of"] = _sort(experts, E)
    act = lambda n, std: (torch.randn(n, D, generator=g, device=dev) * std).bfloat16()  # noqa: E731
    s["X"], s["Ys"] = act(T, 1.0), act(T * k, 0.5)
    s["Xs"], s["Y"] = torch.empty_like(s["Ys"]), torch.empty_like(s["X"])
    if case["grad"]:
        s["dY"], s["dXs"] = act(T, 1e-3), act(T * k, 1e-3)
        s["dYs"], s["dX"], s["dweights"] = s["Xs"], s["Y"], torch.empty_like(s["weights"])
    return s


# ------------------------------------------------------------------ one pass

_handle = None


def _h():
    """The one handle a program keeps."""
    global _handle
    if _handle is None:
        import paper_2609_04526_gb300 as pkg
        _handle = pkg.Handle()
    return _handle


def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "loss":
        return _loss(s["X"], s["W"], s["labels"], s["dloss"] if s["grad"] else None)
    if s["kind"] == "route":
        experts, weights = _route(s["logits"], s["valid"], s["k"], s["norm"])
        out = {"experts": experts, "weights": weights}
        out["offsets"], out["row_of"], out["slot_of"] = _sort(experts, s["E"])
        if s["grad"]:
            out["dlogits"] = _route_grad(s["logits"], experts, s["dweights"], s["norm"])
        return out
    if not s["grad"]:
        return {"Xs": _dispatch(s["X"], s["slot_of"], s["k"]), "Y": _combine(s["Ys"], s["row_of"], s["weights"])}
    dYs, dweights = _combine_grad(s["dY"], s["Ys"], s["row_of"], s["slot_of"], s["weights"])
    return {"dYs": dYs, "dweights": dweights, "dX": _combine(s["dXs"], s["row_of"], None)}


def _run_own(s):
    h = _h()
    if s["kind"] == "loss":
        if s["grad"]:
            h.sq_head_loss_grad(s["X"], s["W"], s["labels"], s["dloss"], loss=s["loss"], lse=s["lse"], dX=s["dX"])
            return {"loss": s["loss"], "lse": s["lse"], "dX": s["dX"]}
        h.sq_head_loss(s["X"], s["W"], s["labels"], loss=s["loss"], lse=s["lse"])
        return {"loss": s["loss"], "lse": s["lse"]}
    if s["kind"] == "route":
        h.sq_route(s["logits"], s["k"], normalize=s["norm"], valid=s["valid"], experts=s["experts"], weights=s["weights"])
        h.sq_sort_tokens(s["experts"], s["E"], offsets=s["offsets"], row_of=s["row_of"], slot_of=s["slot_of"])
        out = {n: s[n] for n in ("experts", "weights", "offsets", "row_of", "slot_of")}
        if s["grad"]:
            h.sq_route_grad(s["logits"], s["experts"], s["dweights"], normalize=s["norm"], dlogits=s["dlogits"])
            out["dlogits"] = s["dlogits"]
        return out
    if not s["grad"]:
        h.sq_dispatch(s["X"], s["row_of"], s["slot_of"], Xs=s["Xs"])
        h.sq_combine(s["Ys"], s["row_of"], s["weights"], Y=s["Y"])
        return {"Xs": s["Xs"], "Y": s["Y"]}
    h.sq_combine_grad(s["dY"], s["Ys"], s["row_of"], s["slot_of"], s["weights"], dYs=s["dYs"], dweights=s["dweights"])
    h.sq_dispatch_grad(s["dXs"], s["row_of"], dX=s["dX"])
    return {"dYs": s["dYs"], "dweights": s["dweights"], "dX": s["dX"]}


# ------------------------------------------------------------------ plain forms

def _route(logits, valid, k, norm):
    """Top-k of each valid token's logits, ties to the lowest expert; softmax weights over all
    experts, or over the chosen ones (norm). A token that is not valid has experts -1, weights 0."""
    on = valid.bool()[:, None]
    z = logits.float()
    top, experts = torch.sort(z, dim=1, descending=True, stable=True)
    e = torch.exp(top - top[:, :1])
    weights = e[:, :k] / (e[:, :k] if norm else e).sum(1, keepdim=True)
    return torch.where(on, experts[:, :k], -1).int(), torch.where(on, weights, 0.0)


def _route_grad(logits, experts, dweights, norm):
    on = experts >= 0
    at = experts.clamp(min=0).long()
    z = logits.float()
    full = torch.softmax(z, dim=1) if not norm else torch.zeros_like(z).scatter_(1, at, torch.softmax(z.gather(1, at), dim=1))
    dw = torch.zeros_like(z).scatter_(1, at, torch.where(on, dweights, 0.0))
    return (full * (dw - (full * dw).sum(1, keepdim=True)) * on[:, :1]).to(logits.dtype)


def _sort(experts, E):
    """Slots t * k + j in the order of their experts, equal ones as they come. Returns offsets
    [E + 1], each slot's row (-1: none) and each row's slot (-1: past the last routed slot)."""
    e = experts.reshape(-1).long()
    key = torch.where(e < 0, E, e)
    order = torch.argsort(key, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.int64, device=e.device).scatter_add_(0, key, torch.ones_like(key))
    offsets = torch.cat([counts.new_zeros(1), counts[:E].cumsum(0)])
    rows = torch.arange(e.numel(), device=e.device)
    row_of = torch.empty_like(e).scatter_(0, order, torch.where(rows < offsets[E], rows, -1))
    return offsets, row_of.view(experts.shape).int(), torch.where(rows < offsets[E], order, -1).int()


def _dispatch(X, slot_of, k):
    token = torch.div(slot_of.clamp(min=0), k, rounding_mode="floor").long()
    return torch.where((slot_of >= 0)[:, None], X.float()[token], 0.0).to(X.dtype)


def _combine(Ys, row_of, weights):
    rows = torch.where((row_of >= 0)[..., None], Ys.float()[row_of.clamp(min=0).long()], 0.0)
    return (rows if weights is None else rows * weights[..., None]).sum(1).to(Ys.dtype)


def _combine_grad(dY, Ys, row_of, slot_of, weights):
    k = row_of.shape[1]
    slot = slot_of.clamp(min=0).long()
    dy = dY.float()
    dYs = torch.where((slot_of >= 0)[:, None], dy[torch.div(slot, k, rounding_mode="floor")] * weights.reshape(-1)[slot][:, None], 0.0)
    rows = Ys.float()[row_of.clamp(min=0).long()]
    return dYs.to(Ys.dtype), torch.where(row_of >= 0, (rows * dy[:, None]).sum(2), 0.0)


def _loss(X, W, labels, dloss):
    on = labels >= 0
    at = labels.clamp(min=0)
    W32 = W.float()
    z = X.float() @ W32.t()
    top = z.max(1).values
    e = torch.exp(z - top[:, None])
    total = e.sum(1)
    lse = torch.where(on, top + torch.log(total), 0.0)
    loss = torch.where(on, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    if dloss is None:
        return {"loss": loss, "lse": lse}
    d = e * (dloss / total)[:, None]
    d.scatter_add_(1, at[:, None], -dloss[:, None])
    dX = torch.where(on[:, None], d @ W32, 0.0).to(X.dtype)
    return {"loss": loss, "lse": lse, "dX": dX}


# ------------------------------------------------------------------ work and exact results

def work(case):
    T = case["T"]
    if case["kind"] == "loss":
        D, V = case["D"], case["V"]
        on = max(1.0, T * (1.0 - case["ignored"]))
        passes = 2 if case["grad"] else 1
        return {"bytes": 2 * V * D + 2 * on * D + 16 * T + (2 * T * D + 4 * T if case["grad"] else 0), "flops": passes * 2.0 * on * D * V}
    E, k = case["E"], case["k"]
    on = max(1.0, T * (1.0 - case["pad"]))
    if case["kind"] == "route":
        size = 2 if case["bf16"] else 4
        fwd = on * E * size + T + T * k * (4 + 4 + 4 + 4) + 8 * (E + 1)
        # the gradient reads the logits again: a training step has the experts' work in between
        back = on * E * size + T * E * size + T * k * 8
        return {"bytes": fwd + (back if case["grad"] else 0), "flops": 4.0 * T * E}
    D = case["D"]
    if not case["grad"]:
        # rows out: the tokens read, T k rows written; rows back: the routed rows read, T written
        return {"bytes": 2 * D * (on + T * k + on * k + T) + T * k * 12, "flops": 2.0 * on * k * D}
    # dY and the experts' rows read, T k rows written; then the routed rows read, T written
    return {"bytes": 2 * D * (on + on * k + T * k + on * k + T) + T * k * 16, "flops": 5.0 * on * k * D}


def exact(case, seed):
    if case["kind"] == "loss" and case["T"] * case["D"] * case["V"] * (4.0 if case["grad"] else 2.0) > 8e12:
        return None  # 64-bit products of this size take too long
    s = prepare(case, seed)
    if case["kind"] == "loss":
        X, W, y = s["X"].double(), s["W"].double(), s["labels"]
        parts = []
        for first in range(0, case["T"], 512):
            x, lab, w = X[first:first + 512], y[first:first + 512], s["dloss"][first:first + 512].double()
            z = torch.mm(x, W.T)
            lse = torch.logsumexp(z, dim=1)
            logp = z - lse[:, None]
            keep = (lab != -100).double()
            here = torch.arange(len(lab), device=lab.device)
            nll = -logp[here, lab.clamp(min=0)]
            part = {"loss": torch.where(keep > 0, nll, 0.0), "lse": torch.where(keep > 0, lse, 0.0)}
            if case["grad"]:
                p = logp.exp()
                p[here, lab.clamp(min=0)] -= 1.0
                part["dX"] = torch.mm(p * (w * keep)[:, None], W)
            parts.append(part)
        return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}
    k = case["k"]
    if case["kind"] == "route":
        z = s["logits"].double()
        p = torch.softmax(z, dim=1)
        # rank of an expert: how many are larger, or equal and before it; done in pieces of tokens
        ranks = []
        for first in range(0, case["T"], 1024):
            c = z[first:first + 1024]
            ahead = c[:, None, :] > c[:, :, None]
            before = torch.ones(case["E"], case["E"], dtype=torch.bool, device=z.device).tril(-1)
            ranks.append((ahead | ((c[:, None, :] == c[:, :, None]) & before)).sum(2))
        rank = torch.cat(ranks)
        live = s["valid"] != 0
        experts = torch.zeros(case["T"], case["E"], dtype=torch.int64, device=z.device)
        experts.scatter_(1, rank, torch.arange(case["E"], device=z.device).expand_as(rank).contiguous())
        experts = experts[:, :k]
        chosen = rank < k
        share = p * chosen
        total = share.sum(1, keepdim=True) if case["norm"] else torch.ones_like(p[:, :1])
        weights = torch.gather(share / total, 1, experts) * live[:, None]
        out = {"experts": torch.where(live[:, None], experts, -1).int(), "weights": weights, "offsets": None, "row_of": None, "slot_of": None}
        if case["grad"]:
            dw = torch.zeros_like(p).scatter_(1, experts, s["dweights"].double())
            q = share / total if case["norm"] else p
            out["dlogits"] = q * (dw - (q * dw).sum(1, keepdim=True)) * live[:, None]
        return out
    rows, slots, w = s["row_of"].long(), s["slot_of"].long(), s["weights"].double()
    used = slots[slots >= 0]
    back = torch.zeros(case["T"], case["D"], dtype=torch.float64, device="cuda")
    if not case["grad"]:
        back.index_add_(0, used // k, s["Ys"][:len(used)].double() * w.reshape(-1)[used][:, None])
        return {"Xs": None, "Y": back}
    back.index_add_(0, used // k, s["dXs"][:len(used)].double())
    dYs = torch.zeros(case["T"] * k, case["D"], dtype=torch.float64, device="cuda")
    dYs[:len(used)] = s["dY"].double()[used // k] * w.reshape(-1)[used][:, None]
    dweights = torch.zeros(case["T"] * k, dtype=torch.float64, device="cuda")
    dweights[used] = (s["Ys"][:len(used)].double() * s["dY"].double()[used // k]).sum(1)
    return {"dYs": dYs, "dweights": dweights.view(rows.shape), "dX": back}
