"""Performance cases of the operators around a layer of experts -- the router's choice, tokens sorted by expert and back -- and of the
global gradient norm with clipping.

A router has a logit for each of E experts and every token; a token goes to k of them, so there are T k slots. The rows that the
experts multiply are sorted by expert, those of one expert in the order of their slots, and rows[t][j] says where slot j of
token t went (-1: nowhere).

  route         ids = the k largest of p = softmax(logits[t]), ties to the lowest index, weights p[ids], or those over their sum; a logit
                of -inf is never chosen (id -1, weight 0)
  route_grad    the gradient of the logits from that of the weights
  dispatch      ids -> offsets [E + 1], rows [T][k], Xs[rows[t][j]] = X[t]
  combine       Y[t] = add[t] + sum over j of weights[t][j] Ys[rows[t][j]]; without weights it is the way back of dispatch
  combine_grad  dYs[rows[t][j]] = weights[t][j] dY[t], dweights[t][j] = <dY[t], Ys[rows[t][j]]>
  norm          norm = the root of the sum of all tensors' squares times `scale`, coef = scale min(1, max_norm / norm)
  clip          norm, and every gradient times coef, in the buffers that the next step takes

Rows that no slot has are left as they were.
"""
import math
import random

import torch

own = False

MAX_NORM = 1.0


# ---------------------------------------------------------------- the cases
def route_case(name, op, tokens, experts, k, normalize, bf16, masked=0, padding=0):
    c = dict(op=op, tokens=tokens, experts=experts, k=k, normalize=normalize, bf16=bf16, masked=masked, padding=padding)
    return dict(c, name=name) if name else c


def token_case(name, op, tokens, experts, k, d, bf16, skew=0.5, padding=0, add=False, weighted=True):
    c = dict(op=op, tokens=tokens, experts=experts, k=k, d=d, bf16=bf16, skew=skew, padding=padding, add=add, weighted=weighted)
    return dict(c, name=name) if name else c


def list_case(name, op, net, sizes, bf16, bf16_out=False):
    c = dict(op=op, net=net, sizes=sizes, bf16=bf16, bf16_out=bf16_out)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: the tokens of sixteen requests, one each
        route_case("route_decode", "route", 16, 64, 4, True, False),
        # a training batch, the logits in bf16, a few experts out of use, the end of the batch padding
        route_case("route_large", "route", 65536, 128, 8, False, True, masked=3, padding=500),
        # its way back
        route_case("route_grad_large", "route_grad", 65536, 128, 8, False, True, masked=3, padding=500),
        # serving: eight tokens to two experts each
        token_case("dispatch_decode", "dispatch", 8, 8, 2, 2048, True),
        # a training batch of wide tokens
        token_case("dispatch_large", "dispatch", 16384, 64, 4, 4096, True, skew=1.0, padding=100),
        # serving: back from the two experts, onto the residual stream
        token_case("combine_decode", "combine", 8, 8, 2, 2048, True, add=True),
        # a training batch of wide tokens, back
        token_case("combine_large", "combine", 16384, 64, 4, 4096, True, skew=1.0, padding=100),
        # gradients of that
        token_case("combine_grad_large", "combine_grad", 16384, 64, 4, 4096, True, skew=1.0, padding=100),
        # fp32 and the odd width of a small network's layer, few tokens
        token_case("combine_grad_f32", "combine_grad", 1000, 10, 2, 577, False, skew=1.0, padding=7),
        # a small network: 34 tensors, most of them a few hundred to a few thousand gradients
        list_case("norm_small", "norm", "basic", "16,5,10", False),
        # the gradients of 32 experts of 2048 x 2048, up and down, in bf16
        list_case("norm_experts", "norm", "experts", "32,2048,2048,2", True),
        # the gradients of ResNet-50, clipped into the buffers that the preconditioner takes in place
        list_case("clip_resnet50", "clip", "bottleneck", "64,3,4,6,3,1000", False),
    ]


def log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: tokens from a single one to a training batch, counts of experts and choices, widths odd and even, a list of tensors."""
    op = rng.choice(["route", "route_grad", "dispatch", "combine", "combine_grad", "norm", "clip"])
    bf16 = rng.random() < 0.6
    for _ in range(1000):
        if op in ("norm", "clip"):
            net = rng.choice(["basic", "bottleneck", "experts"])
            if net == "basic":
                sizes = (log_int(rng, 8, 64), rng.randint(1, 5), rng.choice([10, 100]))
            elif net == "bottleneck":
                sizes = (log_int(rng, 12, 64), rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 6), rng.randint(1, 3), 1000)
            else:
                sizes = (log_int(rng, 1, 32), log_int(rng, 100, 2048), log_int(rng, 100, 2048), rng.randint(1, 2))
            c = list_case(None, op, net, ",".join(map(str, sizes)), bf16, rng.random() < 0.3)
            if work(c)["bytes"] < 1.2e9:
                return c
            continue
        tokens, experts = log_int(rng, 1, 65536), log_int(rng, 2, 512)
        k = min(rng.choice([1, 2, 2, 4, 6, 8]), experts)
        padding = rng.choice([0, 0, rng.randint(0, tokens // 8)])
        if op in ("route", "route_grad"):
            # (a single choice has the weight 1 after normalizing, and a single expert 1 before; its gradient is 0)
            return route_case(None, op, tokens, experts, k, k > 1 and rng.random() < 0.5, bf16, masked=rng.choice([0, 0, rng.randint(0, experts - 2)]), padding=padding)
        d = log_int(rng, 64, 4096)
        if rng.random() < 0.4:
            d += 8 - d % 8
        c = token_case(None, op, tokens, experts, k, d, bf16, skew=round(rng.uniform(0.0, 1.5), 2), padding=padding, add=op == "combine" and rng.random() < 0.5,
                       weighted=op != "combine" or rng.random() < 0.7)
        if work(c)["bytes"] < 1.2e9:
            return c
    raise RuntimeError("no case was found")


def tensor_shapes(case):
    """[d_out][d_in + 1] of every layer of a network, or the weights of experts without biases."""
    n = [int(v) for v in case["sizes"].split(",")]
    if case["net"] == "experts":                          # experts, d_in, d_out, layers
        return [(n[0], n[2], n[1])] * n[3]
    if case["net"] == "basic":                            # width, blocks per stage, classes: 3 x 3 convolutions, projections, FC
        width, blocks, classes = n
        out, c = [(width, 28)], width
        for s in range(3):
            w = width << s
            for b in range(blocks):
                out.append((w, 9 * c + 1))
                if s > 0 and b == 0:
                    out.append((w, c + 1))
                out.append((w, 9 * w + 1))
                c = w
        return out + [(classes, c + 1)]
    width, blocks, classes = n[0], n[1:5], n[5]           # width, four block counts, classes: bottleneck blocks, FC
    out, c = [(width, 148)], width
    for s, nb in enumerate(blocks):
        w = width << s
        for b in range(nb):
            out += [(w, c + 1), (w, 9 * w + 1), (4 * w, w + 1)]
            if b == 0:
                out.append((4 * w, c + 1))
            c = 4 * w
    return out + [(classes, c + 1)]


def work(case):
    es = 2 if case["bf16"] else 4
    if case["op"] in ("norm", "clip"):
        n = sum(math.prod(s) for s in tensor_shapes(case))
        return {"bytes": n * (es + (0 if case["op"] == "norm" else 2 if case["bf16_out"] else 4)), "flops": n * (2 if case["op"] == "norm" else 3)}
    T, E, k = case["tokens"], case["experts"], case["k"]
    S, live = T * k, T - case["padding"]
    if case["op"] == "route":
        return {"bytes": es * T * E + 8 * S, "flops": T * E * (4 + k)}
    if case["op"] == "route_grad":
        read = es * S if case["normalize"] else es * T * E                # of the logits
        return {"bytes": es * T * E + 8 * S + read, "flops": T * (4 * k if case["normalize"] else 6 * E)}
    d = case["d"]
    if case["op"] == "dispatch":
        return {"bytes": 8 * S + 4 * (E + 1) + es * d * live * (1 + k), "flops": 0}
    if case["op"] == "combine":
        return {"bytes": (8 if case["weighted"] else 4) * S + es * d * (live * k + T * (2 if case["add"] else 1)), "flops": 2 * d * live * k}
    return {"bytes": 12 * S + es * d * live * (1 + 2 * k), "flops": 3 * d * live * k}


# ---------------------------------------------------------------- inputs
def sort_rows(ids, experts):
    """(offsets [E + 1], rows as ids) of slots sorted by expert."""
    flat = ids.reshape(-1).long()
    flat = torch.where(flat < 0, experts, flat)
    order = torch.argsort(flat, stable=True)
    rows = torch.empty_like(order)
    rows[order] = torch.arange(order.numel(), device=order.device)
    rows = torch.where(flat < experts, rows, -1)
    counts = (flat[:, None] == torch.arange(experts, device=flat.device)).sum(0) if flat.numel() * experts < 1 << 26 else torch.bincount(flat, minlength=experts + 1)[:experts]
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device=flat.device), torch.cumsum(counts, 0)])
    return offsets.int(), rows.int().view(ids.shape)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, sigma=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device="cuda").mul_(sigma).to(dtype)

    st = dict(case=case)
    dt = torch.bfloat16 if case["bf16"] else torch.float32
    if case["op"] in ("norm", "clip"):
        # gradients whose size differs from tensor to tensor and from row to row by orders of magnitude; a loss scale still on them
        shapes, odt = tensor_shapes(case), torch.bfloat16 if case["bf16_out"] else torch.float32
        st["grads"] = [(normal(*s) * (torch.exp2(normal(*s[:-1], 1, sigma=2.0)) * 1e-3)).to(dt) for s in shapes]
        st["scale"] = torch.rand(1, generator=gen, device="cuda") + 0.5
        st["norm"], st["coef"] = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        st["out"] = [torch.zeros(s, dtype=odt, device="cuda") for s in shapes] if case["op"] == "clip" else None
        st["items"] = None
        return st
    T, E, k = case["tokens"], case["experts"], case["k"]
    live = T - case["padding"]
    if case["op"] in ("route", "route_grad"):
        logits = normal(T, E, sigma=2.0)
        if case["masked"]:
            logits[:, torch.randperm(E, generator=gen, device="cuda")[:case["masked"]]] = -math.inf
        logits[live:] = -math.inf
        st["logits"] = logits.to(dt)
        if case["op"] == "route":
            st["ids"] = torch.zeros(T, k, dtype=torch.int32, device="cuda")
            st["weights"] = torch.zeros(T, k, device="cuda")
        else:
            st["ids"] = plain_route(st["logits"], k, case["normalize"])[0]
            st["dweights"] = normal(T, k)
            st["dlogits"] = torch.zeros_like(st["logits"])
        return st
    # experts are not equally popular, and a token's choices are different ones
    popular = normal(E, sigma=case["skew"])
    ids = torch.topk(normal(T, E) + popular, k, dim=1)[1].int()
    ids[live:] = -1
    d = case["d"]
    st["ids"] = ids
    if case["op"] == "dispatch":
        st["X"] = normal(T, d, dtype=dt)
        st["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        st["rows"] = torch.zeros(T, k, dtype=torch.int32, device="cuda")
        st["Xs"] = torch.zeros(T * k, d, dtype=dt, device="cuda")
        return st
    st["rows"] = sort_rows(ids, E)[1]
    st["weights"] = torch.softmax(normal(T, k), 1) if case["weighted"] else None
    st["Ys"] = normal(T * k, d, dtype=dt)
    if case["op"] == "combine":
        st["Y"] = torch.zeros(T, d, dtype=dt, device="cuda")
        st["add"] = normal(T, d, dtype=dt) if case["add"] else None
    else:
        st["dY"] = normal(T, d, sigma=0.05, dtype=dt)
        st["dYs"] = torch.zeros(T * k, d, dtype=dt, device="cuda")
        st["dweights"] = torch.zeros(T, k, device="cuda")
    return st


# ---------------------------------------------------------------- the plain forms
def plain_softmax(x):
    """Over rows; a row without anything is zero."""
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    s = e.sum(1, keepdim=True)
    return e / torch.where(s > 0, s, 1.0)


def plain_route(logits, k, normalize):
    x = logits.float()
    top, ids = torch.sort(x, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k]
    w = plain_softmax(top.contiguous()) if normalize else torch.gather(plain_softmax(x), 1, ids)
    return torch.where(top > -math.inf, ids, -1).int(), w


def plain_route_grad(st):
    x, ids, dw = st["logits"].float(), st["ids"].long(), st["dweights"]
    has = ids >= 0
    at = ids.clamp(min=0)
    if st["case"]["normalize"]:
        w = plain_softmax(torch.where(has, torch.gather(x, 1, at), -math.inf))
        g = w * (dw - (w * dw).sum(1, keepdim=True))
        return torch.zeros_like(x).scatter_add_(1, at, torch.where(has, g, 0.0)).to(st["logits"].dtype)
    p = plain_softmax(x)
    g = torch.where(has, dw, 0.0)
    inner = (torch.gather(p, 1, at) * g).sum(1, keepdim=True)
    return (p * (torch.zeros_like(p).scatter_add_(1, at, g) - inner)).to(st["logits"].dtype)


def plain_dispatch(st):
    offsets, rows = sort_rows(st["ids"], st["case"]["experts"])
    slot = torch.nonzero(rows.view(-1) >= 0).view(-1)
    st["Xs"][rows.view(-1)[slot].long()] = st["X"][slot // st["case"]["k"]]
    return [offsets, rows, st["Xs"]]


def taken(st):
    """(Ys[rows] in 32 bits, zero where there is none, and whether there is one) for every slot, [T, k, d] and [T, k]."""
    has = st["rows"] >= 0
    x = st["Ys"][st["rows"].clamp(min=0).long().view(-1)].view(*st["rows"].shape, -1).float()
    return x * has[:, :, None], has


def plain_combine(st):
    x = taken(st)[0]
    y = (x if st["weights"] is None else x * st["weights"][:, :, None]).sum(1)
    st["Y"].copy_(y if st["add"] is None else y + st["add"].float())
    return st["Y"]


def plain_combine_grad(st):
    x, has = taken(st)
    dy = st["dY"].float()[:, None, :]
    slot = torch.nonzero(has.view(-1)).view(-1)
    st["dYs"][st["rows"].view(-1)[slot].long()] = (dy * st["weights"][:, :, None]).to(st["dYs"].dtype).view(-1, x.shape[2])[slot]
    return [st["dYs"], (x * dy).sum(2)]


def plain_norm(st):
    flat = torch.cat([g.reshape(-1) for g in st["grads"]])
    scale = st["scale"].double()
    norm = flat.double().square().sum().sqrt() * scale
    coef = scale * torch.clamp(MAX_NORM / norm, max=1.0)
    if st["out"] is None:
        return [norm.float(), coef.float()]
    flat = flat.float() * coef.float()
    parts = torch.split(flat, [g.numel() for g in st["grads"]])
    return [norm.float(), coef.float()] + [p.view(o.shape).to(o.dtype) for p, o in zip(parts, st["out"])]


# ---------------------------------------------------------------- the framework's calls
_context = None


def context():
    """The library context that a training program keeps, with its workspace."""
    global _context
    if _context is None:
        from paper_2007_00784_amd import kfac as K
        ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        _context = (K, K.kfac_create(torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream, ws), ws)
    return _context


def own_run(st):
    K, ctx, _ = context()
    op = st["case"]["op"]
    if op == "route":
        K.kfac_experts_route(ctx, st["logits"], st["ids"], st["weights"], normalize=st["case"]["normalize"])
        return [st["ids"], st["weights"]]
    if op == "route_grad":
        K.kfac_experts_route_grad(ctx, st["logits"], st["ids"], st["dweights"], st["dlogits"], normalize=st["case"]["normalize"])
        return st["dlogits"]
    if op == "dispatch":
        K.kfac_experts_dispatch(ctx, st["ids"], st["X"], st["offsets"], st["rows"], st["Xs"])
        return [st["offsets"], st["rows"], st["Xs"]]
    if op == "combine":
        K.kfac_experts_combine(ctx, st["Ys"], st["rows"], st["weights"], st["Y"], add=st["add"])
        return st["Y"]
    if op == "combine_grad":
        K.kfac_experts_combine_grad(ctx, st["dY"], st["Ys"], st["rows"], st["weights"], st["dYs"], st["dweights"])
        return [st["dYs"], st["dweights"]]
    if st["items"] is None:                                # marshalled once for the buffers of a model
        st["items"] = K.grad_items(st["grads"], st["out"])
    if op == "norm":
        K.kfac_grad_norm_batched(ctx, st["items"], st["norm"], max_norm=MAX_NORM, grad_scale=st["scale"], coef=st["coef"])
        return [st["norm"][0], st["coef"][0]]
    K.kfac_clip_grads_batched(ctx, st["items"], MAX_NORM, st["norm"], st["coef"], grad_scale=st["scale"])
    return [st["norm"][0], st["coef"][0]] + st["out"]


def plain_run(st):
    op = st["case"]["op"]
    if op == "route":
        return list(plain_route(st["logits"], st["case"]["k"], st["case"]["normalize"]))
    if op == "route_grad":
        return plain_route_grad(st)
    if op == "dispatch":
        return plain_dispatch(st)
    if op == "combine":
        return plain_combine(st)
    if op == "combine_grad":
        return plain_combine_grad(st)
    out = plain_norm(st)
    return [x.view(()) for x in out[:2]] + out[2:]


def run(st):
    return own_run(st) if own else plain_run(st)


# ---------------------------------------------------------------- the definition in 64 bits
def exact_choice(logits, k):
    """ids [T, k]: one expert after another, the first of the largest that are left."""
    left = logits.double().clone()
    ids = []
    for _ in range(k):
        best = left.amax(1, keepdim=True)
        first = (left == best).to(torch.uint8).argmax(1)
        ids.append(torch.where(best[:, 0] > -math.inf, first, -1))
        left.scatter_(1, first[:, None], -math.inf)
    return torch.stack(ids, 1).int()


def exact_weights(logits, ids, normalize):
    """(weights [T, k], p [T, E]) by the logarithm of the sum of exponentials."""
    x, at = logits.double(), ids.clamp(min=0).long()
    lse = torch.logsumexp(x, 1, keepdim=True)
    p = torch.where(x > -math.inf, torch.exp(x - lse), 0.0)
    w = torch.where(ids >= 0, torch.gather(p, 1, at), 0.0)
    return (w / w.sum(1, keepdim=True).clamp(min=1e-300) if normalize else w), p


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "route":
        ids = exact_choice(st["logits"], case["k"])
        return [ids, exact_weights(st["logits"], ids, case["normalize"])[0]]
    if op == "route_grad":
        # the Jacobian, one choice after another
        ids = exact_choice(st["logits"], case["k"])
        w, p = exact_weights(st["logits"], ids, case["normalize"])
        out = torch.zeros_like(p)
        hit = torch.zeros_like(p)
        for j in range(case["k"]):
            hit.scatter_add_(1, ids[:, j:j + 1].clamp(min=0).long(), (ids[:, j:j + 1] >= 0).double())
        for j in range(case["k"]):
            g = st["dweights"][:, j:j + 1].double() * w[:, j:j + 1]
            others = p * hit / (p * hit).sum(1, keepdim=True).clamp(min=1e-300) if case["normalize"] else p
            out -= g * others
            out.scatter_add_(1, ids[:, j:j + 1].clamp(min=0).long(), torch.where(ids[:, j:j + 1] >= 0, g, 0.0))
        return out
    if op in ("norm", "clip"):
        scale = float(st["scale"])
        norm = scale * math.sqrt(sum(float(g.double().norm()) ** 2 for g in st["grads"]))
        coef = scale * min(1.0, MAX_NORM / norm)
        out = [torch.tensor(v, dtype=torch.float64, device="cuda") for v in (norm, coef)]
        return out + ([] if st["out"] is None else [g.double() * coef for g in st["grads"]])
    E, k = case["experts"], case["k"]
    flat = st["ids"].view(-1).long()
    S = flat.numel()
    key = torch.where(flat >= 0, flat, E) * S + torch.arange(S, device="cuda")    # all different, in the order of the rows
    rows = torch.searchsorted(torch.sort(key)[0], key)
    rows = torch.where(flat >= 0, rows, -1)
    if op == "dispatch":
        offsets = torch.searchsorted(torch.sort(key)[0], torch.arange(E + 1, device="cuda") * S)
        Xs = st["Xs"].double()
        for j in range(k):
            r = rows.view(-1, k)[:, j]
            Xs[r[r >= 0]] = st["X"].double()[r >= 0]
        return [offsets.int(), rows.int().view(-1, k), Xs]
    rows = rows.view(-1, k)
    if op == "combine":
        y = torch.zeros(st["Y"].shape, dtype=torch.float64, device="cuda") if st["add"] is None else st["add"].double()
        for j in range(k):
            t = torch.nonzero(rows[:, j] >= 0).view(-1)
            y[t] += (1.0 if st["weights"] is None else st["weights"][t, j, None].double()) * st["Ys"][rows[t, j]].double()
        return y
    if op == "combine_grad":
        dYs, dw = st["dYs"].double(), torch.zeros(st["dweights"].shape, dtype=torch.float64, device="cuda")
        for j in range(k):
            t = torch.nonzero(rows[:, j] >= 0).view(-1)
            dy = st["dY"][t].double()
            dYs[rows[t, j]] = st["weights"][t, j, None].double() * dy
            dw[t, j] = (dy * st["Ys"][rows[t, j]].double()).sum(1)
        return [dYs, dw]
