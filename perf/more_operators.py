"""A model's two ends and the update of its matrices, as cases to be timed and compared: the lookup of
token rows with its gradient, the softmax cross entropy of a large vocabulary from the hidden states
with both of its gradients, and the orthogonalised update of a matrix by Newton-Schulz products.

``own`` chooses between two forms of the same pass: False computes it with elementary torch operations
in 32 bits (norms over whole matrices in 64), rounded once at the end; True makes the calls of this
library.  ``exact`` is the same arithmetic from the definitions, in 64 bits.

Inputs are made on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EMBED = dict(T=32, vocab=32000, d=2048, w_bf16=True, o_bf16=True, scale=1.0, none=0.0)
HEAD = dict(T=16, vocab=50000, d=2048, x_bf16=True, g_bf16=False, scale=1.0, none=0.0)
ORTH = dict(op="orth", n=1, rows=1024, cols=1024, g_bf16=False, o_bf16=False, steps=5, decay=0.0, scale=1.0)
# The quintic whose five steps take singular values from 0.01 to 1 near 1.
COEF = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def listed():
    return [
        # the new token of each of 32 sequences: only latency
        dict(EMBED, op="embed", name="embed-decode-32"),
        # prompts of many requests, rows of an odd width, some places padded
        dict(EMBED, op="embed", name="embed-prompts-16381x1023", T=16381, d=1023, w_bf16=False, o_bf16=False,
             scale=math.sqrt(1023), none=0.05),
        # a training step's tokens into the gradient of the table, which holds the head's already
        dict(EMBED, op="embed_back", name="embed-back-8192x2048", T=8192, vocab=50000, scale=1.5),
        # the same as compact rows for the clipping and a sparse optimiser step, many places padded
        dict(EMBED, op="embed_rows", name="embed-rows-20000x1024", T=20000, d=1024, o_bf16=False, none=0.2),
        # the log-probabilities of the 16 tokens that a draft proposed: the head's weight is read once
        dict(HEAD, op="loss", name="loss-decode-16"),
        # the perplexity of prompts, fp32 hidden states, a vocabulary that divides nothing
        dict(HEAD, op="loss", name="loss-prompts-1021x1024", T=1021, vocab=32003, d=1024, x_bf16=False, scale=0.5),
        # a training step at the head: loss, hidden states' gradient, the weight's in 32 bits
        dict(HEAD, op="step", name="step-8192x50000", T=8192, none=0.02),
        # the same of a smaller model with the weight's gradient in 16 bits, a third of the tokens masked
        dict(HEAD, op="step", name="step-2000x32003", T=2000, vocab=32003, d=1024, g_bf16=True, none=0.33),
        # the update of one small weight: only latency
        dict(ORTH, name="orth-64x448", rows=64, cols=448),
        # the four key matrices of a memory layer as one batch, from 16-bit gradients, tall
        dict(ORTH, name="orth-keys-4x1792x448", n=4, rows=1792, cols=448, g_bf16=True, o_bf16=True),
        # the query linear, its 32-bit weight updated in place
        dict(ORTH, name="orth-query-896x2048", rows=896, cols=2048, decay=0.999, scale=-0.02),
        # the projection of the expanded values: long rows
        dict(ORTH, name="orth-proj-1024x16384", rows=1024, cols=16384, o_bf16=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; none costs more than the largest of them."""
    op = rng.choice(["embed", "embed_back", "embed_rows", "loss", "step", "step", "orth", "orth"])
    if op.startswith("embed"):
        return dict(EMBED, op=op, T=_log(rng, 1, 20000), vocab=_log(rng, 500, 60000), d=_log(rng, 64, 2048),
                    w_bf16=rng.random() < 0.5, o_bf16=rng.random() < 0.5, scale=rng.choice([1.0, 0.5, 32.0]),
                    none=rng.choice([0.0, 0.0, 0.1, 0.3]))
    if op in ("loss", "step"):
        c = dict(HEAD, op=op, T=_log(rng, 1, 8192), vocab=_log(rng, 500, 60000), d=8 * _log(rng, 8, 256),
                 x_bf16=rng.random() < 0.7, g_bf16=rng.random() < 0.4, scale=rng.choice([1.0, 1.0, 0.25]),
                 none=rng.choice([0.0, 0.0, 0.1, 0.5]))
        while c["T"] * c["vocab"] * c["d"] > (1 << 39 if c["x_bf16"] else 1 << 37):
            c["T"] = c["T"] // 2 + 1
        return c
    c = dict(ORTH, n=rng.choice([1, 1, 2, 6]), rows=_log(rng, 8, 4096), cols=_log(rng, 8, 8192),
             g_bf16=rng.random() < 0.4, o_bf16=rng.random() < 0.4, steps=rng.choice([5, 5, 5, 3, 6]),
             decay=rng.choice([0.0, 0.0, 0.99]), scale=rng.choice([1.0, 0.2]))
    if rng.random() < 0.5:
        c["rows"], c["cols"] = 8 * (c["rows"] // 8 + 1), 8 * (c["cols"] // 8 + 1)
    while c["n"] * c["steps"] * _small(c) ** 2 * (2 * _long(c) + _small(c)) > 1 << 38:
        c["rows"], c["cols"] = c["rows"] // 2 + 1, c["cols"] // 2 + 1
    return c


def _small(c):
    return min(c["rows"], c["cols"])


def _long(c):
    return max(c["rows"], c["cols"])


# ---------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, shape, std, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _uniform(g, shape, lo, hi):
    return torch.empty(shape, dtype=torch.float32, device=DEV).uniform_(lo, hi, generator=g)


def _type(bf16):
    return torch.bfloat16 if bf16 else torch.float32


def _tokens(g, c):
    """Token ids as a text has them: the r-th most frequent with a share near 1 / r; -1 where padded."""
    rank = torch.exp(_uniform(g, (c["T"],), 0.0, math.log(c["vocab"]))).long().clamp(1, c["vocab"]) - 1
    names = torch.randperm(c["vocab"], generator=g, device=DEV)
    ids = torch.where(_uniform(g, (c["T"],), 0.0, 1.0) < c["none"], -1, names[rank])
    return ids.to(torch.int32)


def _embed_inputs(c, seed):
    g = _gen(seed)
    s = {"ids": _tokens(g, c)}
    if c["op"] == "embed":
        s["table"] = _randn(g, (c["vocab"], c["d"]), 0.5, _type(c["w_bf16"]))
    else:
        s["dout"] = _randn(g, (c["T"], c["d"]), 1e-2, _type(c["o_bf16"]))
    if c["op"] == "embed_back":
        s["dtable"] = _randn(g, (c["vocab"], c["d"]), 1e-3)
    return s


def _head_inputs(c, seed):
    """Hidden states that know some of their targets, so that a target's probability goes from one in
    the vocabulary to about one half; the loss's gradient is that of a mean over the counted tokens."""
    g, T, d = _gen(seed), c["T"], c["d"]
    s = {"w": _randn(g, (c["vocab"], d), 2.0 / math.sqrt(d) / c["scale"], torch.bfloat16), "targets": _tokens(g, c)}
    known = s["w"][s["targets"].clamp(min=0).long()].float()
    much = c["scale"] * (math.log(c["vocab"]) - 1.0) / 4.0      # a known target's score: up to log vocab - 1
    x = _randn(g, (T, d), 1.0) + known * _uniform(g, (T, 1), 0.0, much)
    s["x"] = x.to(_type(c["x_bf16"]))
    if c["op"] == "step":
        n = (s["targets"] >= 0).sum().clamp(min=1)
        s["dloss"] = torch.ones((T,), device=DEV) / n
    return s


def _orth_inputs(c, seed):
    """A momentum as training leaves it: a few strong directions over a broad floor."""
    g, n, m, k = _gen(seed), c["n"], c["rows"], c["cols"]
    r = min(8, m, k)
    strong = torch.bmm(_randn(g, (n, m, r), 1.0), _randn(g, (n, r, k), 0.3 / math.sqrt(r)))
    s = {"g": ((strong + _randn(g, (n, m, k), 1.0)) * 1e-3).to(_type(c["g_bf16"]))}
    s["out"] = _randn(g, (n, m, k), 0.02, _type(c["o_bf16"]))
    return s


def prepare(case, seed):
    c, op = case, case["op"]
    T = c.get("T")
    if op == "orth":
        s = _orth_inputs(c, seed)
    elif op in ("loss", "step"):
        s = _head_inputs(c, seed)
        s["loss"], s["lse"] = torch.empty((T,), device=DEV), torch.empty((T,), device=DEV)
        if op == "step":
            s["dx"] = torch.empty_like(s["x"])
            s["dw"] = torch.empty((c["vocab"], c["d"]), dtype=_type(c["g_bf16"]), device=DEV)
    else:
        s = _embed_inputs(c, seed)
        if op == "embed":
            s["out"] = torch.empty((T, c["d"]), dtype=_type(c["o_bf16"]), device=DEV)
        elif op == "embed_rows":
            s["rows"] = torch.zeros((T,), dtype=torch.int32, device=DEV)
            s["d_rows"] = torch.zeros((T, c["d"]), device=DEV)
            s["n_rows"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
    s["case"] = c
    if own:     # the descriptor and the scratch memory that a program keeps for its calls
        import paper_2411_12364_amd as U
        need = 0
        if op == "orth":
            s["desc"] = U.umem_orth_desc(c["n"], c["rows"], c["cols"], int(c["g_bf16"]), int(c["o_bf16"]),
                                         c["steps"], *COEF, EPS, c["decay"], c["scale"])
            st, need = U.umem_orthogonalize_workspace_size(s["desc"])
            U.check(st)
        elif op in ("loss", "step"):
            s["desc"] = U.umem_head_desc(c["vocab"], c["d"], int(c["x_bf16"]), int(c["g_bf16"]), c["scale"])
            st, need = U.umem_head_loss_workspace_size(s["desc"], T)
            U.check(st)
            if op == "step":
                st, more = U.umem_head_backward_workspace_size(s["desc"], T)
                U.check(st)
                need = max(need, more)
        else:
            s["desc"] = U.umem_embed_desc(c["vocab"], c["d"], int(c["w_bf16"]), int(c["o_bf16"]), c["scale"])
            if op != "embed":
                st, need = U.umem_embed_backward_workspace_size(s["desc"], T)
                U.check(st)
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------- the library's calls

def _own(s):
    import paper_2411_12364_amd as U
    c, op, d, ws = s["case"], s["case"]["op"], s["desc"], s["ws"]
    if op == "orth":
        U.check(U.umem_orthogonalize(d, s["g"], s["out"], ws, ws.numel()), "umem_orthogonalize")
        return s["out"]
    T = c["T"]
    if op == "embed":
        U.check(U.umem_embed(d, T, s["table"], s["ids"], s["out"]), "umem_embed")
        return s["out"]
    if op == "embed_back":
        U.check(U.umem_embed_backward(d, T, s["ids"], s["dout"], s["dtable"], ws, ws.numel()),
                "umem_embed_backward")
        return s["dtable"]
    if op == "embed_rows":
        U.check(U.umem_embed_backward_rows(d, T, s["ids"], s["dout"], s["rows"], s["d_rows"], s["n_rows"], ws,
                                           ws.numel()), "umem_embed_backward_rows")
        return {k: s[k] for k in ("rows", "d_rows", "n_rows")}
    U.check(U.umem_head_loss(d, T, s["x"], s["w"], s["targets"], s["loss"], s["lse"], ws, ws.numel()),
            "umem_head_loss")
    if op == "loss":
        return {"loss": s["loss"], "lse": s["lse"]}
    U.check(U.umem_head_backward(d, T, s["x"], s["w"], s["targets"], s["lse"], s["dloss"], s["dx"], s["dw"], 0, ws,
                                 ws.numel()), "umem_head_backward")
    return {k: s[k] for k in ("loss", "lse", "dx", "dw")}


# ---------------------------------------------------------------------------- the plain form

def _plain_embed(s):
    c, op, ids = s["case"], s["case"]["op"], s["ids"]
    on = ids >= 0
    if op == "embed":
        rows = s["table"][ids.clamp(min=0)].float() * c["scale"]
        return torch.where(on[:, None], rows, 0.0).to(_type(c["o_bf16"]))
    part = torch.where(on[:, None], s["dout"].float() * c["scale"], 0.0)
    if op == "embed_back":
        return s["dtable"].index_add_(0, ids.clamp(min=0), part)
    key, at = torch.sort(torch.where(on, ids, c["vocab"]), stable=True)
    first = torch.ones_like(key, dtype=torch.bool)
    first[1:] = key[1:] != key[:-1]
    place = torch.cumsum(first, 0) - 1
    first = first & (key < c["vocab"])
    rows = torch.zeros_like(ids).index_add_(0, place, torch.where(first, key, 0).to(torch.int32))
    d_rows = torch.zeros((c["T"], c["d"]), device=DEV).index_add_(0, place, part[at])
    return {"rows": rows, "d_rows": d_rows, "n_rows": first.sum().to(torch.int32).reshape(1)}


def _plain_head(s):
    c = s["case"]
    on = s["targets"] >= 0
    y = s["targets"].clamp(min=0).long()[:, None]
    x, w = s["x"].float(), s["w"].float()
    z = (x @ w.t()).mul_(c["scale"])
    top = z.max(dim=1, keepdim=True).values
    goal = z.gather(1, y)
    p = z.sub_(top).exp_()
    total = p.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    out = {"loss": torch.where(on, (lse - goal)[:, 0], 0.0), "lse": lse[:, 0]}
    if c["op"] == "loss":
        return out
    p = p.div_(total).scatter_add_(1, y, torch.full_like(goal, -1.0))
    p = p.mul_((torch.where(on, s["dloss"], 0.0) * c["scale"])[:, None])
    out["dx"] = (p @ w).to(_type(c["x_bf16"]))
    out["dw"] = (p.t() @ x).to(_type(c["g_bf16"]))
    return out


def _plain_step(x, a, b, c):
    gram = torch.bmm(x, x.transpose(1, 2).contiguous())
    return a * x + torch.bmm(b * gram + c * torch.bmm(gram, gram), x)


def _plain_orth(s):
    c = s["case"]
    x = s["g"].float()
    norm = x.double().square().sum(dim=(1, 2), keepdim=True).sqrt().float()
    x = x / (norm + EPS)
    tall = c["rows"] > c["cols"]
    x = x.transpose(1, 2).contiguous() if tall else x
    for _ in range(c["steps"]):
        x = _plain_step(x, *COEF)
    x = (x.transpose(1, 2) if tall else x) * c["scale"]
    x = x + c["decay"] * s["out"].float() if c["decay"] else x
    return s["out"].copy_(x)


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_orth(state) if op == "orth" else _plain_head(state) if op in ("loss", "step") else _plain_embed(state)


# ---------------------------------------------------------------------------- what it takes

def work(case):
    c, op = case, case["op"]
    if op == "orth":
        m, k, n = _small(c), _long(c), c["n"]
        e = m * k
        size = (2 if c["g_bf16"] else 4) + (2 if c["o_bf16"] else 4) * (2 if c["decay"] else 1)
        # two symmetric products of which one half is enough, and one full one
        return {"bytes": n * e * size, "flops": n * c["steps"] * m * m * (k + m + 2 * k)}
    T, d = c["T"], c["d"]
    if op in ("loss", "step"):
        x, flops = (2 if c["x_bf16"] else 4), 2 * T * c["vocab"] * d
        bytes_ = T * (d * x + 12) + 2 * c["vocab"] * d
        if op == "loss":
            return {"bytes": bytes_, "flops": flops}
        return {"bytes": bytes_ + T * (d * x + 4) + c["vocab"] * d * (2 if c["g_bf16"] else 4), "flops": 3 * flops}
    on = T * (1.0 - c["none"])
    # distinct tokens of T draws with a share of 1 / (r ln vocab) for the r-th
    seen = sum(1.0 - math.exp(on * math.log(1.0 - min(0.99, 1.0 / (r * math.log(c["vocab"])))))
               for r in range(1, c["vocab"] + 1))
    o = 2 if c["o_bf16"] else 4
    if op == "embed":
        return {"bytes": T * 4 + seen * d * (2 if c["w_bf16"] else 4) + T * d * o, "flops": T * d}
    per_row = 8 * d if op == "embed_back" else 4 * d + 4
    return {"bytes": T * 4 + on * d * o + seen * per_row, "flops": 2 * on * d}


# ---------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    c, op = case, case["op"]
    if op == "orth":
        s = _orth_inputs(c, seed)
        got = []
        for j in range(c["n"]):
            x = s["g"][j].double()
            x = x / (torch.linalg.vector_norm(x) + EPS)
            a, b, q = COEF
            for _ in range(c["steps"]):     # on the smaller side: (a + b S + c S^2) X of either shape
                if c["rows"] <= c["cols"]:
                    gram = x @ x.t().contiguous()
                    x = a * x + b * (gram @ x) + q * (gram @ (gram @ x))
                else:
                    gram = x.t().contiguous() @ x
                    x = a * x + b * (x @ gram) + q * ((x @ gram) @ gram)
            got.append(c["decay"] * s["out"][j].double() + c["scale"] * x)
        return torch.stack(got)
    if op in ("loss", "step"):
        s = _head_inputs(c, seed)
        x, w, keep = s["x"].double(), s["w"].double(), (s["targets"] >= 0).nonzero()[:, 0]
        goal = s["targets"].long()[keep]
        z = c["scale"] * (x @ w.t().contiguous())
        lse = torch.logsumexp(z, dim=1)
        loss = torch.zeros_like(lse)
        loss[keep] = lse[keep] - z[keep, goal]
        if op == "loss":
            return {"loss": loss, "lse": lse}
        r = torch.exp(z[keep] - lse[keep, None])
        del z
        r[torch.arange(len(keep), device=DEV), goal] -= 1.0
        r *= c["scale"] * s["dloss"].double()[keep, None]
        dx = torch.zeros_like(x)
        dx[keep] = r @ w
        return {"loss": loss, "lse": lse, "dx": dx, "dw": r.t().contiguous() @ x[keep]}
    s = _embed_inputs(c, seed)
    ids = s["ids"].long()
    keep = (ids >= 0).nonzero()[:, 0]
    if op == "embed":
        out = torch.zeros((c["T"], c["d"]), dtype=torch.float64, device=DEV)
        out[keep] = c["scale"] * s["table"].double()[ids[keep]]
        return out
    total = torch.zeros((c["vocab"], c["d"]), dtype=torch.float64, device=DEV)
    total.index_put_((ids[keep],), s["dout"].double()[keep], accumulate=True)
    if op == "embed_back":
        return s["dtable"].double() + c["scale"] * total
    used = torch.unique(ids[keep])
    d_rows = torch.zeros((c["T"], c["d"]), dtype=torch.float64, device=DEV)
    d_rows[:len(used)] = c["scale"] * total[used]
    return {"rows": None, "d_rows": d_rows, "n_rows": None}
