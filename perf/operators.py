"""The operators around the memory layer, as cases to be timed and compared: the norms before and
after a block with its gate and residual scale (and their backward), the global gradient norm and
clipping over the tensors of a training step, and the low-rank adapters of many requests beside a
shared projection.

``own`` chooses between two forms of the same pass: False computes it with elementary torch
operations in 32 bits (sums of squares over many tensors in 64), rounded once at the end; True makes
the calls of this library.  ``exact`` is the same arithmetic from the definitions, in 64 bits.

Inputs are made on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5

BLOCK = dict(T=1, d=2048, norm="layer", norm_out="none", gate="none", sigmoid=False, next=False,
             beta=True, h_bf16=False, y_bf16=False, res_scale=1.0, out_scale=1.0)
ADAPT = dict(op="adapt", T=64, requests=64, n=64, rank=16, d_in=1024, d_out=2048, x_bf16=False,
             o_bf16=False, none=0.0)


def _block(op, **kw):
    return {"op": op, **BLOCK, **kw}


def listed():
    return [
        # one new token of one sequence leaves the memory block and enters the next: only latency
        _block("exit", name="exit-decode-1", T=1, norm_out="rms", gate="channel", next=True),
        # prompts of many requests, a bf16 residual stream, every element with a gate of its own
        _block("exit", name="exit-prompts-4096", T=4096, norm="rms", norm_out="layer", gate="full",
               sigmoid=True, next=True, h_bf16=True, y_bf16=True, res_scale=0.7),
        # the decode batch that the UltraMem layer is timed with enters the block
        _block("enter", name="enter-decode-512", T=512),
        # four prompts of a ragged length, a width that divides nothing
        _block("enter", name="enter-odd-2036x1023", T=2036, d=1023, norm="rms", beta=False,
               h_bf16=True),
        # a training step's tokens on the way back through the entry, at two widths and types
        _block("enter_back", name="enter-back-1001x1024", T=1001, d=1024),
        _block("enter_back", name="enter-back-8192x2048", T=8192, norm="rms", h_bf16=True, y_bf16=True),
        # and through the exit: a gate for each channel; a gate for each token, ragged sizes
        _block("exit_back", name="exit-back-4096x2048", T=4096, norm_out="layer", gate="channel",
               out_scale=0.5),
        _block("exit_back", name="exit-back-333x1500", T=333, d=1500, norm_out="rms", beta=False,
               gate="token", sigmoid=True, h_bf16=True, y_bf16=True, res_scale=0.9),
        # the small parameters of a model: norms, gates and biases, hundreds of bytes to kilobytes each
        dict(op="clip", name="clip-small-96", big=0, width=1, mid=0, small=96, bf16=False, factor=0.3),
        # all gradients of the UltraMem layer at its batch: the touched value rows (their number known
        # on the GPU only), keys, cores, projections, norms
        dict(op="clip", name="clip-ultramem-512", big=43008, width=4096, mid=6, small=24, bf16=False,
             factor=0.5),
        # a decode batch, an adapter of its own for each request
        dict(ADAPT, name="adapt-decode-64"),
        # prompts of sixteen requests in one batch beside the query linear, a few without an adapter
        dict(ADAPT, name="adapt-prompts-4096", T=4096, requests=16, n=12, rank=32, d_in=2048, d_out=896,
             x_bf16=True, none=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; none costs more than the largest of them."""
    op = rng.choice(["enter", "enter_back", "exit", "exit_back", "clip", "adapt", "adapt"])
    if op == "clip":
        big = rng.choice([0, _log(rng, 100, 40000)])
        return dict(op="clip", big=big, width=rng.choice([512, 1000, 1024, 2048]), mid=rng.randint(0, 6),
                    small=rng.randint(1, 150), bf16=rng.random() < 0.3, factor=rng.choice([0.1, 0.5, 2.0]))
    if op == "adapt":
        T = _log(rng, 1, 4096)
        c = dict(ADAPT, T=T, requests=rng.randint(1, min(T, 64)), n=rng.randint(1, 64),
                 rank=rng.choice([8, 16, 16, 32, 64]), d_in=8 * _log(rng, 32, 512),
                 d_out=8 * _log(rng, 32, 512), x_bf16=rng.random() < 0.5, o_bf16=rng.random() < 0.4,
                 none=rng.choice([0.0, 0.0, 0.2, 1.0]))
        while c["T"] * c["rank"] * (c["d_in"] + c["d_out"]) > 1 << 29:
            c["T"] //= 2
            c["requests"] = min(c["requests"], c["T"])
        return c
    c = _block(op, T=_log(rng, 1, 8192), d=_log(rng, 64, 4096), norm=rng.choice(["layer", "rms"]),
               beta=rng.random() < 0.6, h_bf16=rng.random() < 0.4)
    if rng.random() < 0.6:
        c["d"] = max(8, c["d"] // 8 * 8)
    c["y_bf16"] = c["h_bf16"] or rng.random() < 0.2
    c["res_scale"], c["out_scale"] = rng.choice([1.0, 0.7]), rng.choice([1.0, 0.25])
    if op in ("exit", "exit_back"):
        c["norm_out"] = rng.choice(["none", "layer", "rms"])
        c["gate"] = rng.choice(["none", "channel", "token", "full"])
        c["sigmoid"] = rng.random() < 0.5
        c["next"] = op == "exit" and rng.random() < 0.7
    return c


# ---------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, shape, std, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _uniform(g, shape, lo, hi):
    return torch.empty(shape, dtype=torch.float32, device=DEV).uniform_(lo, hi, generator=g)


def _type(bf16):
    return torch.bfloat16 if bf16 else torch.float32


def _rows(g, T, d, bf16):
    """Hidden states: rows of different scales around a mean of their own, a few channels far larger."""
    x = _randn(g, (T, d), 1.0) * _uniform(g, (T, 1), 0.3, 3.0) + _randn(g, (T, 1), 0.2)
    big = torch.randint(0, d, (max(1, d // 256),), generator=g, device=DEV)
    x[:, big] *= 8.0
    return x.to(_type(bf16))


def _block_inputs(c, seed):
    g, T, d, op = _gen(seed), c["T"], c["d"], c["op"]
    s = {"gate": None, "gamma": None, "beta": None}
    hb, yb = c["h_bf16"], c["y_bf16"]

    def params():
        return 1.0 + _randn(g, (d,), 0.2), _randn(g, (d,), 0.1) if c["beta"] else None

    if op in ("enter", "enter_back"):
        s["h"] = _rows(g, T, d, hb)
        s["gamma"], s["beta"] = params()
        if op == "enter_back":
            s["dn"] = _randn(g, (T, d), 1e-2, _type(yb))
            s["dres"] = _randn(g, (T, d), 1e-2, _type(hb))
        return s
    s["y"] = _rows(g, T, d, yb)
    if c["norm_out"] != "none":
        s["gamma"], s["beta"] = params()
    if c["gate"] != "none":
        shape = {"channel": (d,), "token": (T,), "full": (T, d)}[c["gate"]]
        s["gate"] = _randn(g, shape, 1.0, _type(yb and c["gate"] == "full"))
    if op == "exit":
        s["h"] = _rows(g, T, d, hb)
        s["gamma_next"], s["beta_next"] = params() if c["next"] else (None, None)
    else:
        s["dh_out"] = _randn(g, (T, d), 1e-2, _type(hb))
    return s


# Widths of a layer's dense gradients (keys, projections, query linear) and of its small ones.
_MID = [(2, 1792, 448), (2, 1792, 448), (896, 2048), (2048, 1024), (1024, 16384), (4, 2048)]
_SMALL = [2048, 896, 1024, 448, 8, 1, 4096, 2047, 16, 333]


def _clip_inputs(c, seed):
    """Gradients in the sizes of a layer: rows of the value table with their number on the GPU, dense
    ones, small ones; values over several orders of magnitude, as between the tensors of a model."""
    g = _gen(seed)
    grads, n_rows = [], None
    if c["big"]:
        grads.append(_randn(g, (c["big"], c["width"]), 1e-3))
        used = torch.randint(c["big"] - c["big"] // 16, c["big"] + 1, (1,), generator=g, device=DEV)
        n_rows = used.to(torch.int32)
    dt = _type(c["bf16"])
    for i in range(c["mid"]):
        grads.append(_randn(g, _MID[i % len(_MID)], 10.0 ** -(2 + i % 3), dt))
    for i in range(c["small"]):
        grads.append(_randn(g, (_SMALL[i % len(_SMALL)],), 10.0 ** -(i % 4), dt))
    return grads, n_rows


def _adapt_inputs(c, seed):
    """Requests of ragged lengths, their tokens in a run each; each request takes one of n adapters."""
    g, T, R, n = _gen(seed), c["T"], c["requests"], c["n"]
    cuts = torch.sort(torch.randperm(T - 1, generator=g, device=DEV)[:R - 1] + 1).values
    req = torch.bucketize(torch.arange(T, device=DEV), cuts, right=True)
    ids = torch.randint(0, n, (R,), generator=g, device=DEV)
    ids = torch.where(_uniform(g, (R,), 0.0, 1.0) < c["none"], -1, ids)
    return {
        "x": _randn(g, (T, c["d_in"]), 1.0, _type(c["x_bf16"])),
        "ids": ids[req].to(torch.int32),
        "a": _randn(g, (n, c["rank"], c["d_in"]), 1.0 / math.sqrt(c["d_in"]), torch.bfloat16),
        "b": _randn(g, (n, c["d_out"], c["rank"]), 0.3, torch.bfloat16),
        "scale": _uniform(g, (n,), 0.25, 2.0),
        "base": _randn(g, (T, c["d_out"]), 1.0, _type(c["o_bf16"])),
    }


def prepare(case, seed):
    c, op = case, case["op"]
    if op == "clip":
        grads, n_rows = _clip_inputs(c, seed)
        # the clipped value rows, and all other clipped gradients one after another
        s = {"grads": grads, "n_rows": n_rows, "rows_out": torch.zeros_like(grads[0]) if c["big"] else None}
        rest = grads[1:] if c["big"] else grads
        s["flat"] = torch.zeros((sum(x.numel() for x in rest),), dtype=_type(c["bf16"]), device=DEV)
        s["out"] = ([s["rows_out"]] if c["big"] else []) + \
            [v.view(x.shape) for v, x in zip(s["flat"].split([x.numel() for x in rest]), rest)]
        # what the call is given for each tensor: address, where to write, the rows' number on the GPU,
        # rows, elements in a row, type (0 fp32, 1 bf16)
        s["table"] = np.array([[x.data_ptr(), y.data_ptr(),
                                n_rows.data_ptr() if i == 0 and c["big"] else 0,
                                x.shape[0] if x.dim() > 1 else 1,
                                x.numel() // (x.shape[0] if x.dim() > 1 else 1),
                                int(x.dtype == torch.bfloat16)]
                               for i, (x, y) in enumerate(zip(grads, s["out"]))], dtype=np.int64)
        s["max_norm"] = _limit(c, grads)
        s["norm"] = torch.zeros((1,), dtype=torch.float32, device=DEV)
    elif op == "adapt":
        s = _adapt_inputs(c, seed)
        s["out"] = torch.empty_like(s["base"])
    else:
        s = _block_inputs(c, seed)
        like = {"enter": ["n"], "exit": ["h_out"] + ["n_next"] * c["next"], "enter_back": ["dh"],
                "exit_back": ["dh", "dy"]}[op]
        for k in like:
            bf16 = c["y_bf16"] if k in ("n", "n_next", "dy") else c["h_bf16"]
            s[k] = torch.empty((c["T"], c["d"]), dtype=_type(bf16), device=DEV)
        for k in ("gate", "gamma", "beta"):
            if op in ("enter_back", "exit_back"):
                s["d" + k] = torch.empty_like(s[k]) if s[k] is not None else None
    s["case"] = c
    if own:     # the descriptor and the scratch memory that a program keeps for its calls
        import paper_2411_12364_amd as U
        need = 0
        if op == "clip":
            st, need = U.umem_grad_workspace_size(len(s["table"]), s["table"])
            U.check(st)
        elif op == "adapt":
            s["desc"] = U.umem_adapter_desc(c["n"], c["rank"], c["d_in"], c["d_out"],
                                            int(c["x_bf16"]), int(c["o_bf16"]))
            st, need = U.umem_adapter_workspace_size(s["desc"], c["T"])
            U.check(st)
        else:
            norm = {"layer": U.UMEM_NORM_LAYER, "rms": U.UMEM_NORM_RMS, "none": U.UMEM_NORM_NONE}
            gate = {"none": U.UMEM_GATE_NONE, "channel": U.UMEM_GATE_CHANNEL,
                    "token": U.UMEM_GATE_TOKEN, "full": U.UMEM_GATE_FULL}
            s["desc"] = U.umem_block_desc(c["d"], norm[c["norm"]], norm[c["norm_out"]], gate[c["gate"]],
                                          int(c["sigmoid"]), int(c["h_bf16"]), int(c["y_bf16"]), EPS,
                                          c["res_scale"], c["out_scale"])
            if op in ("enter_back", "exit_back"):
                st, need = U.umem_block_backward_workspace_size(s["desc"], c["T"])
                U.check(st)
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    return s


def _limit(c, grads):
    """The clipping threshold of a case: its factor times the norm that its draws have on average."""
    total = grads[0].numel() * 1e-6 if c["big"] else 0.0
    for i, x in enumerate(grads[1:] if c["big"] else grads):
        std = 10.0 ** -(2 + i % 3) if i < c["mid"] else 10.0 ** -((i - c["mid"]) % 4)
        total += x.numel() * std * std
    return c["factor"] * math.sqrt(total)


# ---------------------------------------------------------------------------- the library's calls

def _own(s):
    import paper_2411_12364_amd as U
    c, op, ws = s["case"], s["case"]["op"], s["ws"]
    if op == "clip":
        n, table = len(s["table"]), s["table"]
        U.check(U.umem_grad_norm(n, table, s["norm"], None, ws, ws.numel()), "umem_grad_norm")
        U.check(U.umem_grad_clip(n, table, s["max_norm"], s["norm"]), "umem_grad_clip")
        return {"norm": s["norm"], "rows": s["rows_out"], "rest": s["flat"]}
    d, T = s["desc"], c["T"]
    if op == "adapt":
        U.check(U.umem_adapter_add(d, T, s["x"], s["ids"], s["a"], s["b"], s["scale"], s["base"],
                                   s["out"], ws, ws.numel()), "umem_adapter_add")
        return s["out"]
    if op == "enter":
        U.check(U.umem_block_in(d, T, s["h"], s["gamma"], s["beta"], s["n"]), "umem_block_in")
        return s["n"]
    if op == "exit":
        U.check(U.umem_block_out(d, T, s["h"], s["y"], s["gate"], s["gamma"], s["beta"], s["h_out"],
                                 s["gamma_next"], s["beta_next"], s.get("n_next")), "umem_block_out")
        return {"h_out": s["h_out"], "n_next": s.get("n_next")}
    if op == "enter_back":
        U.check(U.umem_block_in_backward(d, T, s["h"], s["gamma"], s["dn"], s["dres"], s["dh"],
                                         s["dgamma"], s["dbeta"], 0, ws, ws.numel()),
                "umem_block_in_backward")
        return {k: s[k] for k in ("dh", "dgamma", "dbeta")}
    U.check(U.umem_block_out_backward(d, T, s["y"], s["gate"], s["gamma"], s["beta"], s["dh_out"],
                                      s["dh"], s["dy"], s["dgate"], s["dgamma"], s["dbeta"], 0, ws,
                                      ws.numel()), "umem_block_out_backward")
    return {k: s[k] for k in ("dh", "dy", "dgate", "dgamma", "dbeta")}


# ---------------------------------------------------------------------------- the plain form

def _norm(x, kind, gamma, beta):
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    x = x * gamma
    return x if beta is None else x + beta


def _norm_back(x, kind, gamma, dn):
    """(dx, x^) of the norm's input, dn the gradient of its output."""
    if kind == "layer":
        x = x - x.mean(dim=1, keepdim=True)
    r = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
    xh, g = x * r, dn * gamma
    dx = g - xh * (g * xh).mean(dim=1, keepdim=True)
    if kind == "layer":
        dx = dx - g.mean(dim=1, keepdim=True)
    return dx * r, xh


def _gate(c, s):
    """The gate's values in 32 bits, in a shape that spreads over [T, d]."""
    if c["gate"] == "none":
        return None
    g = s["gate"].float()
    g = g[:, None] if c["gate"] == "token" else g
    return 1.0 / (1.0 + torch.exp(-g)) if c["sigmoid"] else g


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "clip":
        n_rows = s["n_rows"]
        grads = [x.float() for x in s["grads"]]
        if c["big"]:
            keep = torch.arange(c["big"], device=DEV)[:, None] < n_rows
            grads[0] = torch.where(keep, grads[0], 0.0)
        norm = torch.stack([x.double().square().sum() for x in grads]).sum().sqrt().float()
        factor = torch.where(norm <= s["max_norm"], 1.0, s["max_norm"] / norm)
        _ = [torch.mul(x, factor, out=y) if y.dtype == x.dtype else y.copy_(x * factor)
             for x, y in zip(grads, s["out"])]
        return {"norm": norm.reshape(1), "rows": s["rows_out"], "rest": s["flat"]}
    if op == "adapt":
        on = s["ids"] >= 0
        i = torch.where(on, s["ids"], 0).long()
        v = torch.bmm(s["a"][i].float(), s["x"].float()[:, :, None])
        v = v * torch.where(on, s["scale"][i], 0.0)[:, None, None]
        delta = torch.bmm(s["b"][i].float(), v)[:, :, 0]
        return (s["base"].float() + delta).to(s["base"].dtype)
    ht, yt = _type(c["h_bf16"]), _type(c["y_bf16"])
    if op == "enter":
        return _norm(s["h"].float(), c["norm"], s["gamma"], s["beta"]).to(yt)
    if op == "exit":
        y = s["y"].float()
        m = y if c["norm_out"] == "none" else _norm(y, c["norm_out"], s["gamma"], s["beta"])
        g = _gate(c, s)
        m = m if g is None else m * g
        h = (c["res_scale"] * s["h"].float() + c["out_scale"] * m).to(ht)
        n = _norm(h.float(), c["norm"], s["gamma_next"], s["beta_next"]).to(yt) if c["next"] else None
        return {"h_out": h, "n_next": n}
    if op == "enter_back":
        dn = s["dn"].float()
        dx, xh = _norm_back(s["h"].float(), c["norm"], s["gamma"], dn)
        return {"dh": (s["dres"].float() + dx).to(ht), "dgamma": (dn * xh).sum(dim=0),
                "dbeta": dn.sum(dim=0) if c["beta"] else None}
    y, dh_out = s["y"].float(), s["dh_out"].float()
    g, dm = _gate(c, s), c["out_scale"] * dh_out
    m = y if c["norm_out"] == "none" else _norm(y, c["norm_out"], s["gamma"], s["beta"])
    out = {"dh": (c["res_scale"] * dh_out).to(ht), "dgate": None, "dgamma": None, "dbeta": None}
    if g is not None:
        dg = dm * m * (g * (1.0 - g)) if c["sigmoid"] else dm * m
        dg = dg.sum(dim=0) if c["gate"] == "channel" else dg.sum(dim=1) if c["gate"] == "token" else dg
        out["dgate"] = dg.to(s["gate"].dtype)
        dm = dm * g
    if c["norm_out"] == "none":
        out["dy"] = dm.expand(c["T"], c["d"]).to(yt)
        return out
    dy, xh = _norm_back(y, c["norm_out"], s["gamma"], dm)
    out.update(dy=dy.to(yt), dgamma=(dm * xh).sum(dim=0), dbeta=dm.sum(dim=0) if c["beta"] else None)
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------- what it takes

def work(case):
    c, op = case, case["op"]
    if op == "clip":
        used = (c["big"] - c["big"] // 32) * c["width"]
        rest = sum(math.prod(_MID[i % len(_MID)]) for i in range(c["mid"]))
        rest += sum(_SMALL[i % len(_SMALL)] for i in range(c["small"]))
        return {"bytes": 8 * used + (4 if c["bf16"] else 8) * rest, "flops": 3 * (used + rest)}
    T = c["T"]
    if op == "adapt":
        r, di, do = c["rank"], c["d_in"], c["d_out"]
        on = 1.0 - c["none"]
        used = c["n"] * (1.0 - (1.0 - 1.0 / c["n"]) ** (c["requests"] * on))
        x, o = (2 if c["x_bf16"] else 4), (2 if c["o_bf16"] else 4)
        return {"bytes": T * (x * di * on + 2 * o * do + 4) + 2 * used * r * (di + do),
                "flops": 2 * T * on * r * (di + do)}
    e, hb, yb, d = T * c["d"], (2 if c["h_bf16"] else 4), (2 if c["y_bf16"] else 4), c["d"]
    gate = {"none": 0, "channel": 4 * d, "token": 4 * T, "full": yb * e}[c["gate"]]
    if op == "enter":
        return {"bytes": e * (hb + yb) + 8 * d, "flops": 8 * e}
    if op == "exit":
        return {"bytes": e * (2 * hb + yb + (yb if c["next"] else 0)) + gate + 16 * d, "flops": 20 * e}
    if op == "enter_back":
        return {"bytes": e * (3 * hb + yb) + 12 * d, "flops": 16 * e}
    return {"bytes": e * (2 * hb + 2 * yb) + 2 * gate + 16 * d, "flops": 20 * e}


# ---------------------------------------------------------------------------- 64 bits

def _norm64(x, kind):
    """(x^, 1 / spread) of each row."""
    mu = x.sum(dim=1, keepdim=True) / x.shape[1] if kind == "layer" else 0.0
    var = ((x - mu) ** 2).sum(dim=1, keepdim=True) / x.shape[1]
    r = 1.0 / torch.sqrt(var + EPS)
    return (x - mu) * r, r


def _affine64(xh, gamma, beta):
    out = xh * gamma.double()
    return out if beta is None else out + beta.double()


def _pull64(xh, r, kind, v):
    """The transposed Jacobian of x -> x^, applied to the rows of v."""
    d = xh.shape[1]
    back = v - xh * ((v * xh).sum(dim=1, keepdim=True) / d)
    if kind == "layer":
        back = back - v.sum(dim=1, keepdim=True) / d
    return r * back


def exact(case, seed):
    c, op = case, case["op"]
    if op == "clip":
        grads, n_rows = _clip_inputs(c, seed)
        g64 = [x.double() for x in grads]
        if c["big"]:
            g64[0][int(n_rows):] = 0.0
        total = sum(float((x * x).sum()) for x in g64)
        limit = _limit(c, grads)
        norm = math.sqrt(total)
        factor = 1.0 if norm <= limit else limit / norm
        return {"norm": torch.tensor([norm], dtype=torch.float64, device=DEV),
                "rows": g64[0] * factor if c["big"] else None,
                "rest": torch.cat([x.reshape(-1) for x in (g64[1:] if c["big"] else g64)]) * factor}
    if op == "adapt":
        s = _adapt_inputs(c, seed)
        out = s["base"].double()
        for j in range(c["n"]):
            at = (s["ids"] == j).nonzero()[:, 0]
            if len(at):
                low = s["x"][at].double() @ s["a"][j].double().t().contiguous()
                out[at] += s["scale"][j].double() * (low @ s["b"][j].double().t().contiguous())
        return out
    s = _block_inputs(c, seed)
    if op == "enter":
        return _affine64(_norm64(s["h"].double(), c["norm"])[0], s["gamma"], s["beta"])
    if op == "enter_back":
        xh, r = _norm64(s["h"].double(), c["norm"])
        dn = s["dn"].double()
        return {"dh": s["dres"].double() + _pull64(xh, r, c["norm"], dn * s["gamma"].double()),
                "dgamma": (dn * xh).sum(dim=0), "dbeta": dn.sum(dim=0) if c["beta"] else None}
    y, kind = s["y"].double(), c["norm_out"]
    xh, r = _norm64(y, kind) if kind != "none" else (None, None)
    m = y if kind == "none" else _affine64(xh, s["gamma"], s["beta"])
    act = slope = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    if c["gate"] != "none":
        z = s["gate"].double()
        z = z.reshape(c["T"], 1) if c["gate"] == "token" else z.reshape(-1, c["d"])
        act = torch.sigmoid(z) if c["sigmoid"] else z
        slope = act * (1.0 - act) if c["sigmoid"] else torch.ones_like(z)
    if op == "exit":
        h = c["res_scale"] * s["h"].double() + c["out_scale"] * act * m
        n = None
        if c["next"]:       # of the residual stream as it is stored
            n = _affine64(_norm64(h.to(_type(c["h_bf16"])).double(), c["norm"])[0], s["gamma_next"], s["beta_next"])
        return {"h_out": h, "n_next": n}
    up = s["dh_out"].double()
    out = {"dh": c["res_scale"] * up, "dgate": None, "dgamma": None, "dbeta": None}
    if c["gate"] != "none":
        dg = c["out_scale"] * up * m * slope
        out["dgate"] = dg.sum(dim=0) if c["gate"] == "channel" else dg.sum(dim=1) if c["gate"] == "token" else dg
    dm = c["out_scale"] * up * act
    if kind == "none":
        out["dy"] = dm
        return out
    out["dgamma"], out["dbeta"] = (dm * xh).sum(dim=0), dm.sum(dim=0) if c["beta"] else None
    out["dy"] = _pull64(xh, r, kind, dm * s["gamma"].double())
    return out
