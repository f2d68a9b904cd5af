"""Performance cases of more operators on feature rows, through the public entry points, beside
their plain forms and a 64-bit reference of every result.

A block between two sparse convolutions adds its input to the features, normalises them, sends
them through dense and through routed products, and keeps what the backward pass will ask for:

  rms      root-mean-square norm of every row with the residual's addition; its output in the
           rows' type or in 8 bits with a scale a row; its gradients, from the rows themselves or
           from their 8-bit copy;
  linear   a product with bias, activation and residual in its epilogue, of rows in bf16, fp32 or
           8 bits; the gradients of its input (through the activation before it), weights, bias;
  scores   routing by sigmoid or softmax scores with a bias for balance, in groups of experts,
           the weights renormalised and scaled; the gradient of the weights;
  pack     rows in 8 bits with a scale a row, as a checkpoint of an activation's input; the
           activation and its gradient from that checkpoint.

`dir` of a case: "fwd", "bwd", or "train" for both in one pass.
"""
import math

import torch

own = False

DEV = "cuda"
F8 = torch.float8_e4m3fn
F8_MAX = 448.0                       # the largest e4m3 number
SMALLEST = 2.0 ** -100               # the smallest largest value a row's scale is made for

# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
BASE = dict(op="rms", dir="fwd", dtype="bf16", n=1, c=64, affine=True, residual=False,
            packed=False, c_out=64, bias=True, act="", pre=False, act_in="", experts=8, k=2,
            score="sigmoid", balance=True, groups=1, top_groups=1, normalize=True, scale=1.0,
            masked=False)


def _case(**kw):
    return dict(BASE, **kw)


def listed():
    return [
        # one handwritten character after its first layer (pen64_vsc3_c1x16): latency
        _case(name="rms_pen1_fwd_f32", n=461, c=16, dtype="f32", residual=True),
        # training on the benchmark's sites (surf128x8_vsc3_c64_bf16): every row joins the stream
        _case(name="rms_surf128_train_bf16", dir="train", n=902504, c=64, residual=True),
        # 16 surfaces of 64^3, normalised for a product that reads 8 bits
        _case(name="rms_surf64_fwd_e4m3", n=348208, c=256, residual=True, packed=True),
        # gradients from 8-bit checkpoints, a width that is no multiple of any vector
        _case(name="rms_odd_bwd_e4m3", dir="bwd", n=87052, c=145, dtype="f32", residual=True,
              packed=True),
        # one row at a time: the weights' bytes
        _case(name="linear_one_fwd_bf16", op="linear", c=512, c_out=2048, act="silu"),
        # a batch of characters in fp32 (pen64_train_f32's sites), widths that are no power of two
        _case(name="linear_pen64_train_f32", op="linear", dir="train", n=29760, c=96, c_out=200,
              dtype="f32", act="relu", residual=True, pre=True, act_in="silu"),
        # the largest: 16 surfaces of 64^3, 256 -> 1024 with its activation, in training
        _case(name="linear_surf64_train_bf16", op="linear", dir="train", n=348208, c=256,
              c_out=1024, act="gelu", pre=True, act_in="gelu"),
        # 8-bit rows through a product wide enough to be bound by the matrix cores, and their part
        # in the backward pass
        _case(name="linear_wide_train_e4m3", op="linear", dir="train", n=16384, c=2048, c_out=2048,
              dtype="e4m3", act_in="silu"),
        # 16 surfaces of 64^3 to 8 of 64 experts from 4 of 8 groups, with a bias for balance
        _case(name="scores_surf64_fwd_f32", op="scores", n=348208, dtype="f32", experts=64, k=8,
              groups=8, top_groups=4, scale=2.5),
        # a batch of characters, softmax scores without groups, some experts closed to some rows
        _case(name="scores_pen64_train_bf16", op="scores", dir="train", n=29760, experts=16, k=2,
              score="softmax", masked=True),
        # an activation's input kept in 8 bits, and its part in the backward pass
        _case(name="pack_surf64_train_bf16", op="pack", dir="train", n=348208, c=256, act="gelu"),
        # a few rows of fp32 features kept
        _case(name="pack_pen1_fwd_f32", op="pack", n=461, c=145, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi):
    """Plane counts: mostly multiples of 16, some of 8, a few odd ones."""
    v, u = _log_int(rng, 8, hi), rng.random()
    if u < 0.6:
        return max(16, v // 16 * 16)
    return max(8, v // 8 * 8) if u < 0.8 else v


def draw(rng):
    """One more case: any operator and direction, 1 to 902,504 rows, 8 to 2048 planes (odd ones
    among them), 2 to 256 experts in 1 to 16 groups, 1 to 8 of them for a row, every type.  The
    elements and the products stay within the listed cases'."""
    while True:
        op = rng.choice(["rms", "rms", "linear", "linear", "linear", "scores", "scores", "pack"])
        c = _case(op=op, dir=rng.choice(["fwd", "bwd", "train"]),
                  dtype=rng.choice(["f32", "bf16", "bf16"]), n=_log_int(rng, 1, 902504),
                  c=_width(rng, 2048), affine=rng.random() < 0.8, residual=rng.random() < 0.6,
                  packed=rng.random() < 0.4, c_out=_width(rng, 2048), bias=rng.random() < 0.8,
                  act=rng.choice(["", "relu", "gelu", "silu"]), pre=rng.random() < 0.4,
                  act_in=rng.choice(["", "relu", "gelu", "silu"]),
                  score=rng.choice(["sigmoid", "sigmoid", "softmax"]),
                  balance=rng.random() < 0.7, normalize=rng.random() < 0.7,
                  scale=rng.choice([1.0, 1.0, 2.5]), masked=rng.random() < 0.3)
        if op == "linear" and c["dtype"] == "bf16" and rng.random() < 0.4:
            c["dtype"] = "e4m3"
        c["groups"] = rng.choice([1, 1, 2, 4, 8, 16])
        c["experts"] = c["groups"] * max(1, _log_int(rng, 2, 256) // c["groups"])
        c["top_groups"] = rng.randint(max(1, c["groups"] // 4), c["groups"])
        c["k"] = min(c["top_groups"] * (c["experts"] // c["groups"]),
                     rng.choice([1, 2, 2, 3, 4, 6, 8, 8]))
        size = {"rms": c["n"] * c["c"], "linear": c["n"] * max(c["c"], c["c_out"]),
                "scores": c["n"] * max(c["experts"], 8 * c["k"]), "pack": c["n"] * c["c"]}[op]
        if size > {"rms": 5.7e7, "linear": 3.5e8, "scores": 2.2e7, "pack": 8.9e7}[op]:
            continue
        if op == "linear" and c["n"] * c["c"] * c["c_out"] > 6.8e10:
            continue
        return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(int(seed) * 13 + 7)

    def __call__(self, shape, std=1.0, dtype=torch.float32, mean=0.0):
        return (torch.randn(shape, generator=self.g, device=DEV) * std + mean).to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def _eight_bits(x):
    """Rows as a checkpoint holds them: (e4m3 values, a scale a row)."""
    top = x.float().abs().amax(1, keepdim=True).clamp(min=SMALLEST)
    return (x.float() * (F8_MAX / top)).to(F8), (top / F8_MAX).reshape(-1)


def prepare(case, seed):
    r, dt, op = _Rand(seed), _dtype(case), case["op"]
    n, c, k, E = case["n"], case["c"], case["k"], case["experts"]
    fwd, back = case["dir"] != "bwd", case["dir"] != "fwd"
    t = dict(case=case)
    if op == "rms":
        # rows of different sizes, as a residual stream has them
        t["x"] = r((n, c), 1.0, dt)
        t["res"] = (r((n, c)) * (0.5 + 2 * r.uniform((n, 1)))).to(dt) if case["residual"] else None
        t["g"] = r(c, 0.2, mean=1.0) if case["affine"] else None
        t["eps"] = 1e-6
        if back:
            t["dy"] = r((n, c), 1.0, dt)
            # what reaches the sum past the norm
            t["dh"] = r((n, c), 1.0, dt) if case["residual"] else None
        if not fwd:
            # kept from the forward pass: the sum (or its 8-bit copy) and its norms
            h = t["x"] if t["res"] is None else (t["x"].float() + t["res"].float()).to(dt)
            t["rstd"] = (h.double().square().mean(1) + t["eps"]).rsqrt().float()
            t["h"], t["h8"] = (None, _eight_bits(h)) if case["packed"] else (h, None)
            t["x"] = t["res"] = None
    elif op == "linear":
        co = case["c_out"]
        x = r((n, c), 1.0, dt)
        t["x"], t["x8"] = (None, _eight_bits(x)) if case["dtype"] == "e4m3" else (x, None)
        t["w"] = r((c, co), 1.0 / math.sqrt(c), dt)
        t["b"] = r(co, 0.1) if case["bias"] else None
        t["res"] = r((n, co), 1.0, dt) if case["residual"] and fwd else None
        if back:
            t["dy"] = r((n, co), 1.0, dt)
            # the input of the activation that this product's input came out of
            t["pre"], t["pre8"] = None, None
            if case["act_in"]:
                t["pre"] = r((n, c), 1.5, dt)
                if case["dtype"] == "e4m3":
                    t["pre"], t["pre8"] = None, _eight_bits(t["pre"])
    elif op == "scores":
        # popular and unpopular experts, and the bias that has grown against it
        lean = r((E,), 0.7)
        x = r((n, E)) + lean
        if case["masked"]:
            x = x.masked_fill(r.uniform(x.shape) < 1 / 6, -math.inf)
            x = x.masked_fill(r.uniform((n, 1)) < 0.01, -math.inf)
        t["logits"] = x.to(dt)
        t["balance"] = r((E,), 0.02) - 0.1 * lean if case["balance"] else None
        if back:
            t["dw"] = r((n, k))
        if not fwd:
            # kept from the forward pass
            t["experts"], t["weights"] = _plain_choice(t, case)
    else:
        x = r((n, c), 1.5, dt)
        t["x"] = x if fwd else None
        if back:
            t["dy"] = r((n, c), 1.0, dt)
        if not fwd:
            t["x8"] = _eight_bits(x)
    return t


# ---------------------------------------------------------------------------
# Plain forms: elementary torch operations in 32 bits (64 where the choice of experts is made)
# ---------------------------------------------------------------------------
def _plain_pack(x):
    """(e4m3 values, scales) of fp32 rows; a row with an infinity or NaN has scale NaN and zeros."""
    top = x.abs().amax(1, keepdim=True)
    fine = top < math.inf
    top = top.clamp(min=SMALLEST)
    q = torch.where(fine, x * (F8_MAX / top), 0.0).to(F8)
    return q, torch.where(fine, top / F8_MAX, math.nan).reshape(-1)


def _plain_unpack(x8):
    return x8[0].float() * x8[1][:, None]


def _plain_act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return z / (1.0 + torch.exp(-2.0 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _plain_slope(z, act):
    """The activation's derivative."""
    if act == "relu":
        return torch.where(z <= 0, 0.0, 1.0)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        a = 2.0 * math.sqrt(2 / math.pi)
        s = 1.0 / (1.0 + torch.exp(-a * (z + 0.044715 * z * z * z)))
        return s + z * s * (1.0 - s) * a * (1.0 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain_rms(t, c):
    out, dt = {}, _dtype(c)
    if c["dir"] != "bwd":
        h = t["x"] if t["res"] is None else (t["x"].float() + t["res"].float()).to(dt)
        hf = h.float()
        rstd = 1.0 / (hf.square().mean(1) + t["eps"]).sqrt()
        y = hf * rstd[:, None]
        y = y if t["g"] is None else y * t["g"]
        if c["packed"]:
            out["q"], out["scale"] = _plain_pack(y)
        else:
            out["y"] = y.to(dt)
        out["rstd"] = rstd
        if t["res"] is not None:
            out["h"] = h
    else:
        rstd = t["rstd"]
        hf = t["h"].float() if t["h8"] is None else _plain_unpack(t["h8"])
    if c["dir"] != "fwd":
        dy, z = t["dy"].float(), hf * rstd[:, None]
        gd = dy if t["g"] is None else dy * t["g"]
        dx = rstd[:, None] * (gd - z * (gd * z).mean(1, keepdim=True))
        out["dx"] = (dx if t["dh"] is None else dx + t["dh"].float()).to(dt)
        if t["g"] is not None:
            out["dgamma"] = (dy * z).sum(0)
    return out


def _plain_linear(t, c):
    out, dt = {}, _dtype(c)
    x = t["x"].float() if t["x8"] is None else _plain_unpack(t["x8"])
    w = t["w"].float()
    if c["dir"] != "bwd":
        z = x @ w
        z = z if t["b"] is None else z + t["b"]
        if c["pre"]:
            out["z"] = z.to(dt)
        y = _plain_act(z, c["act"])
        out["y"] = (y if t["res"] is None else y + t["res"].float()).to(dt)
    if c["dir"] != "fwd":
        dy = t["dy"].float()
        dx = dy @ w.T
        if c["act_in"]:
            pre = t["pre"].float() if t["pre8"] is None else _plain_unpack(t["pre8"])
            dx = dx * _plain_slope(pre, c["act_in"])
        out["dx"] = dx.to(dt)
        out["dw"], out["db"] = x.T @ dy, dy.sum(0)
    return out


def _plain_choice(t, c):
    """(experts [N, k], -1 for none; weights): the largest score first, biased, the lowest index
    among equals, out of the groups whose two best add up to most."""
    x, E, G = t["logits"].double(), c["experts"], c["groups"]
    n, none = len(x), -math.inf
    shut = x == none
    if c["score"] == "softmax":
        top = x.max(1, keepdim=True).values
        s = torch.exp(x - torch.where(top > none, top, 0.0))
        total = s.sum(1, keepdim=True)
        s = s / torch.where(total > 0, total, 1.0)
    else:
        s = 1.0 / (1.0 + torch.exp(-x))
    v = s if t["balance"] is None else s + t["balance"].double()
    v = v.masked_fill(shut, none)
    if G > 1:
        best = torch.sort(v.view(n, G, E // G), dim=2, descending=True).values[:, :, :2]
        worth = torch.where(best > none, best, 0.0).sum(2).masked_fill(best[:, :, 0] == none, none)
        rank = torch.sort(worth, dim=1, descending=True, stable=True).indices
        stay = torch.zeros_like(worth, dtype=torch.bool)
        stay.scatter_(1, rank[:, :c["top_groups"]], True)
        v = v.masked_fill(~stay.repeat_interleave(E // G, 1), none)
    v, e = torch.sort(v, dim=1, descending=True, stable=True)
    v, e = v[:, :c["k"]], e[:, :c["k"]]
    some = v > none
    w = torch.where(some, s.gather(1, e), 0.0)
    if c["normalize"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, 1.0)
    return torch.where(some, e, -1).to(torch.int32), (w * c["scale"]).float()


def _plain_scores(t, c):
    out, E = {}, c["experts"]
    if c["dir"] == "bwd":
        e, w = t["experts"], t["weights"]
    else:
        e, w = _plain_choice(t, c)
        flat = torch.where(e < 0, E, e).reshape(-1).long()
        order = torch.sort(flat, stable=True).indices
        offsets = torch.bincount(flat, minlength=E + 1)[:E].cumsum(0)
        at = torch.arange(flat.numel(), device=DEV)
        pos = torch.empty_like(order)
        pos[order] = at
        out.update(experts=e, weights=w,
                   offsets=torch.cat([offsets.new_zeros(1), offsets]).to(torch.int32),
                   rows=torch.where(at < offsets[-1], order // c["k"], -1).to(torch.int32),
                   pos=torch.where(e < 0, -1, pos.reshape(e.shape)).to(torch.int32))
    if c["dir"] != "fwd":
        x, scale, chosen = t["logits"].float(), c["scale"], e.clamp(min=0).long()
        dw = torch.where(e < 0, 0.0, t["dw"])
        dot = (w * dw).sum(1, keepdim=True)
        dl = torch.zeros_like(x)
        if c["score"] == "softmax":
            if c["normalize"]:
                g = w * (dw - dot / scale)
            else:
                top = x.max(1, keepdim=True).values
                p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
                total = p.sum(1, keepdim=True)
                dl, g = -p / torch.where(total > 0, total, 1.0) * dot, w * dw
        else:
            s = 1.0 / (1.0 + torch.exp(-x.gather(1, chosen)))
            s = torch.where(e < 0, 0.0, s)
            g = dw * scale
            if c["normalize"]:
                total = s.sum(1, keepdim=True)
                g = (g - dot) / torch.where(total > 0, total, 1.0)
            g = g * s * (1.0 - s)
        dl = dl.scatter_add(1, chosen, torch.where(e < 0, 0.0, g))
        out["dlogits"] = dl.to(t["logits"].dtype)
    return out


def _plain_checkpoint(t, c):
    out, dt = {}, _dtype(c)
    x8 = t.get("x8")
    if c["dir"] != "bwd":
        x8 = _plain_pack(t["x"].float())
        out["q"], out["scale"] = x8
    if c["dir"] != "fwd":
        z = _plain_unpack(x8)
        out["a"] = _plain_act(z, c["act"]).to(dt)
        out["dz"] = (t["dy"].float() * _plain_slope(z, c["act"])).to(dt)
    return out


PLAIN = dict(rms=_plain_rms, linear=_plain_linear, scores=_plain_scores, pack=_plain_checkpoint)


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _own_rms(spc, t, c):
    out, rstd = {}, t.get("rstd")
    if c["dir"] != "bwd":
        y, h, rstd = spc.rms_norm_forward(t["x"], t["g"], t["eps"], residual=t["res"],
                                          packed=c["packed"])
        if c["packed"]:
            out.update(q=y.q, scale=y.scale)
        else:
            out["y"] = y
        out["rstd"] = rstd
        if t["res"] is not None:
            out["h"] = h
    else:
        h = t["h"] if t["h8"] is None else spc.Rows8(*t["h8"])
    if c["dir"] != "fwd":
        out["dx"], dg = spc.rms_norm_backward(t["dy"], h, rstd, t["g"], dh=t["dh"])
        if dg is not None:
            out["dgamma"] = dg
    return out


def _own_linear(spc, t, c):
    out = {}
    x = t["x"] if t["x8"] is None else spc.Rows8(*t["x8"])
    if c["dir"] != "bwd":
        y, z = spc.linear_forward(x, t["w"], t["b"], act=c["act"] or None, residual=t["res"],
                                  pre=c["pre"])
        if c["pre"]:
            out["z"] = z
        out["y"] = y
    if c["dir"] != "fwd":
        pre = t["pre"] if t["pre8"] is None else spc.Rows8(*t["pre8"])
        out["dx"] = spc.linear_backward_data(t["dy"], t["w"], act=c["act_in"] or None, pre=pre)
        out["dw"], out["db"] = spc.linear_backward_weight(x, t["dy"])
    return out


def _own_scores(spc, t, c):
    out = {}
    e, w = t.get("experts"), t.get("weights")
    how = dict(score=c["score"], normalize=c["normalize"], scale=c["scale"])
    if c["dir"] != "bwd":
        r = spc.route_scores_forward(t["logits"], c["k"], bias=t["balance"], groups=c["groups"],
                                     top_groups=c["top_groups"], **how)
        e, w = r.experts, r.weights
        out.update(experts=e, weights=w, offsets=r.offsets, rows=r.rows, pos=r.pos)
    if c["dir"] != "fwd":
        out["dlogits"] = spc.route_scores_backward(t["dw"], t["logits"], e, w, **how)
    return out


def _own_checkpoint(spc, t, c):
    out = {}
    if c["dir"] != "bwd":
        x8 = spc.pack_rows(t["x"])
        out.update(q=x8.q, scale=x8.scale)
    else:
        x8 = spc.Rows8(*t["x8"])
    if c["dir"] != "fwd":
        out["a"] = spc.unpack_rows(x8, t["dy"].dtype, act=c["act"] or None)
        out["dz"] = spc.activation_backward(t["dy"], x8, c["act"] or None)
    return out


OWN = dict(rms=_own_rms, linear=_own_linear, scores=_own_scores, pack=_own_checkpoint)


def run(state):
    case = state["case"]
    if own:
        import paper_1706_01307_amd as spc
        return OWN[case["op"]](spc, state, case)
    return PLAIN[case["op"]](state, case)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_act(z, act):
    """(value, derivative)."""
    one = torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0) * one
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if act == "gelu":
        u = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        t = torch.tanh(u)
        return (0.5 * z * (1 + t),
                0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) *
                (1 + 3 * 0.044715 * z ** 2))
    return z, one


def _exact_rows(x8):
    return x8[0].double() * x8[1].double().view(-1, 1)


def _exact_packed(y):
    """What the 8-bit values round, and the scales."""
    top = y.abs().max(1).values.clamp(min=SMALLEST)
    return y * (F8_MAX / top).view(-1, 1), top / F8_MAX


def _exact_rms(t, c):
    out = {}
    if c["dir"] != "bwd":
        h = t["x"].double()
        if t["res"] is not None:
            # the sum as it is kept
            h = (h + t["res"].double()).to(_dtype(c))
            out["h"], h = h.double(), h.double()
        r = ((h ** 2).sum(1, keepdim=True) / c["c"] + t["eps"]) ** -0.5
        y = h * r if t["g"] is None else h * r * t["g"].double()
        out["rstd"] = r[:, 0]
        if c["packed"]:
            out["q"], out["scale"] = _exact_packed(y)
        else:
            out["y"] = y
    else:
        h = t["h"].double() if t["h8"] is None else _exact_rows(t["h8"])
        r = t["rstd"].double().view(-1, 1)
    if c["dir"] != "fwd":
        d = t["dy"].double()
        u = d if t["g"] is None else d * t["g"].double()
        out["dx"] = r * u - h * r ** 3 * ((u * h).sum(1, keepdim=True) / c["c"])
        if t["dh"] is not None:
            out["dx"] = out["dx"] + t["dh"].double()
        if t["g"] is not None:
            out["dgamma"] = (d * h * r).sum(0)
    return out


def _exact_linear(t, c):
    n, w, step = c["n"], t["w"].double(), 1 << 16
    wt, fwd, back = w.t().contiguous(), c["dir"] != "bwd", c["dir"] != "fwd"
    parts = {}
    dw = torch.zeros_like(w)
    for a in range(0, n, step):
        s = slice(a, a + step)
        x = t["x"][s].double() if t["x8"] is None else _exact_rows([v[s] for v in t["x8"]])
        if fwd:
            z = x @ w
            z = z if t["b"] is None else z + t["b"].double()
            if c["pre"]:
                parts.setdefault("z", []).append(z)
            y = _exact_act(z, c["act"])[0]
            parts.setdefault("y", []).append(y if t["res"] is None else y + t["res"][s].double())
        if back:
            d = t["dy"][s].double()
            g = d @ wt
            if c["act_in"]:
                p = (t["pre"][s].double() if t["pre8"] is None
                     else _exact_rows([v[s] for v in t["pre8"]]))
                g = g * _exact_act(p, c["act_in"])[1]
            parts.setdefault("dx", []).append(g)
            dw += x.t().contiguous() @ d
    out = {name: torch.cat(v) for name, v in parts.items()}
    if back:
        out["dw"], out["db"] = dw, t["dy"].double().sum(0)
    return out


def _exact_scores(t, c):
    x = t["logits"].double()
    n, E = x.shape
    k, none, per = c["k"], -math.inf, E // c["groups"]
    cols = torch.arange(E, device=DEV).expand(n, E)
    if c["score"] == "sigmoid":
        s = torch.sigmoid(x)
    else:
        s = torch.nan_to_num(torch.softmax(x, 1), nan=0.0)      # (a row that is all closed)
    out = {}
    if c["dir"] != "bwd":
        left = s + (0 if t["balance"] is None else t["balance"].double())
        left = torch.where(x == none, none, left)
        # the groups, the best left at a time
        worth = torch.zeros((n, c["groups"]), dtype=torch.float64, device=DEV)
        for g in range(c["groups"]):
            two = left[:, g * per:(g + 1) * per].topk(min(2, per), dim=1).values
            worth[:, g] = torch.where(two[:, 0] > none, torch.where(two > none, two, 0.0).sum(1),
                                      none)
        keep, gs = torch.zeros_like(worth, dtype=torch.bool), torch.arange(c["groups"], device=DEV)
        for _ in range(c["top_groups"]):
            w = torch.where(keep, none, worth)
            first = torch.where((w == w.max(1, keepdim=True).values) & ~keep, gs,
                                c["groups"]).min(1).values
            keep |= gs == first[:, None]
        left = torch.where(keep[:, torch.arange(E, device=DEV) // per], left, none)
        # one expert at a time: the largest left, of equal ones the first
        experts = torch.full((n, k), -1, dtype=torch.int64, device=DEV)
        for j in range(k):
            best = left.max(1, keepdim=True).values
            first = torch.where(left == best, cols, E).min(1, keepdim=True).values
            experts[:, j] = torch.where(best[:, 0] > none, first[:, 0], -1)
            left = torch.where((cols == first) & (best > none), none, left)
    else:
        experts = t["experts"].long()
    some = experts >= 0
    chosen = torch.where(some, s.gather(1, experts.clamp(min=0)), 0.0)
    total = chosen.sum(1, keepdim=True)
    total = torch.where(total > 0, total, 1.0) if c["normalize"] else torch.ones_like(total)
    if c["dir"] != "bwd":
        flat = experts.reshape(-1)
        order = torch.argsort(torch.where(flat < 0, E, flat), stable=True)
        used = int((flat >= 0).sum())
        pos, rows = torch.full_like(flat, -1), torch.full_like(flat, -1)
        pos[order[:used]] = torch.arange(used, device=DEV)
        rows[:used] = order[:used] // k
        count = torch.stack([(flat == e).sum() for e in range(E)])
        out = {"experts": experts, "weights": c["scale"] * chosen / total, "rows": rows,
               "pos": pos.view(n, k),
               "offsets": torch.cat([count.new_zeros(1), count.cumsum(0)])}
    if c["dir"] != "fwd":
        # through the scores: the gradient of every score, then of the logits
        d = torch.where(some, t["dw"].double(), 0.0) * c["scale"]
        if c["normalize"]:
            d = (d - (d * chosen / total).sum(1, keepdim=True)) / total
        ds = torch.zeros_like(x)
        ds.scatter_add_(1, experts.clamp(min=0), torch.where(some, d, 0.0))
        if c["score"] == "sigmoid":
            out["dlogits"] = ds * s * torch.sigmoid(-x)
        else:
            out["dlogits"] = s * (ds - (ds * s).sum(1, keepdim=True))
    return out


def _exact_checkpoint(t, c):
    out = {}
    if c["dir"] != "bwd":
        out["q"], out["scale"] = _exact_packed(t["x"].double())
        z = out["q"].float().to(F8).double() * out["scale"].view(-1, 1)
    else:
        z = _exact_rows(t["x8"])
    if c["dir"] != "fwd":
        out["a"], slope = _exact_act(z, c["act"])
        out["dz"] = t["dy"].double() * slope
    return out


EXACT = dict(rms=_exact_rms, linear=_exact_linear, scores=_exact_scores, pack=_exact_checkpoint)


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed), case)


# ---------------------------------------------------------------------------
# Work
# ---------------------------------------------------------------------------
def work(case):
    """Inputs read once, outputs written once; a pass of both directions counts what they share
    once.  Rows in 8 bits take a byte an element and four a row."""
    n, c, co, k, E = case["n"], case["c"], case["c_out"], case["k"], case["experts"]
    fwd, back, op = case["dir"] != "bwd", case["dir"] != "fwd", case["op"]
    e, x8, res = 4 if case["dtype"] == "f32" else 2, n * (c + 4), case["residual"]
    x = e * n * c
    if op == "rms":
        by = 4 * n + 4 * c * case["affine"] * (1 + back)
        if fwd:
            by += x * (1 + 2 * res) + (x8 if case["packed"] else x)
        if back:
            by += x * (2 + res) + (0 if fwd else x8 if case["packed"] else x)
        return {"bytes": by, "flops": n * c * (5 * fwd + 9 * back)}
    if op == "linear":
        by = (x8 if case["dtype"] == "e4m3" else x) + e * c * co
        if fwd:
            by += e * n * co * (1 + res + case["pre"]) + 4 * co * case["bias"]
        if back:
            pre = bool(case["act_in"]) * (x8 if case["dtype"] == "e4m3" else x)
            by += e * n * co + x + pre + 4 * (c + 1) * co
        return {"bytes": by, "flops": 2 * n * c * co * (fwd + 2 * back)}
    if op == "scores":
        m, by = n * k, e * n * E * (1 + back)
        if fwd:
            by += 16 * m + 4 * E * (1 + case["balance"])
        if back:
            by += 4 * m + (0 if fwd else 8 * m)
        if back and not fwd and case["score"] == "softmax" and case["normalize"]:
            by -= e * n * E                        # (nothing asks for the logits)
        return {"bytes": by, "flops": n * E * (6 * fwd + 6 * back)}
    return {"bytes": x8 + x * (fwd + 3 * back), "flops": n * c * (3 * fwd + 20 * back)}
