"""Performance cases of the operators on feature rows, through the public entry points, beside
their plain forms and a 64-bit reference of every result.

A program that has a sparse network's features as rows (one per active site) normalises them,
sends every row to a few of many experts, multiplies each expert's rows by that expert's weights,
puts the results together again and drops some of the elements before they are added back:

  norm      layer norm of every row, and its gradients (rows, scale and shift);
  dropout   elements dropped by a counter-based generator, with the residual added;
  route     the k largest logits of every row, their softmax weights, and the rows grouped by
            expert; its gradient;
  grouped   products grouped by expert with ragged sizes, rows gathered on the way in; input,
            weight and bias gradients;
  combine   the weighted sum of a row's expert outputs; its gradients.

`dir` of a case: "fwd", "bwd", or "train" for both in one pass.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"

# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------
BASE = dict(op="norm", dir="fwd", dtype="bf16", n=1, c=64, affine=True, residual=False, p=0.1,
            experts=8, k=2, normalize=True, masked=False, c_out=64, gather=False, relu=False)


def _case(**kw):
    return dict(BASE, **kw)


def listed():
    return [
        # one handwritten character after its first layer (pen64_vsc3_c1x16): latency
        _case(name="norm_pen1_fwd_f32", n=461, c=16, dtype="f32"),
        # training on the benchmark's sites (surf128x8_vsc3_c64_bf16)
        _case(name="norm_surf128_train_bf16", dir="train", n=902504, c=64),
        # a width that is no multiple of any vector, 4 surfaces of 64^3, gradients
        _case(name="norm_odd_bwd_f32", dir="bwd", n=87052, c=145, dtype="f32"),
        # the benchmark's sites: dropped and added to the block's input
        _case(name="dropout_surf128_fwd_bf16", op="dropout", n=902504, c=64, residual=True),
        # a batch of characters in training, fp32 (pen64_train_f32's sites and planes)
        _case(name="dropout_pen64_train_f32", op="dropout", dir="train", n=29760, c=32,
              dtype="f32", p=0.5),
        # 16 surfaces of 64^3 sent to 2 of 64 experts, fp32 logits
        _case(name="route_surf64_fwd_f32", op="route", n=348208, experts=64, dtype="f32"),
        # a batch of characters, 8 experts of which some are closed to some rows
        _case(name="route_pen64_train_bf16", op="route", dir="train", n=29760, experts=8,
              normalize=False, masked=True),
        # one row at a time through 4 of 32 experts: the weights' bytes
        _case(name="grouped_one_fwd_bf16", op="grouped", n=1, experts=32, k=4, c=512, c_out=2048,
              gather=True, relu=True),
        # a batch of characters in fp32, widths that are no power of two
        _case(name="grouped_pen64_train_f32", op="grouped", dir="train", n=29760, experts=8, c=96,
              c_out=200, gather=True, dtype="f32"),
        # the largest: 16 surfaces of 64^3 through 2 of 16 experts, 256 -> 1024, in training
        _case(name="grouped_surf64_train_bf16", op="grouped", dir="train", n=348208, experts=16,
              c=256, c_out=1024, gather=True, relu=True),
        # those experts' outputs put together, in training
        _case(name="combine_surf64_train_bf16", op="combine", dir="train", n=348208, c=256,
              experts=16),
        # one row's
        _case(name="combine_one_fwd_f32", op="combine", n=1, k=4, c=512, experts=32, dtype="f32",
              residual=True),
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
    among them), 2 to 256 experts, 1 to 8 of them for a row, both types.  The elements and the
    products stay within the listed cases'."""
    while True:
        op = rng.choice(["norm", "norm", "dropout", "dropout", "route", "route", "grouped",
                         "grouped", "grouped", "combine", "combine"])
        c = _case(op=op, dir=rng.choice(["fwd", "bwd", "train"]), dtype=rng.choice(["f32", "bf16"]),
                  n=_log_int(rng, 1, 902504), c=_width(rng, 2048), affine=rng.random() < 0.8,
                  residual=rng.random() < 0.5, p=rng.choice([0.0, 0.1, 0.25, 0.5, 0.9]),
                  experts=_log_int(rng, 2, 256), normalize=rng.random() < 0.5,
                  masked=rng.random() < 0.3, c_out=_width(rng, 2048),
                  gather=rng.random() < 0.6, relu=rng.random() < 0.5)
        c["k"] = min(c["experts"], rng.choice([1, 2, 2, 2, 3, 4, 6, 8]))
        m = c["n"] * c["k"]
        size = {"norm": c["n"] * c["c"], "dropout": c["n"] * c["c"],
                "route": c["n"] * max(c["experts"], 4 * c["k"]),
                "grouped": m * max(c["c"], c["c_out"]), "combine": m * c["c"]}[op]
        if size > (4e8 if op in ("grouped", "combine") else 5.8e7):
            continue
        if op == "grouped" and (m * c["c"] * c["c_out"] > 9e10 or
                                c["experts"] * c["c"] * c["c_out"] > 1.3e8):
            continue
        return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(int(seed) * 11 + 5)

    def __call__(self, shape, std=1.0, dtype=torch.float32, mean=0.0):
        return (torch.randn(shape, generator=self.g, device=DEV) * std + mean).to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def _logits(case, r):
    """Logits with popular and unpopular experts; where some are closed, one in six entries and
    every expert of about one row in a hundred."""
    x = r((case["n"], case["experts"])) + r((case["experts"],), 0.7)
    if case["masked"]:
        x = x.masked_fill(r.uniform(x.shape) < 1 / 6, -math.inf)
        x = x.masked_fill(r.uniform((case["n"], 1)) < 0.01, -math.inf)
    return x.to(_dtype(case))


def _grouping(case, r):
    """Rows sent to k distinct experts each, grouped by expert: (offsets [E + 1], row of every
    position, position of every (row, slot))."""
    n, k, E = case["n"], case["k"], case["experts"]
    e = (r((n, E)) + r((E,), 0.7)).topk(k, dim=1).indices.reshape(-1)
    order = torch.sort(e, stable=True).indices
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = torch.bincount(e, minlength=E).cumsum(0)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(n * k, device=DEV)
    return (offsets.to(torch.int32), (order // k).to(torch.int32),
            pos.reshape(n, k).to(torch.int32))


def prepare(case, seed):
    r, dt, op = _Rand(seed), _dtype(case), case["op"]
    n, c, k, E = case["n"], case["c"], case["k"], case["experts"]
    t = dict(case=case)
    back = case["dir"] != "fwd"
    if op == "norm":
        # rows of different means and sizes, as a residual stream has them
        t["x"] = (r((n, c)) * (0.5 + r.uniform((n, 1))) + r((n, 1), 0.5)).to(dt)
        t["g"], t["b"] = (r(c, 0.2, mean=1.0), r(c, 0.1)) if case["affine"] else (None, None)
        t["eps"] = 1e-5
        if back:
            t["dy"] = r((n, c), 1.0, dt)
        if case["dir"] == "bwd":
            # kept from the forward pass
            x = t["x"].double()
            t["mean"] = x.mean(1).float()
            t["rstd"] = (x.var(1, unbiased=False) + t["eps"]).rsqrt().float()
    elif op == "dropout":
        t["x"] = r((n, c), 1.0, dt)
        t["res"] = r((n, c), 1.0, dt) if case["residual"] else None
        t["seed"], t["offset"] = 0x9E3779B97F4A7C15 ^ (int(seed) * 2654435761), 2 ** 33 + 7
        if back:
            t["dy"] = r((n, c), 1.0, dt)
    elif op == "route":
        t["logits"] = _logits(case, r)
        if back:
            t["dw"] = r((n, k))
        if case["dir"] == "bwd":
            # kept from the forward pass
            t["experts"], t["weights"] = _plain_choice(t["logits"], k, case["normalize"])
    elif op == "grouped":
        t["offsets"], rows, _ = _grouping(case, r)
        t["rows"] = rows if case["gather"] else None
        t["x"] = r((n if case["gather"] else n * k, c), 1.0, dt)
        t["w"] = r((E, c, case["c_out"]), 1.0 / math.sqrt(c), dt)
        t["bias"] = r((E, case["c_out"]), 0.1)
        if back:
            t["dy"] = r((n * k, case["c_out"]), 1.0, dt)
            # the layer's input per position came out of a ReLU
            t["mask"] = r((n * k, c), 1.0, dt) if case["relu"] else None
    else:
        t["offsets"], _, t["pos"] = _grouping(case, r)
        t["y"] = r((n * k, c), 1.0, dt)
        t["w"] = torch.softmax(r((n, k)), 1)
        t["res"] = r((n, c), 1.0, dt) if case["residual"] else None
        if back:
            t["dout"] = r((n, c), 1.0, dt)
    return t


# ---------------------------------------------------------------------------
# Plain forms: elementary torch operations in 32 bits
# ---------------------------------------------------------------------------
def _plain_norm(t, c):
    out, x = {}, t["x"].float()
    if c["dir"] == "bwd":
        mean, rstd = t["mean"], t["rstd"]
    else:
        mean = x.mean(1)
        rstd = 1.0 / ((x - mean[:, None]).square().mean(1) + t["eps"]).sqrt()
    xh = (x - mean[:, None]) * rstd[:, None]
    if c["dir"] != "bwd":
        y = xh if t["g"] is None else xh * t["g"] + t["b"]
        out.update(y=y.to(t["x"].dtype), mean=mean, rstd=rstd)
    if c["dir"] != "fwd":
        dy = t["dy"].float()
        gd = dy if t["g"] is None else dy * t["g"]
        dx = rstd[:, None] * (gd - gd.mean(1, keepdim=True) -
                              xh * (gd * xh).mean(1, keepdim=True))
        out["dx"] = dx.to(t["x"].dtype)
        if t["g"] is not None:
            out.update(dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
    return out


def _plain_words(count, seed, offset):
    """`count` words of Philox4x32-7 (Salmon, Moraes, Dror and Shaw, 2011): four per counter
    (index, offset), under the key `seed`."""
    m32 = 0xFFFFFFFF
    i = torch.arange((count + 3) // 4, device=DEV)
    c0, c1 = i & m32, i >> 32
    c2, c3 = torch.full_like(i, offset & m32), torch.full_like(i, offset >> 32 & m32)
    k0, k1 = seed & m32, seed >> 32 & m32
    for _ in range(7):
        # the 64-bit product wraps into the sign; its halves are masked out of it
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32 & m32) ^ c1 ^ k0, b & m32, (a >> 32 & m32) ^ c3 ^ k1, a & m32)
        k0, k1 = (k0 + 0x9E3779B9) & m32, (k1 + 0xBB67AE85) & m32
    return torch.stack([c0, c1, c2, c3], 1).reshape(-1)[:count]


def _plain_drop(x, t, p, res=None):
    u = _plain_words(x.numel(), t["seed"], t["offset"]).reshape(x.shape)
    y = torch.where(u >= round(p * 2 ** 32), x.float() * (1.0 / (1.0 - p)), 0.0)
    return (y if res is None else res.float() + y).to(x.dtype)


def _plain_dropout(t, c):
    out = {}
    if c["dir"] != "bwd":
        out["y"] = _plain_drop(t["x"], t, c["p"], t["res"])
    if c["dir"] != "fwd":
        out["dx"] = _plain_drop(t["dy"], t, c["p"])
    return out


def _plain_choice(logits, k, normalize):
    """(experts [N, k], -1 for none; weights): largest first, the lowest index among equals."""
    x = logits.float()
    v, e = torch.sort(x, dim=1, descending=True, stable=True)
    v, e = v[:, :k], e[:, :k]
    some = v > -math.inf
    top = torch.where(some[:, :1], v[:, :1], 0.0)
    w = torch.exp(v - top)
    w = w / (w if normalize else torch.exp(x - top)).sum(1, keepdim=True)
    return torch.where(some, e, -1).to(torch.int32), torch.where(some, w, 0.0)


def _plain_route(t, c):
    out, E = {}, c["experts"]
    if c["dir"] == "bwd":
        e, w = t["experts"], t["weights"]
    else:
        e, w = _plain_choice(t["logits"], c["k"], c["normalize"])
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
        wd = torch.where(e < 0, 0.0, w * t["dw"])
        dot = wd.sum(1, keepdim=True)
        if c["normalize"]:
            dl = torch.zeros_like(t["logits"], dtype=torch.float32)
            wd = wd - w * dot
        else:
            x = t["logits"].float()
            top = x.max(1, keepdim=True).values
            p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
            s = p.sum(1, keepdim=True)
            dl = -p / torch.where(s > 0, s, 1.0) * dot
        dl = dl.scatter_add(1, e.clamp(min=0).long(), wd)
        out["dlogits"] = dl.to(t["logits"].dtype)
    return out


def _plain_grouped(t, c):
    out, off = {}, t["offsets"].tolist()
    dt = t["x"].dtype
    x = (t["x"] if t["rows"] is None else t["x"][t["rows"].long()]).float()
    w = t["w"].float()
    spans = [(e, a, b) for e, (a, b) in enumerate(zip(off[:-1], off[1:])) if b > a]
    if c["dir"] != "bwd":
        y = torch.empty((len(x), c["c_out"]), device=DEV)
        for e, a, b in spans:
            y[a:b] = x[a:b] @ w[e] + t["bias"][e]
        out["y"] = (torch.where(y < 0, 0.0, y) if c["relu"] else y).to(dt)
    if c["dir"] != "fwd":
        dy = t["dy"].float()
        dx, dw = torch.empty_like(x), torch.zeros_like(w)
        db = torch.zeros((len(w), c["c_out"]), device=DEV)
        for e, a, b in spans:
            dx[a:b] = dy[a:b] @ w[e].T
            dw[e] = x[a:b].T @ dy[a:b]
            db[e] = dy[a:b].sum(0)
        if t["mask"] is not None:
            dx = torch.where(t["mask"].float() <= 0, 0.0, dx)
        out.update(dx=dx.to(dt), dw=dw, db=db)
    return out


def _plain_combine(t, c):
    out, pos, dt = {}, t["pos"].long(), t["y"].dtype
    y = t["y"].float()
    if c["dir"] != "bwd":
        s = sum(t["w"][:, j:j + 1] * y[pos[:, j]] for j in range(c["k"]))
        out["out"] = (s if t["res"] is None else t["res"].float() + s).to(dt)
    if c["dir"] != "fwd":
        do, dy = t["dout"].float(), torch.zeros_like(y)
        for j in range(c["k"]):
            dy[pos[:, j]] = t["w"][:, j:j + 1] * do
        out["dy"] = dy.to(dt)
        out["dw"] = torch.stack([(do * y[pos[:, j]]).sum(1) for j in range(c["k"])], 1)
    return out


PLAIN = dict(norm=_plain_norm, dropout=_plain_dropout, route=_plain_route, grouped=_plain_grouped,
             combine=_plain_combine)


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------
def _own_norm(spc, t, c):
    out = {}
    mean, rstd = t.get("mean"), t.get("rstd")
    if c["dir"] != "bwd":
        y, mean, rstd = spc.layer_norm_forward(t["x"], t["g"], t["b"], eps=t["eps"])
        out.update(y=y, mean=mean, rstd=rstd)
    if c["dir"] != "fwd":
        out["dx"], dg, db = spc.layer_norm_backward(t["dy"], t["x"], mean, rstd, t["g"])
        if dg is not None:
            out.update(dgamma=dg, dbeta=db)
    return out


def _own_dropout(spc, t, c):
    out = {}
    if c["dir"] != "bwd":
        out["y"] = spc.dropout_forward(t["x"], c["p"], t["seed"], t["offset"], residual=t["res"])
    if c["dir"] != "fwd":
        out["dx"] = spc.dropout_backward(t["dy"], c["p"], t["seed"], t["offset"])
    return out


def _own_route(spc, t, c):
    out = {}
    e, w = t.get("experts"), t.get("weights")
    if c["dir"] != "bwd":
        r = spc.route_forward(t["logits"], c["k"], normalize=c["normalize"])
        e, w = r.experts, r.weights
        out.update(experts=e, weights=w, offsets=r.offsets, rows=r.rows, pos=r.pos)
    if c["dir"] != "fwd":
        out["dlogits"] = spc.route_backward(t["dw"], t["logits"], e, w, normalize=c["normalize"])
    return out


def _own_grouped(spc, t, c):
    out = {}
    if c["dir"] != "bwd":
        out["y"] = spc.grouped_forward(t["x"], t["w"], t["offsets"], rows=t["rows"],
                                       bias=t["bias"], relu=c["relu"])
    if c["dir"] != "fwd":
        out["dx"] = spc.grouped_backward_data(t["dy"], t["w"], t["offsets"], mask=t["mask"])
        out["dw"], out["db"] = spc.grouped_backward_weight(t["x"], t["dy"], t["offsets"],
                                                           rows=t["rows"])
    return out


def _own_combine(spc, t, c):
    out = {}
    if c["dir"] != "bwd":
        out["out"] = spc.combine_forward(t["y"], t["pos"], t["w"], residual=t["res"])
    if c["dir"] != "fwd":
        out["dy"], out["dw"] = spc.combine_backward(t["dout"], t["y"], t["pos"], t["w"],
                                                    offsets=t["offsets"])
    return out


OWN = dict(norm=_own_norm, dropout=_own_dropout, route=_own_route, grouped=_own_grouped,
           combine=_own_combine)


def run(state):
    case = state["case"]
    if own:
        import paper_1706_01307_amd as spc
        return OWN[case["op"]](spc, state, case)
    return PLAIN[case["op"]](state, case)


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_norm(t, c):
    x = t["x"].double()
    n, width = x.shape
    if c["dir"] == "bwd":
        m, r = t["mean"].double().view(n, 1), t["rstd"].double().view(n, 1)
    else:
        m = x.sum(1, keepdim=True) / width
        r = (((x - m) ** 2).sum(1, keepdim=True) / width + t["eps"]) ** -0.5
    one = torch.ones(width, dtype=torch.float64, device=DEV)
    g = one if t["g"] is None else t["g"].double()
    b = 0 * one if t["b"] is None else t["b"].double()
    z, out = (x - m) * r, {}
    if c["dir"] != "bwd":
        out = {"y": z * g + b, "mean": m[:, 0], "rstd": r[:, 0]}
    if c["dir"] != "fwd":
        d = t["dy"].double()
        a1, a2 = (d @ g).view(n, 1) / width, ((d * z) @ g).view(n, 1) / width
        out["dx"] = r * (d * g - a1 - z * a2)
        if t["g"] is not None:
            out["dgamma"], out["dbeta"] = (d * z).sum(0), d.sum(0)
    return out


def _exact_keep(count, seed, offset, p):
    """Which elements stay, with the generator's arithmetic in numpy's unsigned 64 bits."""
    lo, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    idx = np.arange(-(-count // 4), dtype=np.uint64)
    x = [idx & lo, idx >> sh, np.full_like(idx, offset % 2 ** 32),
         np.full_like(idx, offset // 2 ** 32 % 2 ** 32)]
    key = [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32]
    for rnd in range(7):
        kk = [np.uint64((key[0] + rnd * 0x9E3779B9) % 2 ** 32),
              np.uint64((key[1] + rnd * 0xBB67AE85) % 2 ** 32)]
        p0, p1 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(p1 >> sh) ^ x[1] ^ kk[0], p1 & lo, (p0 >> sh) ^ x[3] ^ kk[1], p0 & lo]
    u = np.empty((len(idx), 4), np.uint64)
    for j in range(4):
        u[:, j] = x[j]
    return torch.from_numpy(u.reshape(-1)[:count] >= np.uint64(round(p * 2 ** 32))).to(DEV)


def _exact_dropout(t, c):
    keep = _exact_keep(t["x"].numel(), t["seed"], t["offset"], c["p"]).view(t["x"].shape)
    out, s = {}, 1.0 / (1.0 - c["p"])
    if c["dir"] != "bwd":
        out["y"] = t["x"].double() * keep * s
        if t["res"] is not None:
            out["y"] = out["y"] + t["res"].double()
    if c["dir"] != "fwd":
        out["dx"] = t["dy"].double() * keep * s
    return out


def _exact_route(t, c):
    x = t["logits"].double()
    n, E = x.shape
    k, none = c["k"], -math.inf
    # one expert at a time: the largest left, of equal ones the first
    left, taken = x.clone(), torch.zeros_like(x, dtype=torch.bool)
    cols = torch.arange(E, device=DEV).expand(n, E)
    experts = torch.full((n, k), -1, dtype=torch.int64, device=DEV)
    for j in range(k):
        best = left.max(1, keepdim=True).values
        first = torch.where(left == best, cols, E).min(1, keepdim=True).values
        hit = (cols == first) & (best > none)
        experts[:, j] = torch.where(best[:, 0] > none, first[:, 0], -1)
        taken |= hit
        left = left.masked_fill(hit, none)
    top = x.max(1, keepdim=True).values
    p = torch.exp(x - torch.where(top > none, top, 0.0))
    p = p * taken if c["normalize"] else p
    s = p.sum(1, keepdim=True)
    p = p / torch.where(s > 0, s, 1.0)
    w = torch.where(experts >= 0, p.gather(1, experts.clamp(min=0)), 0.0)
    out = {}
    if c["dir"] != "bwd":
        flat = experts.reshape(-1).cpu().numpy()
        pos, rows, offsets, at = np.full(n * k, -1), np.full(n * k, -1), [0], 0
        for e in range(E):
            got = np.nonzero(flat == e)[0]
            pos[got] = at + np.arange(len(got))
            rows[at:at + len(got)] = got // k
            at += len(got)
            offsets.append(at)
        out = {"experts": experts, "weights": w, "offsets": torch.tensor(offsets, device=DEV),
               "rows": torch.from_numpy(rows).to(DEV),
               "pos": torch.from_numpy(pos.reshape(n, k)).to(DEV)}
    if c["dir"] != "fwd":
        # per expert, the gradient that reaches its weight
        dw = torch.zeros_like(x)
        for j in range(k):
            dw += torch.where(cols == experts[:, j:j + 1], t["dw"][:, j:j + 1].double(), 0.0)
        out["dlogits"] = p * (dw - (p * dw).sum(1, keepdim=True))
    return out


def _exact_grouped(t, c):
    off, E = t["offsets"].cpu().tolist(), c["experts"]
    out = {}
    if c["dir"] != "bwd":
        out["y"] = torch.zeros((off[-1], c["c_out"]), dtype=torch.float64, device=DEV)
    if c["dir"] != "fwd":
        out["dx"] = torch.zeros((off[-1], c["c"]), dtype=torch.float64, device=DEV)
        out["dw"] = torch.zeros((E, c["c"], c["c_out"]), dtype=torch.float64, device=DEV)
        out["db"] = torch.zeros((E, c["c_out"]), dtype=torch.float64, device=DEV)
    for e in range(E):
        for a in range(off[e], off[e + 1], 1 << 16):
            s = slice(a, min(a + (1 << 16), off[e + 1]))
            x = (t["x"][s] if t["rows"] is None else t["x"][t["rows"][s].long()]).double()
            w = t["w"][e].double()
            if c["dir"] != "bwd":
                z = x @ w + t["bias"][e].double()
                out["y"][s] = z.clamp(min=0) if c["relu"] else z
            if c["dir"] != "fwd":
                d = t["dy"][s].double()
                g = d @ w.t().contiguous()
                out["dx"][s] = g if t["mask"] is None else g * (t["mask"][s] > 0)
                out["dw"][e] += x.t().contiguous() @ d
                out["db"][e] += d.sum(0)
    return out


def _exact_combine(t, c):
    n, k, out = c["n"], c["k"], {}
    pos, w = t["pos"].long().reshape(-1), t["w"].double().reshape(-1, 1)
    owner = torch.arange(n, device=DEV).repeat_interleave(k)
    if c["dir"] != "bwd":
        s = torch.zeros((n, c["c"]), dtype=torch.float64, device=DEV)
        if t["res"] is not None:
            s += t["res"].double()
        s.index_add_(0, owner, t["y"][pos].double() * w)
        out["out"] = s
    if c["dir"] != "fwd":
        d = t["dout"].double()[owner]
        dy = torch.zeros(t["y"].shape, dtype=torch.float64, device=DEV)
        out["dy"] = dy.index_copy_(0, pos, d * w)
        out["dw"] = (d * t["y"][pos].double()).sum(1).reshape(n, k)
    return out


EXACT = dict(norm=_exact_norm, dropout=_exact_dropout, route=_exact_route, grouped=_exact_grouped,
             combine=_exact_combine)


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed), case)


# ---------------------------------------------------------------------------
# Work
# ---------------------------------------------------------------------------
def work(case):
    """Inputs read once, outputs written once; a pass of both directions counts what they share
    once.  A gathered row counts once, weights as often as an expert has rows."""
    e, n, c, k, E = (2 if case["dtype"] == "bf16" else 4), case["n"], case["c"], case["k"], \
        case["experts"]
    fwd, bwd, op = case["dir"] != "bwd", case["dir"] != "fwd", case["op"]
    m = n * k
    if op == "norm":
        return {"bytes": e * n * c * (1 + fwd + 2 * bwd) + 8 * n + 8 * c * (1 + bwd),
                "flops": n * c * (8 * fwd + 11 * bwd)}
    if op == "dropout":
        return {"bytes": e * n * c * ((2 + case["residual"]) * fwd + 2 * bwd),
                "flops": n * c * 2 * (fwd + bwd)}
    if op == "route":
        read = fwd or not case["normalize"]
        return {"bytes": e * n * E * (read + bwd) + 16 * m * fwd + 4 * m * bwd +
                8 * m * (not fwd) + 4 * E * fwd, "flops": n * E * (2 * fwd + 3 * bwd)}
    if op == "grouped":
        co = case["c_out"]
        x, w = e * c * (n if case["gather"] else m), e * min(E, m) * c * co
        idx = 4 * m * case["gather"] + 4 * E
        by = x + w + idx + fwd * (e * m * co + 4 * min(E, m) * co)
        if bwd:
            by += e * m * (co + c * (1 + case["relu"])) + 4 * E * (c * co + co)
        return {"bytes": by, "flops": 2 * m * c * co * (fwd + 2 * bwd)}
    return {"bytes": e * c * (m + fwd * n * (1 + case["residual"]) + bwd * (n + m)) +
            m * (8 + 4 * bwd), "flops": m * c * (2 * fwd + 3 * bwd)}
