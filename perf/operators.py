"""The dense layers beside the embedding rows, as cases that can be timed: their plain forms and the library's calls.

A model that reads embedding rows from the cache normalises them, takes them through linear layers, and hands the
gradient of the rows back to the cache's update; between the two passes it keeps activations, in 8 bits where memory
is short.  A case is one such call (or the calls of one layer's backward pass) at one size.

Fields of a case:
  kind      "norm" / "norm_back":      layer norm's forward / backward pass
            "linear" / "linear_back":  y = act(x w^T + bias) + residual, and the gradients of z, x, w and bias
            "pack" / "expand":         activations to 8 bits, and back (through an activation)
  rows      rows of the activations;  dim: their width (linear: the layer's input);  out: the linear layer's output, else 0
  x, y      types of input and output ("f32", "bf16", "f16").  Linear layers: x is the type of x, w, z and dz, y that of the
            output, the residual and dy (the residual stream may stay in f32)
  act       "none", "relu", "gelu" (with erf) or "silu"
  residual  norm_back: a gradient that goes round the norm is added to dx;  linear: a residual is added to y
  keep      what lies between the passes in 8 bits: norm: the normalised rows are packed too / read instead of x;
            linear: the pre-activations z;  linear_back: z, and the layer's input
  x_act     linear_back with keep: the layer's input is this activation of what was kept
  strided   rows lie in a wider matrix

8 bits: blocks of 32 along a row share a step 2^e, the smallest for which the block's largest magnitude rounds to at
most 127 steps; a value is a whole number of steps (ties to even).  q: int8 [rows, pitch], e: uint8 [rows, pitch / 32]
(e + 127), pitch: the width rounded up to 32, with zeros behind the row.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BLOCK = 32
MOST_FLOPS = 4 * 8192 * 4096 * 4096          # the largest listed case
MOST_VALUES = 8192 * 8192


def case(kind, rows, dim, out=0, *, name=None, x="bf16", y="bf16", act="none", residual=False, keep=False, x_act="none", strided=False):
    c = dict(kind=kind, rows=rows, dim=dim, out=out, x=x, y=y, act=act, residual=residual, keep=keep, x_act=x_act, strided=strided)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # eight candidates of 26 fields of 64 floats scored for one request: one wave of work, latency only
        case("norm", 8, 1664, name="norm_request", x="f32", y="bf16"),
        # every looked-up row of the benchmark's batch normalised by itself, kept for the backward pass
        case("norm", 106_496, 64, name="norm_rows", x="f32", y="bf16", keep=True),
        # backward into the rows' gradient: the batch's samples of 26 x 64 floats, the residual stream in f32
        case("norm_back", 4_096, 1_664, name="norm_back_samples", x="f32", y="bf16", residual=True, keep=True),
        # a small model with rows of 10 floats: an odd number of samples, nothing kept in 8 bits
        case("norm_back", 333, 260, name="norm_back_odd", x="f32", y="f32"),
        # first layer of a request: bound by reading the weights
        case("linear", 8, 1_664, 1_024, name="linear_request", act="relu"),
        # first layer of a training batch, pre-activations kept in 8 bits
        case("linear", 4_096, 1_664, 4_096, name="linear_up", act="gelu", keep=True),
        # a wide layer back into a residual stream in f32
        case("linear", 8_192, 4_096, 4_096, name="linear_wide", y="f32", residual=True),
        # a small model all in f32, of sizes that are no multiple of anything
        case("linear", 333, 260, 101, name="linear_odd", x="f32", y="f32", act="silu"),
        # both products and the bias' gradient of a wide layer, from what was kept in 8 bits
        case("linear_back", 8_192, 4_096, 4_096, name="linear_back_wide", act="gelu", keep=True),
        # a narrow layer in f16 of an odd number of samples, from whole activations
        case("linear_back", 1_001, 500, 250, name="linear_back_odd", x="f16", y="f16", act="relu"),
        # checkpoint of a large activation
        case("pack", 8_192, 8_192, name="pack_large"),
        # and the small, odd one of a second layer's input: the activation is computed again from what was kept
        case("expand", 2_047, 1_001, name="expand_odd", x="f32", y="f32", act="gelu"),
    ]


def draw(rng):
    def between(lo, hi):                                   # whole, even over the logarithm
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def width(most):
        return rng.choice((between(1, most), 8 * between(1, most // 8), 64 * between(1, most // 64)))

    kind = rng.choice(("norm", "norm_back", "linear", "linear", "linear_back", "linear_back", "pack", "expand"))
    strided = rng.random() < 0.2
    if kind in ("norm", "norm_back"):
        x, y = rng.choice((("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")))
        dim = width(8_192)
        # where a few values are normalised, their gradient is a difference that nearly vanishes: a relative error of it says nothing
        dim = max(8, dim)
        return case(kind, min(between(1, 131_072), MOST_VALUES // dim), dim, x=x, y=y, keep=rng.random() < 0.5,
                    residual=kind == "norm_back" and rng.random() < 0.5, strided=strided)
    if kind in ("pack", "expand"):
        dim = width(8_192)
        t = rng.choice(("f32", "bf16", "f16"))
        return case(kind, min(between(1, 131_072), MOST_VALUES // dim), dim, x=t, y=t,
                    act=rng.choice(("none", "relu", "gelu", "silu")) if kind == "expand" else "none", strided=strided)
    x = rng.choice(("f32", "bf16", "bf16", "f16"))
    y = "f32" if rng.random() < 0.25 else x
    dim, out = max(4, width(6_144)), max(4, width(6_144))
    flops = (4 if kind == "linear_back" else 2) * dim * out * (8 if x == "f32" else 1)
    rows = max(1, min(rng.choice((between(1, 64), between(1, 32_768))), MOST_FLOPS // flops, MOST_VALUES // max(dim, out)))
    act = rng.choice(("none", "relu", "gelu", "silu"))
    keep = rng.random() < 0.5
    return case(kind, rows, dim, out, x=x, y=y, act=act, keep=keep, residual=kind == "linear" and rng.random() < 0.4,
                x_act=rng.choice(("none", "none", "relu", "gelu")) if keep and kind == "linear_back" else "none", strided=strided)


# ---- inputs -----------------------------------------------------------------------------------------
def pitch(dim):
    return -(-dim // BLOCK) * BLOCK


def rows_of(c, gen, rows, dim, kind, scale=1.0, at=0.0):
    """Activations as a layer sees them: rows of uneven size around `at`, some columns larger than others; a wider matrix under it if the case says so."""
    dev = torch.device("cuda")
    wide = dim + (24 if c["strided"] else 0)
    v = at + torch.randn(rows, wide, generator=gen, device=dev)
    v *= scale * torch.exp(0.5 * torch.randn(rows, 1, generator=gen, device=dev))
    v *= torch.exp(0.3 * torch.randn(1, wide, generator=gen, device=dev))
    return v.to(TYPES[kind])[:, :dim]


def empty_like_rows(c, rows, dim, kind):
    wide = dim + (24 if c["strided"] else 0)
    return torch.empty(rows, wide, dtype=TYPES[kind], device="cuda")[:, :dim]


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dev = torch.device("cuda")
    kind, rows, dim, out = c["kind"], c["rows"], c["dim"], c["out"]

    def vector(n, at, spread):
        return at + spread * torch.randn(n, generator=gen, device=dev)

    def packed(v):
        return pack_plain(v.float())

    def packed_room(rows, dim):
        return torch.empty(rows, pitch(dim), dtype=torch.int8, device=dev), torch.empty(rows, pitch(dim) // BLOCK, dtype=torch.uint8, device=dev)

    s = {"case": c}
    if kind in ("norm", "norm_back"):
        s["gamma"], s["beta"] = vector(dim, 1.0, 0.2), vector(dim, 0.0, 0.2)
        x = rows_of(c, gen, rows, dim, c["x"], 0.05 if c["x"] == "f32" else 1.0, at=0.5)
        if kind == "norm":
            s.update(x=x, to_y=empty_like_rows(c, rows, dim, c["y"]), to_mean=torch.empty(rows, device=dev), to_rstd=torch.empty(rows, device=dev))
            if c["keep"]:
                s["to_packed"] = packed_room(rows, dim)
                s["to_values"] = torch.empty(rows, dim, dtype=TYPES[c["y"]], device=dev)
        else:
            mean = x.double().mean(1)
            rstd = (x.double().var(1, unbiased=False) + EPS).rsqrt()
            s.update(dy=rows_of(c, gen, rows, dim, c["y"]), rstd=rstd.float(), to_dx=empty_like_rows(c, rows, dim, c["x"]),
                     to_dgamma=torch.empty(dim, device=dev), to_dbeta=torch.empty(dim, device=dev))
            if c["keep"]:
                s["packed"] = packed((x.double() - mean[:, None]) * rstd[:, None])
            else:
                s.update(x=x, mean=mean.float())
            if c["residual"]:
                s["residual"] = rows_of(c, gen, rows, dim, c["x"])
    elif kind == "linear":
        s.update(x=rows_of(c, gen, rows, dim, c["x"]), w=(torch.randn(out, dim, generator=gen, device=dev) / math.sqrt(dim)).to(TYPES[c["x"]]),
                 bias=vector(out, 0.0, 0.3), to_y=empty_like_rows(c, rows, out, c["y"]))
        if c["residual"]:
            s["residual"] = rows_of(c, gen, rows, out, c["y"])
        if c["keep"]:
            s["to_packed"] = packed_room(rows, out)
            s["to_values"] = torch.empty(rows, out, dtype=TYPES[c["x"]], device=dev)
    elif kind == "linear_back":
        t = TYPES[c["x"]]
        x, z = rows_of(c, gen, rows, dim, c["x"]), rows_of(c, gen, rows, out, c["x"])
        s.update(dy=rows_of(c, gen, rows, out, c["y"]), w=(torch.randn(out, dim, generator=gen, device=dev) / math.sqrt(dim)).to(t),
                 to_dz=torch.empty(rows, out, dtype=t, device=dev), to_dx=empty_like_rows(c, rows, dim, c["x"]),
                 to_dw=torch.empty(out, dim, dtype=t, device=dev), to_dbias=torch.empty(out, device=dev))
        s["x"] = packed(x) if c["keep"] else x
        s["z"] = None if c["act"] == "none" else packed(z) if c["keep"] else z
    elif kind == "pack":
        s.update(x=rows_of(c, gen, rows, dim, c["x"]), to_packed=packed_room(rows, dim))
    else:
        s.update(packed=packed(rows_of(c, gen, rows, dim, c["x"])), to_y=empty_like_rows(c, rows, dim, c["y"]))
    return s


# ---- the plain forms --------------------------------------------------------------------------------
def pack_plain(v):
    """q and e of the values, as the module's text says."""
    rows, dim = v.shape
    b = torch.nn.functional.pad(v, (0, pitch(dim) - dim)).reshape(rows, -1, BLOCK)
    most = b.abs().amax(2)
    m, k = torch.frexp(most)                               # most = m 2^k with m in [1/2, 1)
    e = (k - 7 + (torch.round(m * 128) > 127)).clamp(-126, 122)
    e = torch.where(most > 0, e, torch.full_like(e, -126))
    q = torch.round(torch.ldexp(b, -e[:, :, None]))
    q = torch.minimum(q.abs(), torch.where(e == 122, 63.0, 127.0)[:, :, None].to(q.dtype)) * torch.sign(q)
    return q.to(torch.int8).reshape(rows, -1), (e + 127).to(torch.uint8)


def values_plain(packed, dim, dtype=torch.float32):
    q, e = packed
    rows = q.shape[0]
    step = torch.ldexp(torch.ones((), dtype=dtype, device=q.device), e.to(torch.int32) - 127)
    return (q.to(dtype).reshape(rows, -1, BLOCK) * step[:, :, None]).reshape(rows, -1)[:, :dim]


def act_plain(act, v):
    if act == "relu":
        return torch.clamp(v, min=0)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v


def slope_plain(act, v):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = 1 / (1 + torch.exp(-v))
        return p * (1 + v * (1 - p))
    return torch.ones_like(v)


def run_plain(s):
    c = s["case"]
    kind, dim, tx, ty = c["kind"], c["dim"], TYPES[c["x"]], TYPES[c["y"]]
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        n = d * rstd
        got = {"y": (n * s["gamma"] + s["beta"]).to(ty), "mean": mean[:, 0], "rstd": rstd[:, 0]}
        if c["keep"]:
            got["kept"] = values_plain(pack_plain(n), dim).to(ty)
        return got
    if kind == "norm_back":
        n = values_plain(s["packed"], dim) if c["keep"] else (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
        if c["residual"]:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(tx), "dgamma": (dy * n).sum(0), "dbeta": dy.sum(0)}
    if kind == "linear":
        z = s["x"].float() @ s["w"].float().t() + s["bias"]
        y = act_plain(c["act"], z)
        if c["residual"]:
            y = y + s["residual"].float()
        got = {"y": y.to(ty)}
        if c["keep"]:
            got["kept"] = values_plain(pack_plain(z), c["out"]).to(tx)
        return got
    if kind == "linear_back":
        # dz is an output of its own, in the layer's type: the products are of what is handed out
        dz = s["dy"].float()
        if c["act"] != "none":
            z = values_plain(s["z"], c["out"]) if c["keep"] else s["z"].float()
            dz = dz * slope_plain(c["act"], z)
        x = act_plain(c["x_act"], values_plain(s["x"], dim)).to(tx) if c["keep"] else s["x"]
        t = dz.to(tx)
        return {"dz": t, "dx": (t.float() @ s["w"].float()).to(tx), "dw": (t.float().t() @ x.float()).to(tx), "dbias": dz.sum(0)}
    if kind == "pack":
        q, e = pack_plain(s["x"].float())
        return {"q": q, "e": e}
    return {"y": act_plain(c["act"], values_plain(s["packed"], dim)).to(ty)}


# ---- the library's calls ----------------------------------------------------------------------------
def run_own(s):
    from paper_2112_07221_amd import dense
    c = s["case"]
    kind, dim = c["kind"], c["dim"]
    act = getattr(dense, "ACT_" + c["act"].upper())
    if kind == "norm":
        kept = dense.Packed(*s["to_packed"], dim) if c["keep"] else None
        dense.layer_norm(s["x"], s["gamma"], s["beta"], s["to_y"], s["to_mean"], s["to_rstd"], packed=kept, eps=EPS)
        got = {"y": s["to_y"], "mean": s["to_mean"], "rstd": s["to_rstd"]}
        if c["keep"]:
            dense.expand(kept, s["to_values"])
            got["kept"] = s["to_values"]
        return got
    if kind == "norm_back":
        x = dense.Packed(*s["packed"], dim) if c["keep"] else s["x"]
        dense.layer_norm_backward(s["dy"], x, s["gamma"], s.get("mean"), s["rstd"], s["to_dx"], s["to_dgamma"], s["to_dbeta"], residual=s.get("residual"))
        return {"dx": s["to_dx"], "dgamma": s["to_dgamma"], "dbeta": s["to_dbeta"]}
    if kind == "linear":
        kept = dense.Packed(*s["to_packed"], c["out"]) if c["keep"] else None
        dense.linear(s["x"], s["w"], s["bias"], s["to_y"], act=act, residual=s.get("residual"), z=kept)
        got = {"y": s["to_y"]}
        if c["keep"]:
            dense.expand(kept, s["to_values"])
            got["kept"] = s["to_values"]
        return got
    if kind == "linear_back":
        x, z = s["x"], s["z"]
        if c["keep"]:
            x = dense.Packed(*x, dim)
            z = None if z is None else dense.Packed(*z, c["out"])
        dense.linear_backward(s["dy"], x, s["w"], z, act, s["to_dz"], s["to_dx"], s["to_dw"], s["to_dbias"], x_act=getattr(dense, "ACT_" + c["x_act"].upper()))
        return {"dz": s["to_dz"], "dx": s["to_dx"], "dw": s["to_dw"], "dbias": s["to_dbias"]}
    if kind == "pack":
        dense.pack(s["x"], dense.Packed(*s["to_packed"], dim))
        return {"q": s["to_packed"][0], "e": s["to_packed"][1]}
    dense.expand(dense.Packed(*s["packed"], dim), s["to_y"], act=act)
    return {"y": s["to_y"]}


def run(state):
    return run_own(state) if own else run_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    c = case
    rows, dim, out, x, y = c["rows"], c["dim"], c["out"], SIZE[c["x"]], SIZE[c["y"]]

    def kept(width):
        return rows * pitch(width) * (1 + 1 / BLOCK)

    n = rows * dim
    if c["kind"] == "norm":
        return {"bytes": n * (x + y) + 8 * (rows + dim) + (kept(dim) if c["keep"] else 0), "flops": 8 * n}
    if c["kind"] == "norm_back":
        return {"bytes": n * (y + x + (x if c["residual"] else 0)) + (kept(dim) + 4 * rows if c["keep"] else n * x + 8 * rows) + 12 * dim, "flops": 14 * n}
    if c["kind"] == "linear":
        return {"bytes": n * x + out * dim * x + 4 * out + rows * out * y * (2 if c["residual"] else 1) + (kept(out) if c["keep"] else 0), "flops": 2 * n * out}
    if c["kind"] == "linear_back":
        z = 0 if c["act"] == "none" else kept(out) if c["keep"] else rows * out * x
        return {"bytes": rows * out * (y + x) + z + (kept(dim) if c["keep"] else n * x) + n * x + 2 * out * dim * x + 4 * out, "flops": 4 * n * out}
    if c["kind"] == "pack":
        return {"bytes": n * x + kept(dim), "flops": 4 * n}
    return {"bytes": kept(dim) + n * y, "flops": 4 * n}


# ---- in 64 bits, from the definitions ---------------------------------------------------------------
def exact(case, seed):
    """A value that is computed and then rounded to 8 bits has no such value: it lies a whole step further where it lies next to a tie."""
    s = prepare(case, seed)
    c = s["case"]
    kind, rows, dim, out = c["kind"], c["rows"], c["dim"], c["out"]

    def unpacked(p, n):                                    # q 2^(e - 127)
        q, e = p
        return (q.double() * torch.exp2(e.double() - 127).repeat_interleave(BLOCK, 1))[:, :n]

    def phi(v):                                            # the normal distribution's function
        return torch.special.ndtr(v)

    def value(act, v):
        return {"none": lambda: v, "relu": lambda: torch.where(v > 0, v, torch.zeros_like(v)), "gelu": lambda: v * phi(v), "silu": lambda: v * torch.sigmoid(v)}[act]()

    def slope(act, v):
        return {"none": lambda: torch.ones_like(v), "relu": lambda: torch.where(v > 0, 1.0, 0.0).double(),
                "gelu": lambda: phi(v) + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi),
                "silu": lambda: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v)}[act]()

    if kind == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        got = {"y": s["gamma"].double() * ((x - mean.unsqueeze(1)) * rstd.unsqueeze(1)) + s["beta"].double(), "mean": mean, "rstd": rstd}
        if c["keep"]:
            got["kept"] = None
        return got
    if kind == "norm_back":
        rstd = s["rstd"].double().unsqueeze(1)
        n = unpacked(s["packed"], dim) if c["keep"] else (s["x"].double() - s["mean"].double().unsqueeze(1)) * rstd
        dy = s["dy"].double()
        h = dy * s["gamma"].double()
        dx = (h - (h.sum(1, keepdim=True) + n * (h * n).sum(1, keepdim=True)) / dim) * rstd
        if c["residual"]:
            dx += s["residual"].double()
        return {"dx": dx, "dgamma": (dy * n).sum(0), "dbeta": dy.sum(0)}
    if kind == "linear":
        y = value(c["act"], torch.addmm(s["bias"].double(), s["x"].double(), s["w"].double().t()))
        got = {"y": y + s["residual"].double() if c["residual"] else y}
        if c["keep"]:
            got["kept"] = None
        return got
    if kind == "linear_back":
        dz = s["dy"].double()
        if c["act"] != "none":
            dz = dz * slope(c["act"], unpacked(s["z"], out) if c["keep"] else s["z"].double())
        x = value(c["x_act"], unpacked(s["x"], dim)) if c["keep"] else s["x"].double()
        handed, taken = dz.to(TYPES[c["x"]]).double(), x.to(TYPES[c["x"]]).double()   # both in the layer's type, as the definition has it
        return {"dz": dz, "dx": torch.mm(handed, s["w"].double()), "dw": torch.mm(handed.t(), taken), "dbias": dz.sum(0)}
    if kind == "pack":
        return None
    return {"y": value(c["act"], unpacked(s["packed"], dim))}
