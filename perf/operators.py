"""The operators around the token mixer, as measurable cases: each once in elementary torch operations and once as the
package's own calls.

One layer runs them in a row: a norm in front of the projections, rotary positions on the queries and keys, the mixer,
the normalised and gated read-out, the output projection, and the join with the residual stream (with the next block's norm).

* ``rotary``, ``rotary_back``  pairs of every q and k head turned by position * frequency, and the gradient (turned back);
* ``gate``, ``gate_back``      y = x / rms(x) * w * act(g) over every head of the mixer's output, and its gradients;
* ``join``, ``join_back``      x' = x + scale * c * u with u = h or h / rms(h) * w_after, y = x' / rms(x') * w_before, and
  the gradients (from x', which a training step keeps).

``own`` chooses: False computes the plain forms (32-bit arithmetic, angles and long sums in 64 bits, one rounding at the
end), True calls the package.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-5


def _case(name, kind, dtype, **more):
    c = dict(name=name, kind=kind, dtype=dtype, mix=0)
    if kind.startswith("rotary"):
        c.update(B=1, T=1, Hq=16, Hk=16, d=128, rotary=128, pairs="halves", scaling="none", factor=1.0, place="zero",
                 layout="bthd")
    elif kind.startswith("gate"):
        c.update(B=1, T=1, H=16, dv=128, act="silu", weight="shared", layout="bthd")
    else:
        c.update(B=1, T=1, D=1024, x_dtype=dtype, after=False, channel=False, scale=1.0, later=True)
    c.update(more)
    return c


def listed():
    return [
        # One user generating text far into a long context: q and k of a single token.
        _case("rotary_token", "rotary", "bf16", place="start"),
        # A training batch at 2K context, 16 heads of width 128.
        _case("rotary_train", "rotary", "bf16", B=8, T=2048),
        # A document of 64K tokens with 32 heads, frequencies blended for eight times the trained length.
        _case("rotary_long", "rotary", "bf16", T=65536, Hq=32, Hk=32, scaling="blend", factor=8.0),
        # Gradients on packed documents in fp32: adjacent pairs, three quarters of a head turned, fewer key heads.
        _case("rotary_back_packed_f32", "rotary_back", "f32", T=4999, Hq=16, Hk=4, d=64, rotary=48, pairs="adjacent", mix=7),
        # The read-out of one token for each sequence of a serving batch.
        _case("gate_token", "gate", "bf16", B=64),
        # The read-out of a prompt batch as the mixer leaves it in the head-major layout.
        _case("gate_prefill", "gate", "bf16", B=8, T=2048, layout="bhtd"),
        # Gradients in a training step at 4K context with 16 heads of width 128.
        _case("gate_back_train", "gate_back", "bf16", B=8, T=4096),
        # Gradients in fp32 on packed documents: sigmoid gate, a weight for every head, the 4-head model shape (256 wide).
        _case("gate_back_packed_f32", "gate_back", "f32", T=2043, H=4, dv=256, act="sigmoid", weight="heads", mix=3),
        # Joining one token's block output and normalising for the next block.
        _case("join_token", "join", "bf16", D=1024),
        # The same over a training batch at 4K context of the 1024-wide model, with a norm behind the block too.
        _case("join_train", "join", "bf16", B=8, T=4096, D=1024, after=True),
        # Gradients of a 2048-wide layer whose residual stream is fp32: both norms and a scale per channel.
        _case("join_back_train", "join_back", "bf16", B=8, T=2048, D=2048, x_dtype="f32", after=True, channel=True, scale=0.5),
        # Gradients in fp32 on a ragged length and an odd width, the last block of a network: nothing flows in from later.
        _case("join_back_ragged_f32", "join_back", "f32", B=2, T=1021, D=1096, channel=True, later=False),
    ]


# The most bytes a drawn case of each operator moves: what the largest listed one does.
MOST_BYTES = {"rotary": 2.1e9, "gate": 6.7e8, "join": 6.0e8}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    kind = rng.choice(["rotary", "rotary", "rotary_back", "gate", "gate_back", "gate_back", "join", "join_back", "join_back"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    shape = rng.random()
    if shape < 0.25:  # one token for each sequence
        B, T, mix = _log_int(rng, 1, 512), 1, 0
    elif shape < 0.45:  # packed documents
        B, T, mix = 1, _log_int(rng, 64, 16384), rng.randrange(1, 1000)
    else:
        B, T, mix = _log_int(rng, 1, 16), _log_int(rng, 2, 16384), 0
    if kind.startswith("rotary"):
        d = rng.choice([32, 64, 64, 128, 128, 128, 256, 8 * rng.randint(1, 40)])
        r = d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2)
        Hq = rng.choice([1, 2, 4, 5, 8, 16, 16, 32])
        scaling = rng.choice(["none", "none", "linear", "base", "blend"])
        c = _case("", kind, dtype, Hq=Hq, Hk=rng.choice([Hq, Hq, 1, 2, 4, 0]), d=d, rotary=r, scaling=scaling,
                  factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 5.5]),
                  pairs=rng.choice(["halves", "adjacent"]), place=rng.choice(["zero", "start", "token"]),
                  layout="bhtd" if not mix and rng.random() < 0.25 else "bthd")
    elif kind.startswith("gate"):
        dv = rng.choice([64, 128, 128, 256, 256, 8 * rng.randint(1, 64)])
        c = _case("", kind, dtype, H=rng.choice([1, 2, 4, 5, 8, 12, 16, 32]), dv=dv, act=rng.choice(["silu", "silu", "sigmoid", "none"]),
                  weight=rng.choice(["shared", "shared", "heads", "none"]),
                  layout="bhtd" if not mix and rng.random() < 0.3 else "bthd")
    else:
        D = rng.choice([512, 768, 1024, 1024, 2048, 2048, 4096, 8192, 8 * rng.randint(1, 2048)])
        c = _case("", kind, dtype, D=D, x_dtype="f32" if rng.random() < 0.3 else dtype, after=rng.random() < 0.5,
                  channel=rng.random() < 0.4, scale=rng.choice([1.0, 1.0, 0.5, 0.22]), later=rng.random() < 0.8)
    c.update(B=B, T=T, mix=mix)
    del c["name"]
    while work(c)["bytes"] > MOST_BYTES[kind.split("_")[0]]:  # too large: fewer sequences, then fewer tokens
        if c["B"] > 1:
            c["B"] = max(1, c["B"] * 2 // 3)
        else:
            c["T"] = max(1, c["T"] * 2 // 3)
    return c


def lengths(case):
    """Document lengths of a packed case: 1 to 4096 tokens, spread over their logarithm, one of them empty."""
    rng = random.Random(case["mix"])
    left, out = case["T"], [0]
    while left > 0:
        n = min(left, _log_int(rng, 1, 4096))
        out.append(n)
        left -= n
    rng.shuffle(out)
    return out


def frequencies(width, base=10000.0, scaling="none", factor=1.0, length=4096):
    """Radians a token for every pair, in 64 bits, and the factor on the turned pairs."""
    i = torch.arange(width // 2, dtype=torch.float64)
    if scaling == "base" and width > 2:
        base = base * factor ** (width / (width - 2))
    f = base ** (-2.0 * i / width)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "blend":  # pairs that turn over 32 times in the trained length stay, those under once are slowed down
        turns = length * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1.0 - keep), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _element(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    el, kind = _element(case["dtype"]), case["kind"]
    B, T = case["B"], case["T"]
    s = {"case": case, "cu": None}
    lead = (B, T)
    if case["mix"]:
        n = lengths(case)
        s["cu"] = torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=dev)
        lead, B = (T,), len(n)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    def heads(H, d, layout=None):
        return (case["B"], H, T, d) if (layout or case["layout"]) == "bhtd" else lead + (H, d)

    if kind.startswith("rotary"):
        f, s["magnitude"] = frequencies(case["rotary"], scaling=case["scaling"], factor=case["factor"])
        s["f"] = f.to(dev)
        s["q"] = normal(*heads(case["Hq"], case["d"])).to(el)
        s["k"] = normal(*heads(case["Hk"], case["d"])).to(el) if case["Hk"] else None
        s["start"] = s["positions"] = None
        if case["place"] == "start":  # sequences that are some way into their context
            s["start"] = torch.randint(0, 131072, (B,), generator=g, device=dev, dtype=torch.int32)
        elif case["place"] == "token":
            s["positions"] = torch.randint(0, 32768, lead, generator=g, device=dev, dtype=torch.int32)
    elif kind.startswith("gate"):
        H, dv = case["H"], case["dv"]
        # the read gate makes some heads of a token loud and most quiet
        x = normal(*heads(H, dv))
        s["x"] = (x * torch.exp(normal(*x.shape[:-1], 1) - 2.0)).to(el)
        s["g"] = None if case["act"] == "none" else (normal(*heads(H, dv, "bthd")) * 1.5).to(el)
        s["w"] = {"none": None, "shared": 1.0 + 0.1 * normal(dv), "heads": 1.0 + 0.1 * normal(H, dv)}[case["weight"]]
        if kind == "gate_back":
            s["dy"] = normal(*heads(H, dv, "bthd")).to(el)
    else:
        D, xel = case["D"], _element(case["x_dtype"])
        loud = 1.0 + 9.0 * (torch.rand(D, generator=g, device=dev) < 0.01).float()  # a few channels carry large values
        s["x"] = (normal(*lead, D) * 2.0 * loud).to(xel)
        s["h"] = (normal(*lead, D) * 0.5).to(el)
        s["w_before"] = 1.0 + 0.1 * normal(D)
        s["w_after"] = 1.0 + 0.1 * normal(D) if case["after"] else None
        s["channel"] = 0.5 + 0.1 * normal(D) if case["channel"] else None
        if kind == "join_back":
            s["dy"] = normal(*lead, D).to(el)
            s["dx_out"] = normal(*lead, D).to(xel) if case["later"] else None
    return s


def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms.

def _angles(s):
    """[tokens..., rotary/2] in 64 bits, laid out to meet [B,T,H,r/2] ([T,H,r/2] packed, [B,H,T,r/2] head-major)."""
    c, cu = s["case"], s["cu"]
    dev = s["f"].device
    if s["positions"] is not None:
        p = s["positions"].double()
    elif cu is not None:
        t = torch.arange(c["T"], dtype=torch.int32, device=dev)
        b = torch.searchsorted(cu, t, right=True) - 1
        p = (t - cu[b]).double()
        if s["start"] is not None:
            p = p + s["start"][b].double()
    else:
        p = torch.arange(c["T"], dtype=torch.float64, device=dev).expand(c["B"], -1)
        if s["start"] is not None:
            p = p + s["start"].double()[:, None]
    a = p[..., None] * s["f"]
    return a.unsqueeze(1 if c["layout"] == "bhtd" else -2)


def _turn(x, cos, sin, r, pairs, el):
    if x is None:
        return None
    y = x.float()
    if pairs == "halves":
        a, b = y[..., : r // 2], y[..., r // 2: r]
        out = torch.cat((a * cos - b * sin, a * sin + b * cos, y[..., r:]), dim=-1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        out = torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2), y[..., r:]), dim=-1)
    return out.to(el)


def _plain_rotary(s, sign=1.0):
    c = s["case"]
    a = _angles(s)
    cos, sin = (a.cos() * s["magnitude"]).float(), (a.sin() * (sign * s["magnitude"])).float()
    el = _element(c["dtype"])
    return {"q": _turn(s["q"], cos, sin, c["rotary"], c["pairs"], el), "k": _turn(s["k"], cos, sin, c["rotary"], c["pairs"], el)}


def _act(name, g):
    """The gate and its derivative."""
    if name == "none":
        return 1.0, None
    p = torch.sigmoid(g)
    if name == "sigmoid":
        return p, p * (1.0 - p)
    return g * p, p * (1.0 + g * (1.0 - p))


def _plain_gate(s):
    c = s["case"]
    x = s["x"].float()
    if c["layout"] == "bhtd":
        x = x.transpose(1, 2)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if s["w"] is not None:
        y = y * s["w"]
    if s["g"] is not None:
        y = y * _act(c["act"], s["g"].float())[0]
    return {"y": y.to(_element(c["dtype"])).contiguous()}


def _plain_gate_back(s):
    c, el = s["case"], _element(s["case"]["dtype"])
    x, dy = s["x"].float(), s["dy"].float()
    if c["layout"] == "bhtd":
        x = x.transpose(1, 2)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    a, da = _act(c["act"], None if s["g"] is None else s["g"].float())
    w = 1.0 if s["w"] is None else s["w"]
    dn = dy * w * a
    dx = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    if c["layout"] == "bhtd":
        dx = dx.transpose(1, 2)
    out = {"dx": dx.to(el).contiguous(), "dg": None if da is None else (dy * n * w * da).to(el), "dw": None}
    if s["w"] is not None:
        p = (dy * n * a).flatten(0, -3 if c["weight"] == "heads" else -2)
        out["dw"] = p.sum(0, dtype=torch.float64).float()
    return out


def _plain_join(s):
    c = s["case"]
    u = s["h"].float()
    if s["w_after"] is not None:
        u = u * torch.rsqrt((u * u).mean(-1, keepdim=True) + EPS) * s["w_after"]
    if s["channel"] is not None:
        u = u * s["channel"]
    x = s["x"].float() + c["scale"] * u
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["w_before"]
    return {"x_out": x.to(_element(c["x_dtype"])), "y": y.to(_element(c["dtype"]))}


def _plain_join_back(s):
    c, el = s["case"], _element(s["case"]["dtype"])
    x, dy = s["x"].float(), s["dy"].float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dn = dy * s["w_before"]
    dx = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    if s["dx_out"] is not None:
        dx = dx + s["dx_out"].float()
    long = lambda t: t.flatten(0, -2).sum(0, dtype=torch.float64).float()
    out = {"dx": dx.to(_element(c["x_dtype"])), "dw_before": long(dy * n), "dw_after": None, "dchannel": None}
    du = c["scale"] * dx
    m = s["h"].float()
    if s["w_after"] is not None:
        rh = torch.rsqrt((m * m).mean(-1, keepdim=True) + EPS)
        m = m * rh
    if s["w_after"] is not None or s["channel"] is not None:
        p = long(du * m)
        if s["w_after"] is not None:
            out["dw_after"] = p if s["channel"] is None else p * s["channel"]
        if s["channel"] is not None:
            out["dchannel"] = p if s["w_after"] is None else p * s["w_after"]
            du = du * s["channel"]
    if s["w_after"] is not None:
        dm = du * s["w_after"]
        du = rh * (dm - m * (dm * m).mean(-1, keepdim=True))
    out["dh"] = du.to(el)
    return out


_plain = {"rotary": _plain_rotary, "rotary_back": lambda s: _plain_rotary(s, -1.0), "gate": _plain_gate,
          "gate_back": _plain_gate_back, "join": _plain_join, "join_back": _plain_join_back}


# ---------------------------------------------------------------------------------------------------------------------
# The package's calls.

def _own_rotary(s):
    import paper_2602_01744_amd as sla

    c = s["case"]
    call = sla.rotary if c["kind"] == "rotary" else sla.rotary_backward
    q, k = call(s["q"], s["k"], s["f"], start=s["start"], positions=s["positions"], cu_seqlens=s["cu"],
                adjacent=c["pairs"] == "adjacent", magnitude=s["magnitude"], head_major=c["layout"] == "bhtd")
    return {"q": q, "k": k}


def _own_gate(s):
    import paper_2602_01744_amd as sla

    c = s["case"]
    return {"y": sla.norm_gate(s["x"], s["g"], s["w"], gate=c["act"], eps=EPS, cu_seqlens=s["cu"],
                               head_major=c["layout"] == "bhtd")}


def _own_gate_back(s):
    import paper_2602_01744_amd as sla

    c = s["case"]
    return sla.norm_gate_backward(s["x"], s["g"], s["w"], s["dy"], gate=c["act"], eps=EPS, cu_seqlens=s["cu"],
                                  head_major=c["layout"] == "bhtd")


def _own_join(s):
    import paper_2602_01744_amd as sla

    x, y = sla.join_norm(s["x"], s["h"], s["w_before"], w_after=s["w_after"], channel_scale=s["channel"],
                         scale=s["case"]["scale"], eps=EPS, cu_seqlens=s["cu"])
    return {"x_out": x, "y": y}


def _own_join_back(s):
    import paper_2602_01744_amd as sla

    g = sla.join_norm_backward(s["x"], s["h"], s["w_before"], s["dy"], s["dx_out"], w_after=s["w_after"],
                               channel_scale=s["channel"], scale=s["case"]["scale"], eps=EPS, cu_seqlens=s["cu"])
    return {"dx": g["dx"], "dw_before": g["dw_before"], "dw_after": g["dw_after"], "dchannel": g["dchannel_scale"], "dh": g["dh"]}


_own = {"rotary": _own_rotary, "rotary_back": _own_rotary, "gate": _own_gate, "gate_back": _own_gate_back,
        "join": _own_join, "join_back": _own_join_back}


# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    """Every tensor read or written once; weights and angles once."""
    es = 2 if case["dtype"] == "bf16" else 4
    n, kind = case["B"] * case["T"], case["kind"]
    if kind.startswith("rotary"):
        e = n * (case["Hq"] + case["Hk"]) * case["d"]
        turned = n * (case["Hq"] + case["Hk"]) * case["rotary"]
        return {"bytes": 2 * e * es + 4 * case["rotary"] + (4 * n if case["place"] == "token" else 0), "flops": 3 * turned}
    if kind.startswith("gate"):
        e = n * case["H"] * case["dv"]
        w = {"none": 0, "shared": 1, "heads": case["H"]}[case["weight"]] * case["dv"] * 4
        gated = case["act"] != "none"
        if kind == "gate":
            return {"bytes": (3 if gated else 2) * e * es + w, "flops": (9 if gated else 4) * e}
        return {"bytes": (5 if gated else 3) * e * es + 2 * w, "flops": (20 if gated else 10) * e}
    e, xs = n * case["D"], 2 if case["x_dtype"] == "bf16" else 4
    w = 4 * case["D"] * (1 + case["after"] + case["channel"])
    if kind == "join":
        return {"bytes": e * 2 * (xs + es) + w, "flops": e * (7 + 4 * case["after"] + case["channel"])}
    reads_h = case["after"] or case["channel"]
    tensors = e * (2 * xs + 2 * es) + (e * xs if case["later"] else 0) + (e * es if reads_h else 0)
    return {"bytes": tensors + 2 * w, "flops": e * (12 + 10 * case["after"] + 3 * case["channel"])}


def exact(case, seed):
    """From the definitions in 64 bits: turned pairs as products of complex numbers, gradients by differentiating the
    definition itself."""
    s = prepare(case, seed)
    kind = case["kind"]
    wide = lambda t: None if t is None else t.double()
    if kind.startswith("rotary"):
        unit = _exact_unit(s, case)
        r = case["rotary"]

        def turn(x):
            if x is None:
                return None
            y = x.double()
            if case["pairs"] == "halves":
                z = torch.complex(y[..., : r // 2], y[..., r // 2: r]) * unit
                y[..., : r // 2], y[..., r // 2: r] = z.real, z.imag
            else:
                z = torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * unit
                y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
            return y

        return {"q": turn(s["q"]), "k": turn(s["k"])}
    back = kind.endswith("_back")
    names = ("x", "g", "w") if kind.startswith("gate") else ("x", "h", "w_before", "w_after", "channel")
    v = {n: wide(s[n]) for n in names}
    if kind == "join_back":  # x is x' there: what the join adds is taken off first, so that the forward gives it back
        with torch.no_grad():
            v["x"] = v["x"] - _exact_update(v, case)
    if back:
        for t in v.values():
            if t is not None:
                t.requires_grad_(True)
    with torch.set_grad_enabled(back):
        if kind.startswith("gate"):
            x = v["x"].transpose(1, 2) if case["layout"] == "bhtd" else v["x"]
            y = x / ((x ** 2).sum(-1, keepdim=True) / case["dv"] + EPS) ** 0.5
            if v["w"] is not None:
                y = torch.einsum("...hd,hd->...hd" if case["weight"] == "heads" else "...hd,d->...hd", y, v["w"])
            if v["g"] is not None:
                y = y * (torch.nn.functional.silu(v["g"]) if case["act"] == "silu" else torch.special.expit(v["g"]))
            if not back:
                return {"y": y}
            y.backward(wide(s["dy"]))
            grad = lambda n: None if v[n] is None else v[n].grad
            return {"dx": grad("x"), "dg": grad("g"), "dw": grad("w")}
        x = v["x"] + _exact_update(v, case)
        y = x / ((x ** 2).sum(-1, keepdim=True) / case["D"] + EPS) ** 0.5 * v["w_before"]
        if not back:
            return {"x_out": x, "y": y}
        if s["dx_out"] is None:
            y.backward(wide(s["dy"]))
        else:
            torch.autograd.backward((y, x), (wide(s["dy"]), wide(s["dx_out"])))
    grad = lambda n: None if v[n] is None else v[n].grad
    return {"dx": grad("x"), "dw_before": grad("w_before"), "dw_after": grad("w_after"), "dchannel": grad("channel"), "dh": grad("h")}


def _exact_unit(s, case):
    """magnitude * e^(i angle) for every token and pair, sequence by sequence."""
    B, T, f = case["B"], case["T"], s["f"]
    counts = lengths(case) if case["mix"] else [T] * B
    first = [0] * len(counts) if s["start"] is None else s["start"].tolist()
    place = torch.cat([torch.arange(p, p + n, dtype=torch.float64) for p, n in zip(first, counts)]).to(f.device)
    if s["positions"] is not None:
        place = s["positions"].double().reshape(-1)
    unit = torch.exp(torch.complex(torch.zeros((), dtype=torch.float64, device=f.device), torch.outer(place, f)))
    unit = s["magnitude"] * (unit if case["kind"] == "rotary" else unit.conj())
    if case["mix"]:
        return unit.view(T, 1, -1)
    return unit.view(B, 1, T, -1) if case["layout"] == "bhtd" else unit.view(B, T, 1, -1)


def _exact_update(v, case):
    u = v["h"]
    if v["w_after"] is not None:
        u = u / ((u ** 2).sum(-1, keepdim=True) / case["D"] + EPS) ** 0.5 * v["w_after"]
    if v["channel"] is not None:
        u = u * v["channel"]
    return case["scale"] * u
