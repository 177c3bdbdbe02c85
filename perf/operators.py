"""The block operations of several requests at once, as cases that can be timed and compared.

A server of a video diffusion model packs the tokens of several requests (users, or the conditional and the
unconditional pass of one) one after the other and runs every block over all of them.  What differs from request to request is
small: the scale, shift and gate that its timestep gives, a low-rank adapter beside each projection, the patch grid that its
tokens are rotated by.  The cases are the block's calls on such a batch:

  linear    y = x W^T + b + s_r (x D_r^T) U_r^T                       lp_linear_adapters
  qkv       the same in three sections, q and k normalised and rotated     lp_qkv_projection_adapters
  norm      y = norm(x) (1 + scale_r) + shift_r                           lp_norm_modulate
  residual  h' = h + gate_r norm(u),  y = norm(h') (1 + scale_r) + shift_r   lp_gated_residual_norm

with r the request of a row.  `own` False: plain torch operations in binary32; True: the library.

Inputs are made on the device from the seed alone.  Activations that a projection reads are N(0, 1) in bf16, weights
N(0, 1 / d_in) in bf16; an adapter's down rows N(0, 1 / d_in) and its up rows 0.05 N(0, 1), so that an adapter of rank 64 adds
about 0.4 to a projection of O(1).  The residual stream has an offset and a spread of its own per channel and a few channels
far larger than the rest, as trained transformers have; scale, shift and gate are 0.3 N(0, 1).
"""
import math

import torch

own = False

EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # The time-conditioning layer of a guided pair of three requests: one row each, d_model 1536. Nothing but latency.
        dict(name="linear-conditioning", kind="linear", lengths="1,1,1,1,1,1", ranks="16,16,0,0,32,32", d_in=1536, d_out=1536, bias=True),
        # Text embeddings of twelve prompts of unequal length, projected to the model's width; every style its own adapter.
        dict(name="linear-prompts", kind="linear", lengths="77,12,226,1,154,33,90,0,181,64,127,8", ranks="8,16,24,32,0,64,16,8,40,32,16,128",
             d_in=4096, d_out=1536, bias=True),
        # Output projection of two guided requests, sub-latents of 33 and 49 frames at 480p cut along the width; the pair shares its adapter.
        dict(name="linear-480p", kind="linear", lengths="3780,3780,7410,7410", ranks="32,32,64,64", d_in=1536, d_out=1536, bias=True),
        # Output projection of the largest and the smallest sub-latent of the 720p configuration, two requests at once, no bias.
        dict(name="linear-720p", kind="linear", lengths="13230,11340", ranks="64,16", d_in=5120, d_out=5120, bias=False),
        # q | k | v of three tiny requests, two of them with adapters.
        dict(name="qkv-tiny", kind="qkv", grids="5x8x5,1x1x1,3x5x7", ranks="8,0,16", heads=4, head_dim=64, bias=True),
        # q | k | v of three requests of 480p sub-latents that differ in length, d_model 1536.
        dict(name="qkv-480p", kind="qkv", grids="9x30x14,9x30x14,13x17x52", ranks="32,32,16", heads=12, head_dim=128, bias=True),
        # q | k | v of the largest sub-latent of the 720p configuration, d_model 5120.
        dict(name="qkv-720p", kind="qkv", grids="21x45x14", ranks="32", heads=40, head_dim=128, bias=True),
        # Modulated layer normalisation in front of a small block's projections: five short requests, the smallest call.
        dict(name="norm-tiny", kind="norm", lengths="1,7,1,30,2", d=256, x="bf16", norm="layer", affine=False, modulated=True),
        # The same over the headline sub-latent, stream held in bf16.
        dict(name="norm-720p", kind="norm", lengths="13230", d=5120, x="bf16", norm="layer", affine=False, modulated=True),
        # Between two halves of a block, normalised before and after (RMS), stream in binary32: four requests at 480p.
        dict(name="residual-480p", kind="residual", lengths="3780,3780,7410,7410", d=1536, x="f32", post="rms", norm="rms", affine=True),
        # The same with the plain gate and a layer normalisation at 720p, two requests.
        dict(name="residual-720p", kind="residual", lengths="13230,11340", d=5120, x="bf16", post="none", norm="layer", affine=False),
        # A width that no vector divides, and the last residual of a model: nothing normalised behind it.
        dict(name="residual-odd", kind="residual", lengths="333,0,778", d=1153, x="f32", post="layer", norm="none", affine=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(values):
    return ",".join(str(v) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def draw(rng):
    """One more case of the same ranges; none costs more than the largest listed one."""
    kind = rng.choice(("linear", "linear", "linear", "qkv", "qkv", "norm", "norm", "residual", "residual"))
    most = {k: max(w[k] for w in map(work, listed())) for k in ("bytes", "flops")}
    rank = lambda: rng.choice((0, 8, 16, 16, 32, 32, 64, 8 * rng.randint(1, 16)))
    while True:
        # a few requests of like size, as a batch of videos is, or many of any
        count = rng.choice((1, 2, 2, 3, 4, _log_int(rng, 5, 48)))
        longest = _log_int(rng, 1, 24570)
        lengths = [rng.choice((longest, rng.randint(longest // 2, longest), rng.randint(0, longest))) for _ in range(count)]
        if sum(lengths) == 0:
            continue
        if kind == "linear":
            c = dict(kind=kind, lengths=_text(lengths), ranks=_text(rank() for _ in lengths), d_in=64 * _log_int(rng, 1, 96),
                     d_out=128 * _log_int(rng, 1, 48), bias=rng.random() < 0.6)
        elif kind == "qkv":
            grids = ["x".join(str(_log_int(rng, 1, top)) for top in (21, 45, 52)) for _ in lengths]
            c = dict(kind=kind, grids=_text(grids), ranks=_text(rank() for _ in lengths), heads=rng.choice((2, 4, 8, 12, 12, 16, 24, 40)),
                     head_dim=rng.choice((64, 128, 128)), bias=rng.random() < 0.6)
        else:
            d = rng.choice((8 * _log_int(rng, 16, 768), 64 * _log_int(rng, 4, 128), _log_int(rng, 65, 5120)))
            c = dict(kind=kind, lengths=_text(lengths), d=d, x=rng.choice(("bf16", "f32")), norm=rng.choice(("layer", "rms")),
                     affine=rng.random() < 0.5)
            if kind == "norm":
                c["modulated"] = rng.random() < 0.8
            else:
                c["post"] = rng.choice(("none", "none", "layer", "rms"))
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"]:
            return c


# ---- what each kind is made of

def _grids(c):
    return [tuple(int(v) for v in g.split("x")) for g in c["grids"].split(",")]


def _lengths(c):
    return [t * h * w for t, h, w in _grids(c)] if c["kind"] == "qkv" else _ints(c["lengths"])


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def work(case):
    lengths = _lengths(case)
    n = sum(lengths)
    if case["kind"] in ("linear", "qkv"):
        ranks = _ints(case["ranks"])
        parts = 3 if case["kind"] == "qkv" else 1
        d_in = case["heads"] * case["head_dim"] if parts == 3 else case["d_in"]
        d_out = 3 * d_in if parts == 3 else case["d_out"]
        kinds = {r: 0 for r in ranks}
        flops, size = 2 * n * d_in * d_out, 2 * (n * d_in + d_in * d_out + n * d_out) + (4 * d_out if case["bias"] else 0)
        for length, rank in zip(lengths, ranks):
            flops += 2 * length * rank * (parts * d_in + d_out)
            kinds[rank] = max(kinds[rank], length)
        # requests of one rank share an adapter: see prepare
        size += sum(2 * rank * (parts * d_in + d_out) for rank, length in kinds.items() if length)
        return {"bytes": size, "flops": flops}
    d, live = case["d"], sum(1 for x in lengths if x)
    wide = 4 if case["x"] == "f32" else 2
    weights = 4 * d * sum(2 if k == "layer" else 1 if k == "rms" else 0 for k in (case["norm"], case.get("post", "none"))) if case["affine"] else 0
    if case["kind"] == "norm":
        return {"bytes": n * d * (wide + 2) + weights + (8 * d * live if case["modulated"] else 0), "flops": 8 * n * d}
    normed = case["norm"] != "none"
    return {"bytes": n * d * (2 * wide + 2 + (2 if normed else 0)) + weights + 4 * d * live * (3 if normed else 1),
            "flops": n * d * (2 + (8 if normed else 0) + (6 if case["post"] != "none" else 0))}


class _Draws:
    """Tensors on the device from one seeded generator."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)

    def f32(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32)

    def bf16(self, *shape, scale=1.0):
        return (self.f32(*shape) * scale).to(torch.bfloat16)

    def stream(self, n, d):
        """The residual stream: an offset and a spread per channel, one channel in 128 twenty times as wide."""
        spread = torch.exp(0.5 * self.f32(d))
        spread[::128] *= 20.0
        return self.f32(n, d) * spread + 0.5 * self.f32(d)


def _inputs(case, seed):
    d = _Draws(seed)
    lengths = _lengths(case)
    n = sum(lengths)
    s = dict(case, lengths=lengths, starts=_starts(lengths), n=n)
    if case["kind"] in ("linear", "qkv"):
        ranks = _ints(case["ranks"])
        parts = 3 if case["kind"] == "qkv" else 1
        d_in = case["heads"] * case["head_dim"] if parts == 3 else case["d_in"]
        d_out = 3 * d_in if parts == 3 else case["d_out"]
        s.update(d_in=d_in, d_out=d_out, parts=parts)
        s["x"] = d.bf16(n, d_in)
        s["w"] = d.bf16(d_out, d_in, scale=d_in ** -0.5)
        s["bias_"] = 0.5 * d.f32(d_out) if case["bias"] else None
        # one adapter for every rank that occurs: requests of one rank are of one user
        kinds = {r: (d.bf16(parts * r, d_in, scale=d_in ** -0.5), d.bf16(d_out, r, scale=0.05), 1.0 if r < 64 else 0.5)
                 for r in sorted(set(ranks)) if r}
        s["adapters"] = [kinds.get(r) for r in ranks]
        if parts == 3:
            s["grids"] = _grids(case)
            s["offsets"] = [(0, 2 * i, 5) for i in range(len(lengths))]
            s["gains"] = [1.0 + 0.2 * d.f32(case["heads"], case["head_dim"]) for _ in range(2)]
        return s
    width = case["d"]
    s["requests_"] = len(lengths)
    s["mod"] = 0.3 * d.f32(len(lengths), 3, width)          # gate, scale, shift of every request
    affine = lambda kind: (1.0 + 0.2 * d.f32(width), 0.1 * d.f32(width) if kind == "layer" else None) if case["affine"] else (None, None)
    s["pre"] = None if case["norm"] == "none" else (case["norm"],) + affine(case["norm"])
    h = d.stream(n, width)
    s["h"] = h if case["x"] == "f32" else h.to(torch.bfloat16)
    if case["kind"] == "residual":
        s["post_"] = None if case["post"] == "none" else (case["post"],) + affine(case["post"])
        s["u"] = d.bf16(n, width)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if not own:
        return s
    from paper_2512_07350_amd import binding as lp
    s["stream"] = torch.cuda.current_stream().cuda_stream
    s["requests"] = lp.make_requests(s["starts"])
    bf16 = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    if s["kind"] in ("linear", "qkv"):
        s["table"] = lp.make_adapters(s["adapters"])
        size = lp.lp_adapter_workspace_size(s["n"], max([a[1].shape[1] for a in s["adapters"] if a] or [0]), s["parts"])
        s["ws"] = (torch.empty(max(size, 16), dtype=torch.uint8, device="cuda"), size)
        if s["kind"] == "linear":
            s["y"] = bf16(s["n"], s["d_out"])
        else:
            s["ropes"] = [lp.make_rope(g, o, None, BASE, head_dim=s["head_dim"]) for g, o in zip(s["grids"], s["offsets"])]
            s["out"] = [bf16(s["n"], s["heads"], s["head_dim"]) for _ in range(3)]
        return s
    kinds = {"layer": lp.LP_NORM_LAYER, "rms": lp.LP_NORM_RMS}
    norm = lambda t: None if t is None else lp.make_norm(kinds[t[0]], EPS, t[1], t[2])
    s["pre_"] = norm(s["pre"])
    gate, scale, shift = (s["mod"][:, i] for i in range(3))
    s["type"] = lp.LP_F32 if s["x"] == "f32" else lp.LP_BF16
    s["y"] = None if s["pre"] is None else bf16(s["n"], s["d"])
    if s["kind"] == "norm":
        s["vectors"] = lp.make_modulation(scale=scale, shift=shift) if s["modulated"] else None
    else:
        s["vectors"] = lp.make_modulation(gate=gate, scale=scale, shift=shift)
        s["after"] = norm(s["post_"])
        s["h_out"] = torch.empty_like(s["h"])
    return s


def run(state):
    """One pass.  Returns its outputs."""
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2512_07350_amd import binding as lp
    if s["kind"] == "linear":
        lp.lp_linear_adapters(s["x"], s["w"], s["bias_"], s["y"], s["requests"], s["d_in"], s["d_out"], s["table"], s["ws"][0], s["ws"][1],
                              s["stream"])
        return s["y"]
    if s["kind"] == "qkv":
        q, k, v = s["out"]
        lp.lp_qkv_projection_adapters(s["x"], s["w"], s["bias_"], s["gains"][0], s["gains"][1], EPS, s["ropes"], q, k, v, s["requests"],
                                      s["heads"], s["head_dim"], s["table"], s["ws"][0], s["ws"][1], s["stream"])
        return [q, k, v]
    if s["kind"] == "norm":
        lp.lp_norm_modulate(s["h"], s["type"], s["y"], s["requests"], s["d"], s["pre_"], s["vectors"], stream=s["stream"])
        return s["y"]
    lp.lp_gated_residual_norm(s["h"], s["type"], s["u"], s["h_out"], s["y"], s["requests"], s["d"], s["after"], s["pre_"], s["vectors"],
                              stream=s["stream"])
    return [s["h_out"]] if s["y"] is None else [s["h_out"], s["y"]]


# ---- the plain forms

def _rows(s):
    """(request, its rows) of the requests that have any."""
    return [(r, slice(a, b)) for r, (a, b) in enumerate(zip(s["starts"], s["starts"][1:])) if b > a]


def _project(s):
    """x W^T + b with the adapters' parts added, binary32 [n, d_out]."""
    x = s["x"].float()
    y = x @ s["w"].float().t()
    if s["bias_"] is not None:
        y += s["bias_"]
    section = s["d_out"] // s["parts"]
    for r, rows in _rows(s):
        if s["adapters"][r] is None:
            continue
        down, up, scale = s["adapters"][r]
        t = (x[rows] @ down.float().t()) * scale
        rank = up.shape[1]
        for p in range(s["parts"]):
            cols = slice(p * section, (p + 1) * section)
            y[rows, cols] += t[:, p * rank:(p + 1) * rank] @ up[cols].float().t()
    return y


def _parts(head_dim):
    hw = 2 * (head_dim // 6)
    return head_dim - 2 * hw, hw, hw


def _angles(s):
    """The rotation of every pair of a head, [n, head_dim / 2], in turns of 2 pi radians; positions times frequencies need 64 bits."""
    per_axis = [BASE ** (-torch.arange(0, p, 2, device="cuda", dtype=torch.float64) / p) for p in _parts(s["head_dim"])]
    out = []
    for grid, offset in zip(s["grids"], s["offsets"]):
        axes = [torch.arange(g, device="cuda", dtype=torch.float64) + o for g, o in zip(grid, offset)]
        where = torch.cartesian_prod(*axes).reshape(-1, 3)
        out.append(torch.cat([where[:, i:i + 1] * f for i, f in enumerate(per_axis)], dim=1))
    return torch.cat(out)


def _plain(s):
    if s["kind"] == "linear":
        return _project(s).to(torch.bfloat16)
    if s["kind"] == "qkv":
        y = _project(s).view(s["n"], 3, s["heads"], s["head_dim"])
        angle = _angles(s)
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        out = []
        for i in range(2):
            z = y[:, i]
            z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + EPS) * s["gains"][i]
            a, b = z[..., 0::2], z[..., 1::2]
            out.append(torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2).to(torch.bfloat16))
        return out + [y[:, 2].to(torch.bfloat16)]
    h = s["h"].float()
    gate, scale, shift = (_spread(s, s["mod"][:, i]) for i in range(3))
    if s["kind"] == "norm":
        y = _norm(h, s["pre"])
        return (y * (1.0 + scale) + shift if s["modulated"] else y).to(torch.bfloat16)
    u = s["u"].float()
    h = h + gate * (u if s["post_"] is None else _norm(u, s["post_"]))
    out = [h.to(s["h"].dtype)]
    if s["pre"] is not None:
        out.append((_norm(h, s["pre"]) * (1.0 + scale) + shift).to(torch.bfloat16))
    return out


def _spread(s, per_request):
    """A vector of every request, for every row."""
    of_row = torch.cat([torch.full((n,), r, dtype=torch.int64, device="cuda") for r, n in enumerate(s["lengths"])])
    return per_request[of_row]


def _norm(x, how):
    kind, weight, bias = how
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if weight is not None:
        x = x * weight
    return x if bias is None else x + bias


# ---- the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    wide = lambda t: t.double()
    if s["kind"] in ("linear", "qkv"):
        y = torch.empty(s["n"], s["d_out"], dtype=torch.float64, device="cuda")
        section = s["d_out"] // s["parts"]
        for r, rows in _rows(s):
            w = wide(s["w"])
            if s["adapters"][r] is not None:              # the weights this request's rows see: W + s U D
                down, up, factor = s["adapters"][r]
                for p in range(s["parts"]):
                    at = slice(p * section, (p + 1) * section)
                    w[at] += factor * (wide(up[at]) @ wide(down[p * up.shape[1]:(p + 1) * up.shape[1]]))
            y[rows] = wide(s["x"][rows]) @ w.t()
        if s["bias_"] is not None:
            y = y + wide(s["bias_"])
        if s["kind"] == "linear":
            return y
        q, k, v = (y[:, p * section:(p + 1) * section].reshape(s["n"], s["heads"], s["head_dim"]) for p in range(3))
        return [_turned(s, q, wide(s["gains"][0])), _turned(s, k, wide(s["gains"][1])), v.contiguous()]
    gate, scale, shift = (torch.repeat_interleave(wide(s["mod"][:, i]), torch.tensor(s["lengths"], device="cuda"), dim=0) for i in range(3))
    h = wide(s["h"])
    if s["kind"] == "norm":
        y = _standard(h, s["pre"])
        return y + y * scale + shift if s["modulated"] else y
    u = wide(s["u"])
    h = h + gate * (u if s["post_"] is None else _standard(u, s["post_"]))
    if s["pre"] is None:
        return [h]
    y = _standard(h, s["pre"])
    return [h, y + y * scale + shift]


def _standard(x, how):
    kind, weight, bias = how
    if kind == "layer":
        mean = x.sum(-1, keepdim=True) / x.shape[-1]
        y = (x - mean) / torch.sqrt(((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    else:
        y = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    if weight is not None:
        y = y * weight.double()
    return y if bias is None else y + bias.double()


def _turned(s, z, gain):
    """Per-head RMS normalisation, then every pair of elements as a complex number times e^(i angle)."""
    z = z / torch.sqrt((z ** 2).sum(-1, keepdim=True) / s["head_dim"] + EPS) * gain
    pair = torch.view_as_complex(z.reshape(s["n"], s["heads"], -1, 2).contiguous())
    turns = []
    for (gt, gh, gw), off in zip(s["grids"], s["offsets"]):
        i = torch.arange(gt * gh * gw, device="cuda")
        coords = (i // (gh * gw) + off[0], i // gw % gh + off[1], i % gw + off[2])
        cols = []
        for axis, p in enumerate(_parts(s["head_dim"])):
            for j in range(p // 2):
                cols.append(coords[axis].double() * math.pow(BASE, -2.0 * j / p))
        turns.append(torch.stack(cols, dim=1))
    angle = torch.cat(turns)
    return torch.view_as_real(pair * torch.polar(torch.ones_like(angle), angle)[:, None]).reshape(z.shape)
