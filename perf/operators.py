"""What a transformer layer does between its residual stream and the attention call, forward and backward, as cases.

Three operators, each with its gradients:

``norm``   layer normalisation of ``[B, N, C]`` rows with a gain and a bias, shared (``affine``) or one pair for each batch
           entry with gain ``1 + scale`` (``modulated``, as diffusion transformers condition their layers).
``rope``   rotary positions of Q and K: pairs of neighbouring channels (``interleaved``) or of channels half the rotary
           part apart (``half``), over all or part of a head, positions on one or three axes, frequencies scaled for
           sequences longer than those of training; Q and K may lie in one packed projection.
``prep``   the gradient of the Q/K preparation (RMS normalisation with gains, rotary embedding, factor on Q).

``own`` decides what ``run`` computes them with: plain torch operations, or the library's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
THETA = 10000.0


def _norm(name, direction, dtype, B, N, C, form):
    return {"name": name, "op": "norm", "direction": direction, "dtype": dtype, "B": B, "N": N, "C": C, "form": form}


def _rope(name, direction, dtype, B, N, H, Hk, d, rot, layout, axes, scaling, packed, far):
    return {"name": name, "op": "rope", "direction": direction, "dtype": dtype, "B": B, "N": N, "H": H, "Hk": Hk, "d": d,
            "rot": rot, "layout": layout, "axes": axes, "scaling": scaling, "packed": packed, "far": far}


def _prep(name, dtype, B, H, grid_h, grid_w, n_text, d, ntk, q_factor):
    return {"name": name, "op": "prep", "direction": "bwd", "dtype": dtype, "B": B, "H": H, "grid_h": grid_h, "grid_w": grid_w,
            "n_text": n_text, "d": d, "ntk": ntk, "q_factor": q_factor}


def listed():
    return [
        # conditioning vectors, one token for the conditional and one for the unconditional half: latency
        _norm("norm_fwd_1_token", "fwd", "bf16", 2, 1, 768, "modulated"),
        # full-precision evaluation of a small picture (24 x 40 grid, 130 text tokens), an odd number of channels
        _norm("norm_fwd_24x40_odd_f32", "fwd", "f32", 1, 24 * 40 + 130, 1003, "affine"),
        # a layer of the largest picture (512 x 512 grid, 512 text tokens), 16 heads of 128: the largest call
        _norm("norm_fwd_8k", "fwd", "bf16", 1, 512 * 512 + 512, 2048, "modulated"),
        # distillation of a layer at 2048 px, 24 heads of 64
        _norm("norm_bwd_2048px", "bwd", "bf16", 1, 128 * 128 + 512, 1536, "modulated"),
        # gradients in full precision, landscape pictures that fill no tile, odd number of channels, shared weights
        _norm("norm_bwd_67x120_odd_f32", "bwd", "f32", 2, 67 * 120 + 300, 1003, "affine"),
        # one new token a sequence far into a long context, halves of both guidance branches
        _rope("rope_fwd_1_token", "fwd", "bf16", 2, 1, 24, 8, 128, 128, "half", 1, "parts", False, 1000000),
        # Q and K of the ordinary 1024 px layer out of its packed projection into heads, positions on three axes
        _rope("rope_fwd_1024px_packed", "fwd", "bf16", 1, 64 * 64 + 512, 24, 24, 128, 128, "interleaved", 3, "ntk", True, 0),
        # long sequence, half of each head turned, three query heads to a key head, frequencies scaled by parts
        _rope("rope_fwd_64k_part", "fwd", "bf16", 1, 256 * 256 + 512, 24, 8, 128, 64, "half", 1, "parts", False, 0),
        # gradients in full precision, ragged batch of two, heads of 80 channels of which 40 turn
        _rope("rope_bwd_67x120_part_f32", "bwd", "f32", 2, 67 * 120 + 300, 12, 12, 80, 40, "half", 1, "linear", False, 0),
        # gradient check of the tiny configuration
        _prep("prep_bwd_tiny_f32", "f32", 1, 2, 16, 16, 16, 64, 1.0, 1.0),
        # distillation at the training resolution, and of a layer at 4096 px with the high-resolution factors
        _prep("prep_bwd_1024px", "bf16", 1, 24, 64, 64, 512, 128, 1.0, 1.0),
        _prep("prep_bwd_4096px", "bf16", 1, 24, 256, 256, 512, 128, 10.0, 1.07),
    ]


def _elements(c):
    """Elements of the largest tensors of a case, those that set its cost."""
    if c["op"] == "norm":
        return c["B"] * c["N"] * c["C"]
    if c["op"] == "rope":
        return c["B"] * c["N"] * (c["H"] + c["Hk"]) * c["d"]
    return 2 * c["B"] * c["H"] * (c["n_text"] + c["grid_h"] * c["grid_w"]) * c["d"]


def draw(rng):
    def spread(lo, hi):
        return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    op = rng.choice(("norm", "norm", "rope", "rope", "prep"))
    direction = rng.choice(("fwd", "bwd"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        heads, d = rng.choice((2, 8, 12, 16, 24)), rng.choice((64, 128))
        C = rng.choice((heads * d, heads * d, spread(64, 8192)))
        c = _norm("", direction, dtype, rng.choice((1, 1, 2, 3)), spread(1, 262656), C, rng.choice(("affine", "modulated")))
        shrink = ("N",)
    elif op == "rope":
        d = rng.choice((64, 128, 128, 40, 72, 80, 96, 256))
        rot = rng.choice((d, d, d // 2, max(2, d // 4 // 2 * 2)))
        H = rng.choice((2, 8, 12, 16, 24))
        axes = rng.choice((1, 1, 3)) if rot >= 16 else 1
        c = _rope("", direction, dtype, rng.choice((1, 1, 2)), spread(1, 66048), H, rng.choice((H, H, H // 2, 1)), d, rot,
                  rng.choice(("half", "interleaved")), axes, rng.choice(("none", "linear", "ntk", "parts")),
                  rng.random() < 0.4, rng.choice((0, 0, 1000, 1000000)) if axes == 1 else 0)
        shrink = ("N",)
    else:
        c = _prep("", dtype, rng.choice((1, 1, 2)), rng.choice((2, 8, 12, 16, 24)), spread(1, 256), spread(1, 256),
                  rng.choice((0, 16, 77, 128, 300, 512)), rng.choice((64, 128)), rng.choice((1.0, 2.0, 10.0)),
                  rng.choice((1.0, 1.07)))
        shrink = ("grid_h", "grid_w")
    del c["name"]
    most = max(_elements(x) * x_size for x, x_size in ((y, 2 if y["dtype"] == "bf16" else 4) for y in listed()
                                                      if y["op"] == op and y["direction"] == direction))
    while _elements(c) * (2 if dtype == "bf16" else 4) > most:
        key = max(shrink, key=c.get)
        c[key] = max(1, c[key] * 3 // 4)
    return c


# ---- inputs ----------------------------------------------------------------------------------------------------------


def _axis_dims(rot, axes):
    """Channels of each axis' group: all of them, or an eighth and two equal rests as in (16, 56, 56) of 128."""
    if axes == 1:
        return (rot,)
    first = rot // 8 // 2 * 2
    second = (rot - first) // 4 * 2
    return (first, second, rot - first - second)


def _frequencies(dim, scaling, factor=8.0, trained=4096.0, fast=32.0, slow=1.0):
    """Angular frequencies of a group of ``dim`` channels, theta^(-2k/dim), scaled for ``factor`` times the trained length."""
    out = []
    for k in range(dim // 2):
        base = THETA * factor ** (dim / (dim - 2)) if scaling == "ntk" and dim > 2 else THETA
        w = base ** (-2.0 * k / dim)
        if scaling == "linear":
            w /= factor
        elif scaling == "parts":  # frequencies that turn often within the trained length stay, slow ones are interpolated
            keep = min(1.0, max(0.0, (trained * w / (2 * math.pi) - slow) / (fast - slow)))
            w *= keep + (1.0 - keep) / factor
        out.append(w)
    return out


def _grid_positions(grid_h, grid_w, n_text, dev):
    """Text tokens at the origin, image tokens at (0, row, column)."""
    pos = torch.zeros(n_text + grid_h * grid_w, 3, dtype=torch.int32, device=dev)
    p = torch.arange(grid_h * grid_w, device=dev)
    pos[n_text:, 1] = p // grid_w
    pos[n_text:, 2] = p % grid_w
    return pos


def prepare(case, seed):
    dev, dtype = torch.device("cuda"), DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32)

    s = {"case": case, "op": case["op"], "direction": case["direction"]}
    if case["op"] == "norm":
        B, N, C = case["B"], case["N"], case["C"]
        # a residual stream: channels of their own mean and size, a few of them far larger than the rest
        size = torch.exp(0.5 * normal(C))
        size[:: max(1, C // 5)] *= 8.0
        x = normal(B, N, C)
        x *= size
        x += 0.5 + 0.5 * normal(C)
        s["x"] = x.to(dtype)
        del x
        if case["form"] == "modulated":  # shift, scale and gate of the layer in one row a batch entry, in the stream's type
            modulation = (0.3 * normal(B, 3 * C)).to(dtype)
            s["bias"], s["weight"] = modulation[:, :C], modulation[:, C:2 * C]
            s["offset"] = 1.0
        else:
            s["weight"], s["bias"] = 1.0 + 0.2 * normal(C), 0.2 * normal(C)
            s["offset"] = 0.0
        s["mean"], s["rstd"] = (torch.empty(B, N, device=dev, dtype=torch.float32) for _ in range(2))
        if case["direction"] == "fwd":
            s["y"] = torch.empty_like(s["x"])
        else:
            s["dy"] = normal(B, N, C).to(dtype)
            wide = s["x"].float()
            s["mean"].copy_(wide.mean(-1))
            wide -= s["mean"].unsqueeze(-1)
            s["rstd"].copy_(torch.rsqrt(wide.square_().mean(-1) + EPS))
            del wide
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = (torch.empty(s["weight"].shape, device=dev, dtype=s["weight"].dtype) for _ in range(2))
    elif case["op"] == "rope":
        B, N, H, Hk, d = (case[k] for k in ("B", "N", "H", "Hk", "d"))
        if case["axes"] == 3:
            n_text = min(512, N // 4)
            width = math.isqrt(N - n_text)
            s["positions"] = _grid_positions(-(-(N - n_text) // width), width, n_text, dev)[:N].unsqueeze(0).contiguous()
        else:
            start = torch.randint(0, case["far"] + 1, (B, 1), generator=gen, device=dev, dtype=torch.int32)
            s["positions"] = (start + torch.arange(N, device=dev, dtype=torch.int32)).unsqueeze(-1).contiguous()
        s["axes_dim"] = _axis_dims(case["rot"], case["axes"])
        s["freqs"] = torch.tensor([w for dim in s["axes_dim"] for w in _frequencies(dim, case["scaling"])], dtype=torch.float64)
        s["factor"] = 0.1 * math.log(8.0) + 1.0 if case["scaling"] == "parts" else 1.0
        heads = [torch.empty(B, h, N, d, device=dev, dtype=dtype) for h in (H, Hk)]
        if case["packed"]:  # the projection's rows: query heads, key heads, value heads of each token
            rows = torch.zeros(B, N, H + 2 * Hk, d, device=dev, dtype=dtype)
            packed = [rows[:, :, :H].transpose(1, 2), rows[:, :, H:H + Hk].transpose(1, 2)]
        else:
            packed = [torch.empty_like(t) for t in heads]
        src, dst = (packed, heads) if case["direction"] == "fwd" else (heads, packed)
        for t in src:
            t.copy_(normal(*t.shape))
        (s["q"], s["k"]), (s["q_out"], s["k_out"]) = src, dst
    else:
        B, H, d = case["B"], case["H"], case["d"]
        s["geometry"] = (case["grid_h"], case["grid_w"], case["n_text"])
        N = case["n_text"] + case["grid_h"] * case["grid_w"]
        for name in ("q", "k", "dq_rot", "dk_rot"):
            s[name] = normal(B, H, N, d).to(dtype)
        for name in ("dq", "dk"):
            s[name] = torch.empty(B, H, N, d, device=dev, dtype=dtype)
        s["gain_q"], s["gain_k"] = 1.0 + 0.1 * normal(d), 1.0 + 0.1 * normal(d)
        s["dgain_q"], s["dgain_k"] = (torch.empty(d, device=dev, dtype=torch.float32) for _ in range(2))
        s["axes_dim"] = (d // 8, d * 7 // 16, d * 7 // 16)
    return s


# ---- the operators ---------------------------------------------------------------------------------------------------


def _norm_fwd(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    gain, bias = s["offset"] + s["weight"].float(), s["bias"].float()
    if gain.dim() == 2:
        gain, bias = gain.unsqueeze(1), bias.unsqueeze(1)
    return (x * rstd * gain + bias).to(s["x"].dtype), mean.squeeze(-1), rstd.squeeze(-1)


def _norm_bwd(s):
    x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"].unsqueeze(-1)
    x = (x - s["mean"].unsqueeze(-1)) * rstd
    gain = s["offset"] + s["weight"].float()
    rows = (1,) if gain.dim() == 2 else (0, 1)
    g = dy * (gain.unsqueeze(1) if gain.dim() == 2 else gain)
    dx = rstd * (g - g.mean(-1, keepdim=True) - x * (g * x).mean(-1, keepdim=True))
    kind = s["weight"].dtype
    return dx.to(s["x"].dtype), (dy * x).sum(rows).to(kind), dy.sum(rows).to(kind)


def _turn(a, b, cos, sin):
    return a * cos - b * sin, a * sin + b * cos


def _rope_plain(s):
    case = s["case"]
    rot, half = case["rot"], case["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(len(s["axes_dim"])), torch.tensor([n // 2 for n in s["axes_dim"]]))
    angle = s["positions"].double()[:, :, axis.to("cuda")] * s["freqs"].to("cuda")
    if case["direction"] == "bwd":
        angle = -angle
    cos, sin = (s["factor"] * torch.cos(angle)).float().unsqueeze(1), (s["factor"] * torch.sin(angle)).float().unsqueeze(1)

    def turned(x):
        x = x.float()
        if case["layout"] == "half":
            lo, hi = _turn(x[..., :half], x[..., half:rot], cos, sin)
            return torch.cat((lo, hi, x[..., rot:]), -1)
        even, odd = _turn(x[..., 0:rot:2], x[..., 1:rot:2], cos, sin)
        return torch.cat((torch.stack((even, odd), -1).flatten(-2), x[..., rot:]), -1)

    return s["q_out"].copy_(turned(s["q"])), s["k_out"].copy_(turned(s["k"]))


def _prep_bwd(s):
    case = s["case"]
    axis = torch.repeat_interleave(torch.arange(3), torch.tensor([n // 2 for n in s["axes_dim"]])).to("cuda")
    freqs = torch.tensor([w for dim in s["axes_dim"] for w in _ntk(dim, case["ntk"])], dtype=torch.float64).to("cuda")
    angle = _grid_positions(*s["geometry"], "cuda").double()[:, axis] * freqs
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def grads(x, dy, gain, factor):
        kind, x, dy = x.dtype, x.float(), dy.float()
        even, odd = _turn(dy[..., 0::2], dy[..., 1::2], cos, -sin)
        u = factor * torch.stack((even, odd), -1).flatten(-2)
        inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        x = x * inv
        t = u * gain
        return (inv * (t - x * (t * x).mean(-1, keepdim=True))).to(kind), (u * x).sum((0, 1, 2))

    dq, dgain_q = grads(s["q"], s["dq_rot"], s["gain_q"], case["q_factor"])
    dk, dgain_k = grads(s["k"], s["dk_rot"], s["gain_k"], 1.0)
    return dq, dk, dgain_q, dgain_k


def _ntk(dim, ntk):
    base = THETA * ntk ** (dim / (dim - 2)) if dim > 2 else THETA
    return [base ** (-2.0 * k / dim) for k in range(dim // 2)]


def _with_the_library(s):
    from paper_2412_16112_b200 import binding as clear

    case = s["case"]
    if s["op"] == "norm" and s["direction"] == "fwd":
        clear.clear_layer_norm_fwd(s["x"], s["y"], s["weight"], s["bias"], s["mean"], s["rstd"], weight_offset=s["offset"], eps=EPS)
        return s["y"], s["mean"], s["rstd"]
    if s["op"] == "norm":
        return clear.clear_layer_norm_bwd(s["x"], s["dy"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"],
                                          weight_offset=s["offset"])
    if s["op"] == "rope":
        call = clear.clear_rope_fwd if s["direction"] == "fwd" else clear.clear_rope_bwd
        layout = clear.ROPE_HALF if case["layout"] == "half" else clear.ROPE_INTERLEAVED
        return call(s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], s["freqs"], s["axes_dim"], layout, s["factor"])
    return clear.clear_qk_norm_rope_bwd(s["q"], s["k"], s["dq_rot"], s["dk_rot"], s["dq"], s["dk"], *s["geometry"], s["axes_dim"],
                                        s["gain_q"], s["gain_k"], s["dgain_q"], s["dgain_k"], theta=THETA,
                                        ntk_factor=case["ntk"], eps=EPS, q_factor=case["q_factor"])


def run(s):
    if own:
        return _with_the_library(s)
    if s["op"] == "norm":
        return _norm_fwd(s) if s["direction"] == "fwd" else _norm_bwd(s)
    return _rope_plain(s) if s["op"] == "rope" else _prep_bwd(s)


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    n = _elements(case)
    if case["op"] == "norm":
        rows, fwd = case["B"] * case["N"], case["direction"] == "fwd"
        params = case["C"] * (case["B"] * size if case["form"] == "modulated" else 4)
        # x in, y out; or x and dy in, dx out; mean and rstd of each row; gain and bias, or the gain and two gradients
        return {"bytes": float((2 if fwd else 3) * n * size + 8 * rows + (2 if fwd else 3) * params),
                "flops": float((8 if fwd else 14) * n)}
    if case["op"] == "rope":
        turned = n // case["d"] * case["rot"]
        positions = 4 * case["N"] * (case["axes"] if case["axes"] == 3 else case["B"])
        return {"bytes": float(2 * n * size + positions), "flops": float(3 * turned)}
    # q, k and the gradients of their rotated forms in, two gradients out; two gains and their gradients
    return {"bytes": float(3 * n * size + 16 * case["d"]), "flops": float(15 * n)}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm_fwd(s) if case["direction"] == "fwd" else _exact_norm_bwd(s)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    return _exact_prep(case, s)


def _exact_norm_fwd(s):
    x = s["x"].double()
    w, bias = (s[name].double().reshape(-1, 1, x.shape[-1]) for name in ("weight", "bias"))
    var, mean = torch.var_mean(x, dim=-1, correction=0)
    rstd = (var + EPS) ** -0.5
    return torch.addcmul(bias, (x - mean[..., None]) * rstd[..., None], w + s["offset"]), mean, rstd


def _exact_norm_bwd(s):
    dy, rstd = s["dy"].double(), s["rstd"].double()
    C = dy.shape[-1]
    w = (s["weight"].double() + s["offset"]).reshape(-1, C).expand(dy.shape[0], C)
    h = torch.einsum("bnc,bn->bnc", s["x"].double() - s["mean"].double()[..., None], rstd)
    dw, db = torch.einsum("bnc,bnc->bc", dy, h), torch.einsum("bnc->bc", dy)
    along, level = torch.einsum("bnc,bnc,bc->bn", dy, h, w) / C, torch.einsum("bnc,bc->bn", dy, w) / C
    dx = torch.einsum("bnc,bn->bnc", dy * w[:, None] - level[..., None] - h * along[..., None], rstd)
    return (dx, dw.sum(0), db.sum(0)) if s["weight"].dim() == 1 else (dx, dw, db)


def _exact_rope(case, s):
    """Pairs as complex numbers, times the unit number of their angle."""
    pairs = torch.tensor([n // 2 for n in s["axes_dim"]], device="cuda")
    place = torch.repeat_interleave(s["positions"].double(), pairs, dim=-1)
    angle = torch.einsum("bnp,p->bnp", place, s["freqs"].to("cuda"))[:, None]
    turn = torch.polar(torch.full_like(angle, s["factor"]), -angle if case["direction"] == "bwd" else angle)
    rot = case["rot"]

    def turned(x):
        x = x.double()
        if case["layout"] == "half":
            z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
            return torch.cat((z.real, z.imag, x[..., rot:]), -1)
        z = torch.view_as_complex(x[..., :rot].unflatten(-1, (rot // 2, 2)).contiguous()) * turn
        return torch.cat((torch.view_as_real(z).flatten(-2), x[..., rot:]), -1)

    return turned(s["q"]), turned(s["k"])


def _exact_prep(case, s):
    """Through the derivative of the preparation itself."""
    grid_h, grid_w, n_text = s["geometry"]
    pad = torch.zeros(n_text, device="cuda", dtype=torch.float64)
    row = torch.arange(grid_h, device="cuda", dtype=torch.float64).repeat_interleave(grid_w)
    col = torch.arange(grid_w, device="cuda", dtype=torch.float64).repeat(grid_h)

    def angles(place, dim):
        base = THETA * case["ntk"] ** (dim / (dim - 2)) if dim > 2 else THETA
        return torch.outer(place, base ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim))

    first, second, third = s["axes_dim"]
    still = torch.zeros(n_text + grid_h * grid_w, first // 2, device="cuda", dtype=torch.float64)
    turn = torch.exp(1j * torch.cat((still, angles(torch.cat((pad, row)), second), angles(torch.cat((pad, col)), third)), -1))

    def grads(x, dy, gain, factor):
        x, gain = x.double().requires_grad_(), gain.double().requires_grad_()
        unit = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
        y = torch.view_as_real(torch.view_as_complex(unit.unflatten(-1, (-1, 2))) * turn).flatten(-2) * factor
        return torch.autograd.grad(y, (x, gain), dy.double())

    dq, dgain_q = grads(s["q"], s["dq_rot"], s["gain_q"], case["q_factor"])
    dk, dgain_k = grads(s["k"], s["dk_rot"], s["gain_k"], 1.0)
    return dq, dk, dgain_q, dgain_k
