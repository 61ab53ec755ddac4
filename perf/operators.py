"""The operators of a training step on packed rows, as timed cases.

``rope``   rotary positions of the query and key rows: angles from coordinates that a row finds through an index, half or
           interleaved pairs, the whole head or part of it, forward and inverse (the way of the gradient).
``attn``   attention over packed sequences with its row statistics, and its gradients: one forward and one backward pass.
``norm``   the backward pass of LayerNorm over packed rows, with the gradients of gamma and beta and, where the rows have a
           residual branch, its gradient added.
``clip``   the norm over the gradients of a whole model, clipped into the tensors that the optimiser reads.

Geometry: head dim 64 with 3, 6, 12 or 16 heads, 197 and 577 tokens an image as in the package's workloads, generic sizes
besides.  Activations and gradients are N(0, 1) or a small multiple of it; kept tokens are spread over a batch at random, so that
every image has another length, and the class token is always among them.
"""
import math

import torch

own = False
DEV = "cuda:0"
D = 64
EPS = 1e-6
_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token of a serving loop at a far position
        {"name": "rope_token", "kind": "rope", "B": 1, "N": 1, "keep": 1.0, "Hq": 12, "Hk": 12, "D": 64, "rot": 64, "axes": 1,
         "layout": "half", "far": 100000, "scaling": "none", "inverse": False, "dtype": "f16"},
        # patches of 384 x 384 images behind a pruning point, two axes, coordinates through the gather index
        {"name": "rope_patches_bs64", "kind": "rope", "B": 64, "N": 577, "keep": 0.5, "Hq": 12, "Hk": 12, "D": 64, "rot": 64, "axes": 2,
         "layout": "half", "far": 0, "scaling": "none", "inverse": False, "dtype": "bf16"},
        # gradients of a long text batch: shared key heads, half of the head rotated, frequencies scaled by parts
        {"name": "rope_long_inverse", "kind": "rope", "B": 2, "N": 16387, "keep": 1.0, "Hq": 16, "Hk": 4, "D": 128, "rot": 64, "axes": 1,
         "layout": "interleaved", "far": 1000000, "scaling": "parts", "inverse": True, "dtype": "f16"},
        # the smallest training step: two images of a 3-head model
        {"name": "attn_tiny", "kind": "attn", "B": 2, "N": 197, "H": 3, "keep": 0.6, "fused": False, "dtype": "f16"},
        # fine-tuning at 80 % pruned, fused QKV
        {"name": "attn_bs32_keep20", "kind": "attn", "B": 32, "N": 197, "H": 12, "keep": 0.2, "fused": True, "dtype": "bf16"},
        # an unpruned layer in front of the pruning point
        {"name": "attn_bs64_dense", "kind": "attn", "B": 64, "N": 197, "H": 12, "keep": 1.0, "fused": True, "dtype": "f16"},
        # 384 x 384 images, unpruned
        {"name": "attn_384_dense", "kind": "attn", "B": 32, "N": 577, "H": 12, "keep": 1.0, "fused": True, "dtype": "bf16"},
        # two images of the smallest model
        {"name": "norm_tiny", "kind": "norm", "rows": 394, "cap": 394, "C": 192, "residual": False, "dtype": "f16"},
        # the packed rows of a pruned batch in buffers made for the whole one
        {"name": "norm_bs32_keep20", "kind": "norm", "rows": 1289, "cap": 6304, "C": 768, "residual": True, "dtype": "bf16"},
        # the rows of 128 unpruned images of a 16-head model
        {"name": "norm_bs128_wide", "kind": "norm", "rows": 25216, "cap": 25216, "C": 1024, "residual": True, "dtype": "f16"},
        # all gradients of a 3-head, 12-block model, fp32, a good part of the tensors tiny
        {"name": "clip_small", "kind": "clip", "H": 3, "depth": 12, "src": "f32", "dst": "f32", "scale": 1.0, "max_norm": 1.0},
        # bf16 gradients of a 16-head, 12-block model into fp32, a loss scale undone on the way
        {"name": "clip_large_bf16", "kind": "clip", "H": 16, "depth": 12, "src": "bf16", "dst": "f32", "scale": 0.0078125, "max_norm": 1.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: odd row counts, batches up to the listed largest, every layout and type."""
    kind = rng.choice(("rope", "attn", "attn", "norm", "clip"))
    half = rng.choice(("f16", "bf16"))
    if kind == "rope":
        d = rng.choice((64, 64, 80, 128))
        hq = rng.choice((3, 6, 12, 16))
        axes = rng.choice((1, 2))
        rot = rng.choice((d, d // 2, 20))
        rows = _log_int(rng, 1, max(1, 32774 * 16 * 128 // (hq * d) // 2))
        n = rng.choice((1, 197, 577)) if axes == 2 else max(1, rows)
        return {"kind": kind, "B": max(1, rows // n), "N": n, "keep": 1.0 if axes == 1 else round(rng.uniform(0.1, 1.0), 2), "Hq": hq,
                "Hk": rng.choice((hq, hq, 3 if hq % 3 == 0 else 4)), "D": d, "rot": rot, "axes": axes, "layout": rng.choice(("half", "interleaved")),
                "far": 0 if axes == 2 else _log_int(rng, 1000, 1000000), "scaling": rng.choice(("none", "linear", "base", "parts")),
                "inverse": rng.choice((False, True)), "dtype": half}
    if kind == "attn":
        n = rng.choice((197, 577, _log_int(rng, 1, 900)))
        h = rng.choice((3, 6, 12, 16))
        most = int(32 * 12 * 577 * 577 / (h * n * n))
        rows = 64 * 197 * 12 // (h * n)
        return {"kind": kind, "B": _log_int(rng, 1, max(1, min(128, most, rows))), "N": n, "H": h, "keep": round(rng.uniform(0.1, 1.0), 2),
                "fused": rng.choice((False, True)), "dtype": half}
    if kind == "norm":
        c = rng.choice((192, 384, 768, 1024, 8 * _log_int(rng, 1, 256)))
        cap = _log_int(rng, 1, max(1, min(25216, 25216 * 1024 // c)))
        return {"kind": kind, "rows": max(1, int(cap * rng.choice((1.0, 1.0, rng.uniform(0.1, 1.0))))), "cap": cap, "C": c,
                "residual": rng.choice((False, True)), "dtype": half}
    src = rng.choice(("f32", "f16", "bf16"))
    return {"kind": kind, "H": rng.choice((1, 2, 3, 5, 6, 8)), "depth": rng.choice((1, 4, 8, 12)), "src": src, "dst": rng.choice((src, "f32")),
            "scale": rng.choice((1.0, 0.0078125)), "max_norm": rng.choice((0.5, 1.0, 1e9))}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 11)


def _randn(gen, dtype, *shape, times=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * times).to(_DTYPES[dtype])


def _rows(case):
    """Kept rows of the whole batch: the class token of every image and a share of the others."""
    return case["B"] + int(round(case["keep"] * case["B"] * (case["N"] - 1)))


def _kept(case, seed):
    """Flat padded positions of the kept rows and the lengths of the images: the tokens that score highest over the whole batch."""
    gen = torch.Generator().manual_seed(int(seed) * 31 + 7)
    score = torch.rand(case["B"], case["N"], generator=gen)
    score[:, 0] = 2.0
    keep = torch.zeros(case["B"] * case["N"], dtype=torch.bool)
    keep[score.reshape(-1).topk(_rows(case)).indices] = True
    return keep.nonzero().reshape(-1), keep.reshape(case["B"], -1).sum(dim=1)


def _frequencies(case):
    """Radians per unit of a coordinate, one for each pair; the pairs of an axis are consecutive."""
    pairs = case["rot"] // 2 // case["axes"]
    p = torch.arange(pairs, dtype=torch.float64)
    base, factor, length = 10000.0, 8.0, 4096.0
    if case["scaling"] == "base" and pairs > 1:
        base *= factor ** (pairs / (pairs - 1))
    f = base ** (-p / pairs)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        kept = ((length * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f * kept + f / factor * (1.0 - kept)
    return f.repeat(case["axes"])


def _parameters(case):
    """Sizes of the gradients of an encoder: embedding, positions, blocks of qkv, projection, two MLP layers and two norms, head."""
    c = case["H"] * D
    block = [(c,), (c,), (3 * c, c), (3 * c,), (c, c), (c,), (c,), (c,), (4 * c, c), (4 * c,), (c, 4 * c), (c,)]
    return [(1, 1, c), (1, 197, c), (c, 768), (c,)] + block * case["depth"] + [(c,), (c,), (1000, c), (1000,)]


def prepare(case, seed):
    kind, gen, dt = case["kind"], _gen(seed), case.get("dtype")
    if kind == "rope":
        flat, _ = _kept(case, seed)
        rows = flat.numel()
        q, k = _randn(gen, dt, rows, case["Hq"], case["D"]), _randn(gen, dt, rows, case["Hk"], case["D"])
        if case["axes"] == 2:
            # the class token at the origin, patches on a square grid; a row finds its token through the gather index
            side = max(1, math.isqrt(case["N"] - 1))
            t = torch.arange(max(1, case["N"]), device=DEV) - 1
            coords = torch.stack((t // side, t % side), dim=1).clamp(min=0).float()
            coords[0] = 0
            index = flat.to(torch.int32).to(DEV)
        else:
            coords = torch.arange(case["far"], device=DEV, dtype=torch.float32).reshape(-1, 1)
            index = torch.randint(0, case["far"], (rows,), generator=gen, device=DEV, dtype=torch.int32)
        return {"case": case, "q": q, "k": k, "coords": coords, "index": index, "freqs": _frequencies(case).to(DEV),
                "q_out": torch.empty_like(q), "k_out": torch.empty_like(k), "amplitude": 1.0 if case["scaling"] != "parts" else 0.1 * math.log(8.0) + 1.0}
    if kind == "attn":
        _, lengths = _kept(case, seed)
        rows, h = int(lengths.sum()), case["H"]
        cu = torch.zeros(case["B"] + 1, dtype=torch.int32)
        cu[1:] = torch.cumsum(lengths, 0)
        if case["fused"]:
            q, k, v = _randn(gen, dt, rows, 3, h, D).unbind(1)
            dq, dk, dv = torch.empty(rows, 3, h, D, device=DEV, dtype=_DTYPES[dt]).unbind(1)
        else:
            q, k, v = (_randn(gen, dt, rows, h, D) for _ in range(3))
            dq, dk, dv = (torch.empty(rows, h, D, device=DEV, dtype=_DTYPES[dt]) for _ in range(3))
        return {"case": case, "q": q, "k": k, "v": v, "do": _randn(gen, dt, rows, h, D), "cu": cu.to(DEV), "scale": D ** -0.5,
                "lengths": lengths.to(DEV), "longest": int(lengths.max()), "rows": rows, "o": torch.empty(rows, h, D, device=DEV, dtype=_DTYPES[dt]),
                "lse": torch.empty(rows, h, device=DEV), "dq": dq, "dk": dk, "dv": dv}
    if kind == "norm":
        rows, cap, c = case["rows"], case["cap"], case["C"]
        x = _randn(gen, dt, cap, c, times=2.0) + 0.5
        return {"case": case, "x": x, "dy": _randn(gen, dt, cap, c), "gamma": _randn(gen, dt, c, times=0.3) + 1, "rows": rows,
                "res": _randn(gen, dt, cap, c) if case["residual"] else None, "rows_dev": torch.tensor([rows], dtype=torch.int32, device=DEV),
                "dx": torch.zeros_like(x), "dgamma": torch.empty(c, device=DEV), "dbeta": torch.empty(c, device=DEV), "workspace": None}
    grads = [_randn(gen, case["src"], *size, times=0.02 * (1 + i % 5) / case["scale"]) for i, size in enumerate(_parameters(case))]
    # the optimiser's gradients lie behind one another in one buffer
    flat = torch.empty(sum(g.numel() for g in grads), dtype=_DTYPES[case["dst"]], device=DEV)
    return {"case": case, "grads": grads, "flat": flat, "outs": [o.view_as(g) for o, g in zip(flat.split([g.numel() for g in grads]), grads)],
            "norm": torch.empty(1, dtype=torch.float64, device=DEV), "plan": None}


def _rope_plain(s):
    case = s["case"]
    rot, pairs = case["rot"], case["rot"] // 2
    # far positions: the angle in 64 bits, brought to one turn
    at = s["coords"][s["index"].long() % s["coords"].shape[0]].double().repeat_interleave(pairs // case["axes"], dim=1)
    turn = at * (s["freqs"] / (2 * math.pi))
    angle = ((turn - torch.round(turn)) * (2 * math.pi)).float()[:, None, :]
    cos, sin = torch.cos(angle) * s["amplitude"], torch.sin(angle) * (-s["amplitude"] if case["inverse"] else s["amplitude"])

    def turned(x):
        y = x.float()
        a, b = (y[..., :pairs], y[..., pairs:rot]) if case["layout"] == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
        u, w = a * cos - b * sin, a * sin + b * cos
        front = torch.cat((u, w), dim=-1) if case["layout"] == "half" else torch.stack((u, w), dim=-1).flatten(-2)
        return torch.cat((front, y[..., rot:]), dim=-1).to(x.dtype)

    return {"q": turned(s["q"]), "k": turned(s["k"])}


def _attn_plain(s):
    b, n, h = s["case"]["B"], s["longest"], s["case"]["H"]
    first = s["cu"][:-1].long()
    there = torch.arange(n, device=DEV)[None, :] < s["lengths"][:, None]
    slot = torch.where(there, first[:, None] + torch.arange(n, device=DEV)[None, :], 0)

    def padded(x):                                             # [B, H, n, D] in 32 bits, zeros behind a sequence
        return (x.float()[slot] * there[:, :, None, None]).permute(0, 2, 1, 3).contiguous()

    def packed(x):
        return x.permute(0, 2, 1, 3)[there]

    q, k, v, do = padded(s["q"]), padded(s["k"]), padded(s["v"]), padded(s["do"])
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * s["scale"]
    score = score.masked_fill(~there[:, None, None, :], -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(dim=-1, keepdim=True)
    p = p / total
    o = torch.matmul(p, v)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = p * (dp - (do * o).sum(dim=-1, keepdim=True)) * s["scale"]
    rows_there = there[:, None, :, None]
    ds, p = ds * rows_there, p * rows_there
    dt = s["q"].dtype
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1)[there]
    return {"o": packed(o).to(dt), "lse": lse, "dq": packed(torch.matmul(ds, k)).to(dt),
            "dk": packed(torch.matmul(ds.transpose(-1, -2).contiguous(), q)).to(dt),
            "dv": packed(torch.matmul(p.transpose(-1, -2).contiguous(), do)).to(dt)}


def _norm_plain(s):
    n = s["rows"]
    x, dy, gamma = s["x"][:n].float(), s["dy"][:n].float(), s["gamma"].float()
    centred = x - x.mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt((centred * centred).mean(dim=1, keepdim=True) + EPS)
    xh, w = centred * rstd, dy * gamma
    dx = rstd * (w - w.mean(dim=1, keepdim=True) - xh * (w * xh).mean(dim=1, keepdim=True))
    if s["res"] is not None:
        dx = dx + s["res"][:n].float()
    return {"dx": dx.to(s["x"].dtype), "dgamma": (dy * xh).sum(dim=0), "dbeta": dy.sum(dim=0)}


def _clip_plain(s):
    case = s["case"]
    scale, dst = case["scale"], _DTYPES[case["dst"]]
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt() * abs(scale)
    factor = (torch.where(torch.isfinite(norm), torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0), torch.ones_like(norm)) * scale).float()
    return {"norm": norm.reshape(1), "flat": torch.cat([(g.float() * factor).to(dst).reshape(-1) for g in s["grads"]])}


def run(s):
    case = s["case"]
    if not own:
        return {"rope": _rope_plain, "attn": _attn_plain, "norm": _norm_plain, "clip": _clip_plain}[case["kind"]](s)
    from paper_2604_15408_amd import binding
    if case["kind"] == "rope":
        binding.ragged_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["coords"], s["freqs"], index=s["index"], layout=case["layout"],
                            amplitude=s["amplitude"], inverse=case["inverse"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if case["kind"] == "attn":
        # the host knows the tokens of an unpruned image, not what is left of it
        binding.ragged_attn_lse(s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu"], case["N"], s["scale"])
        binding.ragged_attn_backward(s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["dq"], s["dk"], s["dv"], s["cu"], case["N"], s["scale"])
        return {"o": s["o"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if case["kind"] == "norm":
        if s["workspace"] is None:                             # kept by the program, like every buffer of its step
            s["workspace"] = torch.empty(binding.layernorm_backward_workspace(case["cap"], case["C"]), dtype=torch.uint8, device=DEV)
        binding.ragged_layernorm_backward(s["x"], s["gamma"], s["dy"], s["dx"], s["dgamma"], s["dbeta"], s["workspace"], residual_grad=s["res"],
                                          rows_dev=s["rows_dev"], eps=EPS)
        return {"dx": s["dx"][:s["rows"]], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if s["plan"] is None:                                      # made once for the tensors of a model
        s["plan"] = binding.GradPlan(s["grads"], s["outs"])
    binding.ragged_grad_clip(s["plan"], s["norm"], case["max_norm"], scale=case["scale"])
    return {"norm": s["norm"], "flat": s["flat"]}


def work(case):
    kind = case["kind"]
    if kind == "rope":
        values = _rows(case) * (case["Hq"] + case["Hk"])
        return {"bytes": 4 * values * case["D"] + 4 * _rows(case) * (1 + case["axes"]), "flops": 3 * values * case["rot"]}
    if kind == "attn":
        n, c = case["N"], case["H"] * D
        rows, spread = _rows(case), case["B"] * (n - 1) * case["keep"] * (1 - case["keep"])
        squares = rows * rows / case["B"] + spread
        # q, k, v and the output's gradient in; o, the row statistics and three gradients out; 2 + 5 products
        return {"bytes": 8 * rows * c * 2 + 4 * rows * case["H"], "flops": 14 * squares * c}
    if kind == "norm":
        return {"bytes": case["rows"] * case["C"] * 2 * (4 if case["residual"] else 3) + case["C"] * 10, "flops": 14 * case["rows"] * case["C"]}
    values = sum(math.prod(size) for size in _parameters(case))
    return {"bytes": values * (_DTYPES[case["src"]].itemsize + _DTYPES[case["dst"]].itemsize), "flops": 3 * values}


def exact(case, seed):
    """The definitions in 64 bits: rotations as complex products, gradients by differentiation, sequences one by one."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        rot, per = case["rot"], case["rot"] // 2 // case["axes"]
        at = s["coords"].double()[s["index"].long() % s["coords"].shape[0]]
        angle = torch.cat([at[:, a:a + 1] * s["freqs"][a * per:(a + 1) * per] for a in range(case["axes"])], dim=1)
        unit = torch.polar(torch.full_like(angle, s["amplitude"]), -angle if case["inverse"] else angle)[:, None, :]
        out = {}
        for name in ("q", "k"):
            x = s[name].double()
            y = x.clone()
            first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * unit
            y[..., first], y[..., second] = z.real, z.imag
            out[name] = y
        return out
    if kind == "attn":
        parts = {"o": [], "lse": [], "dq": [], "dk": [], "dv": []}
        ends = s["cu"].tolist()
        for lo, hi in zip(ends[:-1], ends[1:]):
            q, k, v = (s[t][lo:hi].double().transpose(0, 1).contiguous().requires_grad_() for t in ("q", "k", "v"))
            score = s["scale"] * (q @ k.transpose(1, 2).contiguous())
            lse = torch.logsumexp(score, dim=-1)
            o = torch.exp(score - lse[..., None]) @ v
            grads = torch.autograd.grad(o, (q, k, v), s["do"][lo:hi].double().transpose(0, 1).contiguous())
            for name, t in zip(("o", "dq", "dk", "dv"), (o.detach(), *grads)):
                parts[name].append(t.transpose(0, 1))
            parts["lse"].append(lse.detach().transpose(0, 1))
        return {name: torch.cat(p) for name, p in parts.items()}
    if kind == "norm":
        n = s["rows"]
        x, gamma = s["x"][:n].double().requires_grad_(), s["gamma"].double().requires_grad_()
        beta = torch.zeros_like(gamma).requires_grad_()
        y = (x - x.mean(1, keepdim=True)) * (x.var(1, unbiased=False, keepdim=True) + EPS).rsqrt() * gamma + beta
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dy"][:n].double())
        return {"dx": dx if s["res"] is None else dx + s["res"][:n].double(), "dgamma": dgamma, "dbeta": dbeta}
    norm = abs(case["scale"]) * math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
    factor = case["scale"] * min(1.0, case["max_norm"] / (norm + 1e-6))
    return {"norm": torch.tensor([norm], dtype=torch.float64), "flat": torch.cat([g.double().reshape(-1) * factor for g in s["grads"]])}
