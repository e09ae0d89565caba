"""What the block-scaled 8-bit float path and the fused norms between a block's linears are measured on.

Operators
  quantize   bf16 rows -> e4m3 codes with one fp32 scale per row and 128 channels, on request behind the block rotation
  weights    the same for a weight matrix, one scale per 128 x 128 block
  linear     the product of such codes with its scales, bias and activation
  norm       branch output -> optional norm, gate and residual add -> norm and modulation; output in bf16 or as codes
  backward   the gradients of `norm`

`run` computes them in elementary torch operations, or with `own` set through the library's entry points.  The tensors have the
shapes and the outlier structure of the image and video models of ``workloads.py``: a Gaussian bulk, one channel in a hundred
heavy tailed, weights of standard deviation 0.02.
"""
import math

import torch

own = False

BLOCK = 128
TOP = 448.0            # largest e4m3 number
TINY = 2.0 ** -100     # block maxima below this are scaled as if they were this
EPS = 1e-6


# --------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a single token of a text projection: launch and host time are what is paid for
        {"name": "quantize_1", "op": "quantize", "M": 1, "K": 4096, "rotated": True, "pad": 0},
        # the input of a 1024 px block's linears, both guidance halves
        {"name": "quantize_32768", "op": "quantize", "M": 32768, "K": 1152, "rotated": True, "pad": 0},
        # the widest layer of a block prepared when a model is loaded
        {"name": "weights_4608", "op": "weights", "N": 4608, "K": 1152, "rotated": True},
        # a single token against a wide layer: the weights are streamed once
        {"name": "linear_1", "op": "linear", "M": 1, "K": 4096, "N": 16384, "act": 0, "bias": True, "pad": 0},
        # one layer of a small batch
        {"name": "linear_256", "op": "linear", "M": 256, "K": 1024, "N": 1024, "act": 0, "bias": True, "pad": 0},
        # an odd image size: nothing is a multiple of a tile, GELU behind it, the output inside a wider buffer
        {"name": "linear_2057_gelu", "op": "linear", "M": 2057, "K": 1152, "N": 4624, "act": 1, "bias": True, "pad": 48},
        # the second linear of a 1024 px block
        {"name": "linear_32768", "op": "linear", "M": 32768, "K": 4608, "N": 1152, "act": 0, "bias": True, "pad": 0},
        # one token between two sub-blocks with RMS norms before and after, weights, residual stream in fp32
        {"name": "norm_1_rms", "op": "norm", "M": 1, "D": 4096, "norm": "rms", "post": "rms", "stream": "fp32", "rps": 1,
         "gate": False, "mod": False, "weight": True, "alpha": 1.0, "fp8": False},
        # adaLN: gate, residual, LayerNorm and modulation of 32 samples of 1024 tokens
        {"name": "norm_32768", "op": "norm", "M": 32768, "D": 1152, "norm": "layer", "post": "none", "stream": "bf16", "rps": 1024,
         "gate": True, "mod": True, "weight": False, "alpha": 1.0, "fp8": False},
        # the same, its output rotated and quantized for the next linear, an odd number of tokens per sample
        {"name": "norm_fp8_8190", "op": "norm", "M": 8190, "D": 1152, "norm": "layer", "post": "none", "stream": "bf16", "rps": 273,
         "gate": True, "mod": True, "weight": False, "alpha": 1.0, "fp8": True},
        # gradients of the adaLN form
        {"name": "backward_16384", "op": "backward", "M": 16384, "D": 1152, "norm": "layer", "post": "none", "stream": "bf16", "rps": 256,
         "gate": True, "mod": True, "weight": False, "alpha": 1.0},
        # gradients with RMS norms before and after, weights and an fp32 stream, few rows
        {"name": "backward_517_rms", "op": "backward", "M": 517, "D": 4096, "norm": "rms", "post": "rms", "stream": "fp32", "rps": 517,
         "gate": False, "mod": False, "weight": True, "alpha": 0.5},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "weights", "linear", "linear", "linear", "norm", "norm", "backward"])
    if op == "quantize":
        K = BLOCK * _log_int(rng, 1, 128)                                  # 128 ... 16384
        return {"op": op, "M": min(_log_int(rng, 1, 32768), 32768 * 1152 // K), "K": K, "rotated": rng.random() < 0.7, "pad": 8 * rng.randint(0, 8)}
    if op == "weights":
        return {"op": op, "N": 16 * _log_int(rng, 4, 512), "K": BLOCK * _log_int(rng, 1, 64), "rotated": rng.random() < 0.7}
    if op == "linear":
        K, N = BLOCK * _log_int(rng, 1, 64), 16 * _log_int(rng, 8, 512)    # 128 ... 8192 on both sides
        M = min(_log_int(rng, 1, 32768), 32768 * 4608 * 1152 // (K * N), 32768 * 4608 // max(K, N))
        return {"op": op, "M": max(1, M), "K": K, "N": N, "act": rng.choice([0, 0, 1]), "bias": rng.random() < 0.7, "pad": 8 * rng.randint(0, 8)}
    fp8 = op == "norm" and rng.random() < 0.4
    D = BLOCK * _log_int(rng, 1, 64) if fp8 else 8 * _log_int(rng, 16, 1024)   # 128 ... 8192
    M = max(1, min(_log_int(rng, 1, 32768), (16384 if op == "backward" else 32768) * 1152 // D))
    kind = rng.choice(["ada", "ada", "sandwich", "all"])
    case = {"op": op, "M": M, "D": D, "norm": rng.choice(["layer", "rms"]), "post": "none" if kind == "ada" else rng.choice(["layer", "rms"]),
            "stream": rng.choice(["bf16", "bf16", "fp32"]), "rps": M if kind == "sandwich" else min(M, _log_int(rng, 1, 4096)),
            "gate": kind != "sandwich", "mod": kind != "sandwich", "weight": kind != "ada", "alpha": rng.choice([1.0, 1.0, 0.5])}
    # per-token modulation of everything is M * D parameters three times over: samples of at least 16 tokens above that
    if M // case["rps"] > 512:
        case["rps"] = max(case["rps"], 16)
    if op == "norm":
        case["fp8"] = fp8
    return case


# ------------------------------------------------------------------------------------------------------------ inputs
class _Inputs:
    """Tensors drawn on the device from one seed."""

    def __init__(self, seed):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(int(seed))

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda", dtype=torch.float32)

    def activations(self, M, K, pad=0):
        """[M, K] with row stride K + pad: N(0, 1), one channel in a hundred Student-t with three degrees of freedom."""
        x = self.randn(M, K + pad)
        n = max(1, K // 100)
        ch = torch.randperm(K, generator=self.gen, device="cuda")[:n]
        x[:, ch] = self.randn(M, n) / torch.sqrt((self.randn(M, n, 3) ** 2).sum(-1) / 3.0)
        return x.to(torch.bfloat16)[:, :K]

    def weight(self, N, K):
        return (self.randn(N, K) * 0.02).to(torch.bfloat16)

    def rotation(self, K, side):
        """The +-1 diagonal and the smoothing factors of one time-step group, as a program holds them: the fused fp32 vector of the plain
        form, and the library's handle where it is used."""
        signs = torch.where(self.randn(K) < 0, -1.0, 1.0).double()
        smooth = torch.exp(0.3 * self.randn(K))
        d = smooth.double()
        vec = (signs * (d if side == "act" else 1.0 / d) * 2.0 ** -3.5).float()
        return {"signs": signs.cpu().numpy().astype("int8"), "smooth": smooth.cpu().numpy(), "vec": vec, "rot": None}


def _handle(r):
    if own and r is not None:
        from paper_2503_06564_b200 import trdq
        K = len(r["signs"])
        r["rot"] = trdq.Rotation(K, [0, 1000], r["signs"].reshape(1, K), r["smooth"].reshape(1, K))
    return r


def _samples(case):
    return -(-case["M"] // case["rps"])


def prepare(case, seed):
    i = _Inputs(seed)
    s = {"case": case}
    if case["op"] == "quantize":
        s["x"] = i.activations(case["M"], case["K"], case["pad"])
        s["r"] = _handle(i.rotation(case["K"], "act") if case["rotated"] else None)
    elif case["op"] == "weights":
        s["w"] = i.weight(case["N"], case["K"])
        s["r"] = _handle(i.rotation(case["K"], "weight") if case["rotated"] else None)
    elif case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        s["q"], s["sx"] = _plain_codes(i.activations(M, K).float())
        s["qw"], s["sw"] = _plain_weight_codes(i.weight(N, K).float())
        s["bias"] = (i.randn(N) * 0.5).to(torch.bfloat16) if case["bias"] else None
        s["out"] = torch.empty((M, N + case["pad"]), dtype=torch.bfloat16, device="cuda")[:, :N]
    else:
        M, D, S = case["M"], case["D"], _samples(case)
        stream = torch.float32 if case["stream"] == "fp32" else torch.bfloat16
        s["x"] = (2.0 * i.activations(M, D).float()).to(stream)
        s["b"] = i.activations(M, D)
        # the modulation of a block comes out of one linear: shift, scale and gate are column ranges of its output
        mod = (0.3 * i.randn(S, 3 * D)).to(torch.bfloat16) if case["gate"] or case["mod"] else None
        s["shift"], s["scale"] = (mod[:, :D], mod[:, D:2 * D]) if case["mod"] else (None, None)
        s["gate"] = mod[:, 2 * D:] if case["gate"] else None
        s["weight"] = (1.0 + 0.1 * i.randn(D)).to(torch.bfloat16) if case["weight"] else None
        s["post_weight"] = (1.0 + 0.1 * i.randn(D)).to(torch.bfloat16) if case["weight"] and case["post"] != "none" else None
        if case["op"] == "backward":
            s["dh"] = i.randn(M, D).to(torch.bfloat16)
            s["dr"] = i.randn(M, D).to(stream)
        elif case["fp8"]:
            s["r"] = _handle(i.rotation(D, "act"))
    return s


# -------------------------------------------------------------------------------------------------------- plain forms
def _butterfly(v, h):
    a = v.view(v.shape[0], -1, 2, h)
    return torch.stack((a[:, :, 0] + a[:, :, 1], a[:, :, 0] - a[:, :, 1]), 2).reshape(v.shape)


def _rotate(v, vec):
    """(v o vec) BlockDiag(H_128), the butterfly stages one after the other."""
    v = v * vec
    v = _butterfly(_butterfly(_butterfly(v, 1), 2), 4)
    return _butterfly(_butterfly(_butterfly(_butterfly(v, 8), 16), 32), 64)


def _plain_codes(v):
    """fp32 [M, K] -> e4m3 codes [M, K], fp32 scales [K / 128, M]."""
    b = v.view(v.shape[0], -1, BLOCK)
    top = b.abs().amax(2)
    floor = top.clamp_min(TINY)
    codes = (b * (TOP / floor).unsqueeze(2)).to(torch.float8_e4m3fn).view(v.shape)
    return codes, torch.where(top > 0, floor / TOP, 0.0).t().contiguous()


def _plain_weight_codes(v):
    """fp32 [N, K] -> e4m3 codes [N, K], fp32 scales [ceil(N / 128), K / 128]."""
    N, K = v.shape
    nb = -(-N // BLOCK)
    p = torch.zeros((nb * BLOCK, K), dtype=torch.float32, device=v.device)
    p[:N] = v
    p = p.view(nb, BLOCK, K // BLOCK, BLOCK)
    top = p.abs().amax((1, 3))
    floor = top.clamp_min(TINY)
    codes = (p * (TOP / floor)[:, None, :, None]).to(torch.float8_e4m3fn).view(nb * BLOCK, K)
    return codes[:N], torch.where(top > 0, floor / TOP, 0.0)


def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(0.7978845608028654 * (x + 0.044715 * x * x * x)))


def _plain_linear(s):
    q, sx, qw, sw = s["q"], s["sx"], s["qw"], s["sw"]
    a = q.float() * sx.t().repeat_interleave(BLOCK, 1)
    w = qw.float() * sw.repeat_interleave(BLOCK, 0)[: qw.shape[0]].repeat_interleave(BLOCK, 1)
    y = a @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if s["case"]["act"]:
        y = _gelu(y)
    s["out"].copy_(y)
    return s["out"]


def _normalised(v, kind):
    """(v - mean) / sqrt(var + eps), or v / sqrt(mean square + eps); and the factor."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    f = torch.rsqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * f, f


def _per_row(p, case):
    return p.float().repeat_interleave(case["rps"], 0)[: case["M"]]


def _per_sample(g, case):
    """Sums over the rows of each sample."""
    M, rps, S = case["M"], case["rps"], _samples(case)
    if S * rps != M:
        g = torch.cat((g, torch.zeros((S * rps - M, g.shape[1]), dtype=g.dtype, device=g.device)))
    return g.view(S, rps, -1).sum(1)


def _plain_norm(s):
    case = s["case"]
    u = s["b"].float()
    if case["post"] != "none":
        u = _normalised(u, case["post"])[0]
    if s["post_weight"] is not None:
        u = u * s["post_weight"].float()
    if case["gate"]:
        u = u * _per_row(s["gate"], case)
    r = (case["alpha"] * s["x"].float() + u).to(s["x"].dtype)
    h = _normalised(r.float(), case["norm"])[0]
    if s["weight"] is not None:
        h = h * s["weight"].float()
    if case["mod"]:
        h = h * (1.0 + _per_row(s["scale"], case)) + _per_row(s["shift"], case)
    if not case["fp8"]:
        return {"r": r, "h": h.to(torch.bfloat16)}
    codes, scales = _plain_codes(_rotate(h, s["r"]["vec"]))
    return {"r": r, "codes": codes, "scales": scales}


def _norm_gradient(dn, n, f, kind):
    g = dn - n * (dn * n).mean(1, keepdim=True)
    if kind == "layer":
        g = g - dn.mean(1, keepdim=True)
    return g * f


def _plain_backward(s):
    """s["x"] stands for the stored sum r."""
    case = s["case"]
    n, f = _normalised(s["x"].float(), case["norm"])
    dh = s["dh"].float()
    out = {}
    dn = dh
    hw = n
    if s["weight"] is not None:
        hw = n * s["weight"].float()
    if case["mod"]:
        out["dshift"] = _per_sample(dh, case)
        out["dscale"] = _per_sample(dh * hw, case)
        dn = dn * (1.0 + _per_row(s["scale"], case))
    if s["weight"] is not None:
        out["dweight"] = (dn * n).sum(0)
        dn = dn * s["weight"].float()
    dr = s["dr"].float() + _norm_gradient(dn, n, f, case["norm"])
    out["dx"] = (case["alpha"] * dr).to(s["x"].dtype)
    m, fp = (s["b"].float(), None) if case["post"] == "none" else _normalised(s["b"].float(), case["post"])
    du = dr
    if case["gate"]:
        out["dgate"] = _per_sample(dr * (m if s["post_weight"] is None else m * s["post_weight"].float()), case)
        du = du * _per_row(s["gate"], case)
    if s["post_weight"] is not None:
        out["dpost_weight"] = (du * m).sum(0)
        du = du * s["post_weight"].float()
    if case["post"] != "none":
        du = _norm_gradient(du, m, fp, case["post"])
    out["db"] = du.to(torch.bfloat16)
    return out


def _plain(s):
    op = s["case"]["op"]
    if op == "quantize":
        x = s["x"].float()
        codes, scales = _plain_codes(x if s["r"] is None else _rotate(x, s["r"]["vec"]))
        return {"codes": codes, "scales": scales}
    if op == "weights":
        w = s["w"].float()
        codes, scales = _plain_weight_codes(w if s["r"] is None else _rotate(w, s["r"]["vec"]))
        return {"codes": codes, "scales": scales}
    if op == "linear":
        return {"y": _plain_linear(s)}
    return _plain_norm(s) if op == "norm" else _plain_backward(s)


# ---------------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    from paper_2503_06564_b200 import trdq
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        codes, scales = trdq.trdq_fp8_quantize(s["x"], None if s["r"] is None else s["r"]["rot"], 0)
        return {"codes": codes, "scales": scales}
    if op == "weights":
        codes, scales = trdq.trdq_fp8_quantize_weights(s["w"], None if s["r"] is None else s["r"]["rot"], 0)
        return {"codes": codes, "scales": scales}
    if op == "linear":
        return {"y": trdq.trdq_fp8_linear(s["q"], s["sx"], s["qw"], s["sw"], s["bias"], s["out"], case["act"])}
    kinds = {"none": trdq.NORM_NONE, "layer": trdq.NORM_LAYER, "rms": trdq.NORM_RMS}
    given = dict(gate=s["gate"], shift=s["shift"], scale=s["scale"], weight=s["weight"], post_weight=s["post_weight"],
                 norm=kinds[case["norm"]], post_norm=kinds[case["post"]], rows_per_sample=case["rps"], eps=EPS, res_scale=case["alpha"])
    if op == "backward":
        g = trdq.trdq_gated_norm_backward(s["x"], s["b"], s["dh"], s["dr"], **given)
        return {k: v for k, v in g.items() if v is not None}
    if case["fp8"]:
        r, codes, scales = trdq.trdq_gated_norm_fp8(s["r"]["rot"], 0, s["x"], s["b"], **given)
        return {"r": r, "codes": codes, "scales": scales}
    r, h = trdq.trdq_gated_norm(s["x"], s["b"], **given)
    return {"r": r, "h": h}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def _hadamard():
    """Entry (i, j) is -1 to the number of bits that i and j share."""
    n = torch.arange(BLOCK, device="cuda")
    both = n[:, None] & n[None, :]
    bits = sum((both >> k) & 1 for k in range(7))
    return (1 - 2 * (bits & 1)).double()


def _exact_rotated(v, r):
    if r is None:
        return v
    blocks = (v * r["vec"].double()).reshape(v.shape[0], -1, BLOCK)
    return (blocks @ _hadamard()).reshape(v.shape)


def _nearest_e4m3(v):
    """The nearest e4m3 number, ties to the even code: 4 significant bits, spacing at least 2^-9."""
    _, e = torch.frexp(v)
    step = torch.exp2((e - 4).clamp_min(-9).double())
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _exact_norm(v, kind):
    c = v - v.mean(1, keepdim=True) if kind == "layer" else v
    return c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)


def _exact_forward(case, p, r=None):
    """(r, h) in double from the double inputs p; `r` given: h from it."""
    rows = torch.arange(case["M"], device="cuda") // case["rps"]
    if r is None:
        u = p["b"] if case["post"] == "none" else _exact_norm(p["b"], case["post"])
        u = u * p["post_weight"] if p["post_weight"] is not None else u
        u = u * p["gate"][rows] if p["gate"] is not None else u
        r = case["alpha"] * p["x"] + u
    h = lambda r: _exact_norm(r, case["norm"]) * (1.0 if p["weight"] is None else p["weight"])  # noqa: E731
    m = lambda h: h if p["scale"] is None else h * (1.0 + p["scale"][rows]) + p["shift"][rows]  # noqa: E731
    return r, lambda r: m(h(r))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        v = _exact_rotated(s["x"].double(), s["r"]).view(case["M"], -1, BLOCK)
        scale = v.abs().amax(2) / TOP
        return {"codes": _nearest_e4m3(v / scale.unsqueeze(2)).view(case["M"], -1), "scales": scale.t().contiguous()}
    if op == "weights":
        N, K = case["N"], case["K"]
        v = _exact_rotated(s["w"].double(), s["r"])
        scale = torch.stack([b.reshape(b.shape[0], -1, BLOCK).abs().amax((0, 2)) for b in v.split(BLOCK)]) / TOP
        each = scale[torch.arange(N, device="cuda") // BLOCK].unsqueeze(2)
        return {"codes": _nearest_e4m3(v.view(N, -1, BLOCK) / each).view(N, K), "scales": scale}
    if op == "linear":
        rows = torch.arange(case["N"], device="cuda") // BLOCK
        a = (s["q"].double().view(case["M"], -1, BLOCK) * s["sx"].double().t().unsqueeze(2)).view(case["M"], -1)
        w = (s["qw"].double().view(case["N"], -1, BLOCK) * s["sw"].double()[rows].unsqueeze(2)).view(case["N"], -1)
        y = torch.matmul(a, w.t())
        y = y if s["bias"] is None else y + s["bias"].double()
        if case["act"]:
            y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
        return {"y": y}
    names = ("x", "b", "gate", "shift", "scale", "weight", "post_weight")
    p = {k: None if s[k] is None else s[k].double() for k in names}
    if op == "norm":
        r, h = _exact_forward(case, p)
        h = h(r.to(s["x"].dtype).double())
        if not case["fp8"]:
            return {"r": r, "h": h}
        scale = _exact_rotated(h, s["r"]).view(case["M"], -1, BLOCK).abs().amax(2) / TOP
        # a code next to a border between two of them depends on the last bits of the row's statistics: no value for it
        return {"r": r, "codes": None, "scales": scale.t().contiguous()}
    # gradients by differentiating the definition; the stored sum stands where alpha x + gate u stood
    leaf = {k: None if v is None else v.requires_grad_() for k, v in p.items()}
    stored = leaf["x"]
    zero = dict(leaf, x=torch.zeros_like(stored).requires_grad_())
    r, h = _exact_forward(case, zero)
    r = r + (stored - r).detach()
    loss = (h(r) * s["dh"].double()).sum() + (r * s["dr"].double()).sum()
    want = {"dx": zero["x"], "db": leaf["b"], "dgate": leaf["gate"], "dshift": leaf["shift"], "dscale": leaf["scale"],
            "dweight": leaf["weight"], "dpost_weight": leaf["post_weight"]}
    want = {k: v for k, v in want.items() if v is not None}
    return dict(zip(want, torch.autograd.grad(loss, list(want.values()))))


# ------------------------------------------------------------------------------------------------------------- the work
def work(case):
    if case["op"] == "quantize":
        M, K = case["M"], case["K"]
        return {"bytes": 3 * M * K + 4 * M * K // BLOCK + (4 * K if case["rotated"] else 0), "flops": (8 if case["rotated"] else 1) * M * K}
    if case["op"] == "weights":
        N, K = case["N"], case["K"]
        return {"bytes": 3 * N * K + 4 * -(-N // BLOCK) * K // BLOCK + (4 * K if case["rotated"] else 0), "flops": (8 if case["rotated"] else 1) * N * K}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        scales = 4 * (M + -(-N // BLOCK)) * K // BLOCK
        return {"bytes": M * K + N * K + 2 * M * N + scales + (2 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    M, D, S = case["M"], case["D"], _samples(case)
    stream = 4 if case["stream"] == "fp32" else 2
    params = S * D * ((1 if case["gate"] else 0) + (2 if case["mod"] else 0))
    weights = D * ((1 if case["weight"] else 0) + (1 if case["weight"] and case["post"] != "none" else 0))
    if case["op"] == "backward":
        grads = 4 * (params + weights)
        read = 2 * params + 2 * weights - (2 * S * D if case["mod"] else 0)   # the shift itself is not needed
        return {"bytes": M * D * (3 * stream + 6) + read + grads, "flops": 25 * M * D}
    out = M * D + 4 * M * D // BLOCK + 4 * D if case["fp8"] else 2 * M * D
    return {"bytes": M * D * (2 * stream + 2) + out + 2 * params + 2 * weights, "flops": (20 if case["fp8"] else 12) * M * D}
