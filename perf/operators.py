"""Four operators of an attention module's training step, as cases to be timed
through the Python entry points, each beside its plain form:

  bias   relpos_bias_fwd: the learned relative position bias of the attention
         logits, one value per head and bucket of the position difference,
         added to a pair bias where there is one
  grad   relpos_bias_bwd: the gradient of that table from the attention
         backward's dbias
  ortho  orthogonalize: the Newton-Schulz orthogonalisation of a matrix or of a
         stack of matrices
  muon   FusedMuonSWA.step: momentum, orthogonalised update, weight decay and
         the weight average, over all matrices of a module or of a model

`own` selects what `run` calls: the library (True) or the plain form in
elementary torch operations (False).
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_COEFS = (3.4445, -4.7750, 2.0315)
_STEPS = 5
_EPS = 1e-7
_LR, _MOMENTUM, _DECAY, _SWA = 0.02, 0.95, 0.01, 0.999

# matrices of one MSA row attention module: q, k, v, gate and output weights, and the pair bias's
_MODULE = "5x256x256,1x8x128"
# ragged ones: embedders, heads and the structure module of an AlphaFold-sized model, and a few of odd sizes
_RAGGED = "1x23x256,1x50x128,1x128x65,1x256x49,2x128x22,1x518x384,1x384x1152,2x37x101,1x1x300,1x259x7"
# every matrix of an AlphaFold-sized model: count x rows x columns
_MODEL = ("4x4x64,104x4x128,52x8x128,1x23x256,8x32x64,96x32x256,1x50x128,1x64x25,4x64x64,9x64x128,14x64x256,"
          "1x128x15,2x128x22,1x128x39,32x128x64,1x128x65,1144x128x128,1x128x384,52x128x512,52x128x1024,1x256x39,"
          "1x256x49,38x256x64,481x256x256,48x256x1024,1x384x256,10x384x384,1x384x1152,52x512x128,1x518x384,"
          "48x1024x256,1x1152x384")


def _bias(batch, heads, rows, cols, scheme, reach, chains=1, base=False, dtype="bf16"):
    return {"kind": "bias", "batch": batch, "heads": heads, "rows": rows, "cols": cols, "scheme": scheme,
            "reach": reach, "chains": chains, "base": base, "dtype": dtype}


def _grad(batch, heads, rows, cols, scheme, reach, chains=1):
    return {"kind": "grad", "batch": batch, "heads": heads, "rows": rows, "cols": cols, "scheme": scheme,
            "reach": reach, "chains": chains}


def _ortho(count, rows, cols, dtype):
    return {"kind": "ortho", "count": count, "rows": rows, "cols": cols, "dtype": dtype}


def _muon(shapes):
    return {"kind": "muon", "shapes": shapes}


def listed():
    return [
        # one new token against a long cache of keys, buckets growing with the distance
        dict(_bias(8, 8, 1, 4097, "log", 16), name="bias_token"),
        # MSA row attention at the 256-residue crop: offsets clipped at 32, added to the pair bias
        dict(_bias(1, 8, 256, 256, "clip", 32, base=True), name="bias_crop"),
        # two complexes of four chains in fp32, one bias plane each, added to the pair bias
        dict(_bias(2, 4, 250, 250, "clip", 32, chains=4, base=True, dtype="f32"), name="bias_chains_f32"),
        # a long sequence of odd length, many heads
        dict(_bias(1, 16, 2049, 2049, "log", 64), name="bias_long"),
        # the table's gradient at the 256-residue crop
        dict(_grad(1, 8, 256, 256, "clip", 32), name="grad_crop"),
        # two complexes of three chains, odd length
        dict(_grad(2, 4, 383, 383, "clip", 32, chains=3), name="grad_chains"),
        # a long sequence, many buckets
        dict(_grad(1, 16, 2048, 2048, "log", 128), name="grad_long"),
        # one attention projection
        dict(_ortho(1, 128, 128, "bf16"), name="ortho_one"),
        # the first weight of every pair transition of an AlphaFold-sized model
        dict(_ortho(52, 512, 128, "f32"), name="ortho_transitions"),
        # one large matrix
        dict(_ortho(1, 2048, 2048, "bf16"), name="ortho_large"),
        # ragged matrices in one step
        dict(_muon(_RAGGED + "," + _MODULE), name="muon_ragged"),
        # every matrix of an AlphaFold-sized model in one step
        dict(_muon(_MODEL), name="muon_model"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["bias", "bias", "grad", "grad", "ortho", "ortho", "muon"])
    if kind in ("bias", "grad"):
        heads = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
        scheme = rng.choice(["clip", "log"])
        reach = _log_int(rng, 4, 128)
        chains = rng.choice([1, 1, 2, 3, 5])
        cols = _log_int(rng, 16, 2048)
        rows = 1 if kind == "bias" and rng.random() < 0.25 else max(1, cols - rng.choice([0, 0, 0, 1, 7]))
        batch = rng.choice([1, 1, 2, 3]) if rows * cols < (1 << 20) else 1
        if kind == "grad":
            return _grad(batch, heads, rows, cols, scheme, reach, chains)
        return _bias(batch, heads, rows, cols, scheme, reach, chains, rng.random() < 0.5, rng.choice(["bf16", "f32"]))
    if kind == "ortho":
        dtype = rng.choice(["bf16", "f32"])
        most = 2048 if dtype == "bf16" else 512
        rows, cols = _log_int(rng, 8, most), _log_int(rng, 8, most)
        count = max(1, min(rng.choice([1, 1, 3, 16, 48]), (1 << 22) // (rows * cols)))
        return _ortho(count, rows, cols, dtype)
    shapes = ["%dx%dx%d" % (_log_int(rng, 1, 24), _log_int(rng, 2, 600), _log_int(rng, 2, 600))
              for _ in range(rng.randint(2, 8))]
    return _muon(",".join(shapes))


def _groups(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _edges(scheme, reach):
    """Ascending first offsets of every bucket but the lowest."""
    if scheme == "clip":  # one bucket per offset, the ends take all that lies beyond
        return list(range(1 - reach, reach + 1))
    # per direction: single offsets up to half the reach, then widths growing by powers to 16 times the reach
    half = max(1, reach // 2)
    far = sorted({max(half + 1, int(round(half * (32.0 ** (k / max(1, reach - half)))))) for k in range(1, reach - half + 1)})
    side = list(range(1, half + 1)) + far
    return [1 - e for e in reversed(side)] + side


def _positions(gen, batch, n, chains):
    """Residue numbers: ascending with a few gaps, restarting at each chain, and chain numbers."""
    step = 1 + (torch.rand(batch, n, generator=gen, device="cuda") < 0.02).int() * \
        torch.randint(0, 40, (batch, n), generator=gen, device="cuda").int()
    pos = step.cumsum(1)
    cut = torch.rand(batch, n, generator=gen, device="cuda")
    seg = (torch.arange(n, device="cuda").float() / n * chains + 0.5 * (cut[:, :1] - 0.5)).round().clamp(0, chains - 1)
    seg = seg.int()
    first = torch.where(seg[:, 1:] != seg[:, :-1], pos[:, 1:], torch.zeros_like(pos[:, 1:])).cummax(1).values if n > 1 \
        else torch.zeros_like(pos[:, 1:])
    first = torch.cat([torch.zeros_like(pos[:, :1]), first], 1)
    return (pos - first).int().contiguous(), seg.contiguous()


def _matrices(gen, count, m, n, scale):
    """Gradients as training gives them: a few strong directions over noise."""
    k = min(4, m, n)
    strong = torch.randn(count, m, k, generator=gen, device="cuda") @ \
        torch.randn(count, k, n, generator=gen, device="cuda")
    return (torch.randn(count, m, n, generator=gen, device="cuda") + strong).mul_(scale)


def prepare(case, seed):
    gen = _gen(seed)
    s = {"case": case}
    if case["kind"] in ("bias", "grad"):
        b, h, li, lj = case["batch"], case["heads"], case["rows"], case["cols"]
        pos, seg = _positions(gen, b, max(li, lj), case["chains"])
        s["edges"] = torch.tensor(_edges(case["scheme"], case["reach"]), dtype=torch.int32, device="cuda")
        s["pos_i"], s["pos_j"] = pos[:, -li:].contiguous(), pos[:, :lj].contiguous()
        many = case["chains"] > 1
        s["seg_i"] = seg[:, -li:].contiguous() if many else None
        s["seg_j"] = seg[:, :lj].contiguous() if many else None
        buckets = s["edges"].numel() + 1 + int(many)
        if case["kind"] == "bias":
            s["table"] = torch.randn(h, buckets, generator=gen, device="cuda")
            s["base"] = torch.randn(b, h, li, lj, generator=gen, device="cuda").to(_DT[case["dtype"]]) \
                if case["base"] else None
        else:
            s["dbias"] = torch.randn(b, h, li, lj, generator=gen, device="cuda") * 0.01
    elif case["kind"] == "ortho":
        s["x"] = _matrices(gen, case["count"], case["rows"], case["cols"], 1e-3).to(_DT[case["dtype"]])
    else:
        # the parameters of one kind follow each other in one flat buffer, as the program keeps them
        flat = lambda scale: torch.cat([_matrices(gen, c, m, n, scale).reshape(-1) for c, m, n in _groups(case)])
        s["grad"], s["momentum"] = flat(1e-3), flat(1e-4)
        s["param"] = torch.randn(s["grad"].numel(), generator=gen, device="cuda") * 0.02
        s["swa"] = s["param"] + 1e-4 * torch.randn(s["grad"].numel(), generator=gen, device="cuda")
    return s


def _views(case, flat):
    """The flat buffer as one [count, rows, columns] view per kind of matrix."""
    groups = _groups(case)
    parts = flat.split([c * m * n for c, m, n in groups])
    return [p.view(c, m, n) for p, (c, m, n) in zip(parts, groups)]


# ---- plain forms

def _bucket(s):
    offset = s["pos_i"].long().unsqueeze(2) - s["pos_j"].long().unsqueeze(1)
    bucket = torch.searchsorted(s["edges"].long(), offset, right=True)
    if s["seg_i"] is None:
        return bucket
    return torch.where(s["seg_i"].unsqueeze(2) == s["seg_j"].unsqueeze(1), bucket, s["edges"].numel() + 1)


def _plain_bias(s):
    out = s["table"][:, _bucket(s)].transpose(0, 1)
    if s["base"] is not None:
        out = out + s["base"].float()
    return out.to(_DT[s["case"]["dtype"]]).contiguous()


def _plain_grad(s):
    buckets = s["edges"].numel() + 1 + int(s["seg_i"] is not None)
    d = s["dbias"].transpose(1, 2)                                           # [B, Li, H, Lj]
    member = (_bucket(s).unsqueeze(3) == torch.arange(buckets, device="cuda")).float()
    return torch.matmul(d, member).double().sum((0, 1)).float()              # sums over j, then over b and i


def _plain_ortho(x):
    x = x.float()
    if x.shape[1] > x.shape[2]:
        return _plain_ortho(x.transpose(1, 2).contiguous()).transpose(1, 2).contiguous()
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt().clamp(min=_EPS)
    x = (x.double() / norm).float()
    for _ in range(_STEPS):
        gram = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = _COEFS[0] * x + torch.bmm(_COEFS[1] * gram + _COEFS[2] * torch.bmm(gram, gram), x)
    return x


def _plain_muon(s):
    s["momentum"].mul_(_MOMENTUM).add_(s["grad"], alpha=1 - _MOMENTUM)
    update = s["grad"] * (1 - _MOMENTUM) + s["momentum"] * _MOMENTUM
    step = torch.cat([(_plain_ortho(v) * math.sqrt(max(1.0, v.shape[1] / v.shape[2]))).reshape(-1)
                      for v in _views(s["case"], update)])
    s["param"].mul_(1 - _LR * _DECAY).sub_(step, alpha=_LR)
    s["swa"].mul_(_SWA).add_(s["param"], alpha=1 - _SWA)
    return {"param": s["param"], "momentum": s["momentum"], "swa": s["swa"]}


# ---- the library's calls

def _own_bias(s):
    from paper_2404_11068_amd import relpos
    return relpos.relpos_bias_fwd(s["pos_i"], s["pos_j"], s["edges"], s["table"], seg_i=s["seg_i"], seg_j=s["seg_j"],
                                  base=s["base"], dtype=_DT[s["case"]["dtype"]])


def _own_grad(s):
    from paper_2404_11068_amd import relpos
    return relpos.relpos_bias_bwd(s["pos_i"], s["pos_j"], s["edges"], s["dbias"], seg_i=s["seg_i"], seg_j=s["seg_j"])


def _own_ortho(s):
    from paper_2404_11068_amd import optim
    return optim.orthogonalize(s["x"], steps=_STEPS, coefs=_COEFS, eps=_EPS)


def _own_muon(s):
    from paper_2404_11068_amd import optim
    if "optimizer" not in s:  # built once, as a program builds its optimizer
        lists = [[m for v in _views(s["case"], s[k]) for m in v.unbind(0)] for k in ("param", "grad", "momentum", "swa")]
        s["optimizer"] = optim.FusedMuonSWA(*lists, lr=_LR, momentum_decay=_MOMENTUM, weight_decay=_DECAY,
                                            swa_decay=_SWA, steps=_STEPS, coefs=_COEFS, eps=_EPS)
    s["optimizer"].step()
    return {"param": s["param"], "momentum": s["momentum"], "swa": s["swa"]}


def run(state):
    kind = state["case"]["kind"]
    if own:
        if kind == "bias":
            return _own_bias(state)
        if kind == "grad":
            return _own_grad(state)
        return _own_ortho(state) if kind == "ortho" else _own_muon(state)
    if kind == "bias":
        return _plain_bias(state)
    if kind == "grad":
        return _plain_grad(state)
    if kind == "ortho":
        return _plain_ortho(state["x"]).to(_DT[state["case"]["dtype"]])
    return _plain_muon(state)


def _newton_schulz_flops(m, n):
    """Per step: the Gram matrix and its square, half of each by symmetry, and the product with the matrix."""
    r, c = min(m, n), max(m, n)
    return _STEPS * (r * r * c + r * r * r + 2 * r * r * c)


def work(case):
    if case["kind"] in ("bias", "grad"):
        b, h, li, lj = case["batch"], case["heads"], case["rows"], case["cols"]
        buckets = len(_edges(case["scheme"], case["reach"])) + 1 + int(case["chains"] > 1)
        index = 4 * b * (li + lj) * (2 if case["chains"] > 1 else 1) + 4 * buckets
        size = 4 if case["kind"] == "grad" or case["dtype"] == "f32" else 2
        each = 2 if case["kind"] == "bias" and case["base"] else 1
        return {"bytes": b * h * li * lj * size * each + 4 * h * buckets + index, "flops": b * h * li * lj * (each - 1)
                if case["kind"] == "bias" else b * h * li * lj}
    if case["kind"] == "ortho":
        n = case["count"] * case["rows"] * case["cols"]
        return {"bytes": 2 * n * (2 if case["dtype"] == "bf16" else 4),
                "flops": case["count"] * _newton_schulz_flops(case["rows"], case["cols"])}
    # read parameter, gradient, momentum and average, write all but the gradient
    return {"bytes": 28 * sum(c * m * n for c, m, n in _groups(case)),
            "flops": sum(c * _newton_schulz_flops(m, n) for c, m, n in _groups(case))}


# ---- from the definitions, in 64 bits

def _exact_ortho(x):
    """Newton-Schulz as what it is, an odd polynomial of the singular values: the gain on X is the product of the
    steps' polynomials of the Gram matrix, which all commute with it."""
    x = x.double()
    if x.shape[1] > x.shape[2]:
        return _exact_ortho(x.transpose(1, 2).contiguous()).transpose(1, 2).contiguous()
    x = x / torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True).clamp(min=_EPS)
    one = torch.eye(x.shape[1], dtype=torch.float64, device=x.device).expand(x.shape[0], -1, -1).contiguous()
    gram, gain = torch.bmm(x, x.transpose(1, 2).contiguous()), one
    for _ in range(_STEPS):
        p = _COEFS[0] * one + _COEFS[1] * gram + _COEFS[2] * torch.bmm(gram, gram)
        gain, gram = torch.bmm(p, gain), torch.bmm(torch.bmm(p, gram), p)
    return torch.bmm(gain, x)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("bias", "grad"):
        d = s["pos_i"].cpu().long()[:, :, None] - s["pos_j"].cpu().long()[:, None, :]
        bucket = torch.zeros_like(d)
        for e in s["edges"].tolist():
            bucket += d >= e
        if s["seg_i"] is not None:
            bucket[s["seg_i"].cpu()[:, :, None] != s["seg_j"].cpu()[:, None, :]] = s["edges"].numel() + 1
        if case["kind"] == "bias":
            out = torch.stack([row.double()[bucket] for row in s["table"].cpu()], 1)
            return out if s["base"] is None else out + s["base"].cpu().double()
        n = s["edges"].numel() + 1 + int(s["seg_i"] is not None)
        return torch.stack([torch.bincount(bucket.reshape(-1), s["dbias"][:, h].cpu().double().reshape(-1), n)
                            for h in range(case["heads"])])
    if case["kind"] == "ortho":
        return _exact_ortho(s["x"])
    g, m, p, w = (s[k].double() for k in ("grad", "momentum", "param", "swa"))
    m = _MOMENTUM * m + (1 - _MOMENTUM) * g
    u = (1 - _MOMENTUM) * g + _MOMENTUM * m
    o = torch.cat([(_exact_ortho(v) * max(1.0, v.shape[1] / v.shape[2]) ** 0.5).reshape(-1) for v in _views(case, u)])
    p = p - _LR * _DECAY * p - _LR * o
    return {"param": p, "momentum": m, "swa": _SWA * w + (1 - _SWA) * p}
