"""A worker's operators around a push, as cases that can be timed and compared:
scaled embedding lookups, their gradient by sorted tokens (as a message's rows
or as a dense array), the global norm of many gradients and clipping by it, and
layer norm in both directions.

A case is a dict of plain values:
  op        "embed", "grad" (ids and summed rows of a message, in n slots),
            "grad_dense" (an array of all rows), "norm", "clip", "ln" or "ln_grad"
  n, d      tokens (rows) and width
  V, zipf   rows of the table, and the exponent of the ids' popularity law
  modulo    64-bit hashed ids folded into the rows instead of row numbers
  pad       share of the positions that hold the padding id (ragged batches);
            what the gradient holds there is never to be used
  type, out_type            "f32", "bf16" or "f16", of the input (weights,
            gradients, x) and of the output
  extra     columns between the rows of the input that do not belong to it
  parts, total              tensors of a norm and their elements together
  pack      the clipped gradients go to one flat float32 array (the dense
            gradient of a message) instead of tensors of their own type
  param     type of layer norm's weight and bias
"""
import math
import random

import torch

own = False

MAX_NORM = 1.0
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

TOKENS = dict(V=32_768, zipf=1.05, modulo=False, pad=0.0, type="bf16", out_type="bf16", extra=0)
NORMS = dict(type="f32", out_type="f32", pack=False)
LAYER = dict(type="bf16", param="f32", extra=0)


def listed():
    return [
        # one new token for each of 64 sequences: the time is the call's and the launch's
        dict(TOKENS, name="embed-tokens-64x1024", op="embed", n=64, d=1024),
        # a batch of prompts, from float32 weights as the server keeps them to 16-bit activations
        dict(TOKENS, name="embed-prompts-131072x1024", op="embed", n=131_072, d=1024, V=131_072,
             type="f32", pad=0.1),
        # one worker's message of a small model: 256 samples of 26 one-hot fields
        dict(TOKENS, name="grad-message-6656x16", op="grad", n=6_656, d=16, V=100_000, zipf=1.1,
             type="f32", out_type="f32"),
        # one worker's message of a large one: 1,024 samples of 40 fields
        dict(TOKENS, name="grad-message-40960x64", op="grad", n=40_960, d=64, V=1_000_000,
             type="f32", out_type="f32", pad=0.05),
        # the embedding gradient of a long step over tokens, all rows of the table
        dict(TOKENS, name="grad-dense-262144x2048", op="grad_dense", n=262_144, d=2048, V=131_072,
             out_type="f32", pad=0.02),
        # the norm of a small message: its rows and the dense gradient's tensors
        dict(NORMS, name="norm-message-306k", op="norm", parts=7, total=306_496),
        # the same message clipped before its push
        dict(NORMS, name="clip-message-306k", op="clip", parts=7, total=306_496),
        # a large dense network's 16-bit gradients, clipped into the message's float32 array
        dict(NORMS, name="clip-pack-64M", op="clip", parts=148, total=64_000_000, type="bf16", pack=True),
        # single tokens of 16 sequences
        dict(LAYER, name="ln-16x1024", op="ln", n=16, d=1024),
        # a long batch
        dict(LAYER, name="ln-32768x4096", op="ln", n=32_768, d=4096),
        # an odd width, in float32
        dict(LAYER, name="ln-grad-5003x1001-f32", op="ln_grad", n=5_003, d=1_001, type="f32"),
        # a long batch, backwards
        dict(LAYER, name="ln-grad-32768x2048", op="ln_grad", n=32_768, d=2048, param="bf16"),
    ]


def _between(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v - 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(["embed", "grad", "grad_dense", "norm", "clip", "ln", "ln_grad"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("norm", "clip"):
        pack = op == "clip" and rng.random() < 0.5
        most = 200 if pack or op == "norm" else 48
        total = _between(rng, 1_000, 100_000_000)
        return dict(NORMS, op=op, parts=min(_between(rng, 1, most), total), total=total, type=kind,
                    out_type=kind, pack=pack)
    d = _between(rng, 8, 4096)
    if rng.random() < 0.6:  # most widths are multiples of eight, the others as they come
        d = max(8, d // 8 * 8)
        d = d + 8 if d == 3072 else d
    n = _between(rng, 1, min(262_144, (1 << 26) // d))
    extra = rng.choice([0, 0, 0, 8, 3])
    if op in ("ln", "ln_grad"):
        return dict(LAYER, op=op, n=n, d=d, type=kind, param=rng.choice(["f32", kind]), extra=extra)
    V = _between(rng, 100, min(1_000_000, (1 << 27) // d))
    out = "f32" if op != "embed" else rng.choice(["f32", kind])
    return dict(TOKENS, op=op, n=n, d=d, V=V, zipf=rng.choice([1.05, 1.1, 1.2]), modulo=rng.random() < 0.3,
                pad=rng.choice([0.0, 0.0, 0.05, 0.5]), type=kind, out_type=out, extra=extra)


# ---- inputs ---------------------------------------------------------------------------

def _part_sizes(case):
    """A few matrices and many small vectors, of ragged sizes that sum to the total."""
    r = random.Random(case["parts"])
    share = [math.exp(r.uniform(0.0, 7.0)) for _ in range(case["parts"])]
    left = case["total"] - case["parts"]
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[0] += case["total"] - sum(sizes)
    return sizes


def _popularity(case):
    p = torch.arange(1, case["V"] + 1, dtype=torch.float64).pow(-case["zipf"])
    return p / p.sum()


def _rows(g, n, d, dtype, extra, mean=0.0, std=1.0):
    """n rows of d values, `extra` columns of something else between them."""
    whole = torch.empty(n, d + extra, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // (d + extra))
    for a in range(0, n, step):
        b = min(n, a + step)
        whole[a:b] = torch.randn(b - a, d + extra, generator=g, device="cuda") * std + mean
    return whole[:, :d]


def _ids(case, g):
    """Zipf ranks through a bijection onto the rows, so that hot rows lie anywhere; a share
    of the positions holds the padding id."""
    V, n = case["V"], case["n"]
    cdf = _popularity(case).cuda().cumsum(0)
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.searchsorted(cdf, u).clamp_(max=V - 1)
    a = 7919
    while math.gcd(a, V) != 1:
        a += 2
    ids = (rank * a + 12_345) % V
    pad = -1
    if case["modulo"]:  # hashed 64-bit ids that fall on these rows
        ids = ids + V * torch.randint(0, 1 << 40, (n,), generator=g, device="cuda")
        pad = -(1 << 62)
    masked = torch.rand(n, generator=g, device="cuda") < case["pad"]
    return torch.where(masked, torch.full_like(ids, pad), ids), pad, masked


def _data(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7_919 + 17)
    op, dtype = case["op"], DTYPES[case["type"]]
    s = {"op": op, "case": case}
    if op in ("norm", "clip"):
        s["grads"] = [_rows(g, 1, k, dtype, 0, std=0.01).view(-1) for k in _part_sizes(case)]
        return s
    n, d = case["n"], case["d"]
    if op in ("ln", "ln_grad"):
        x = _rows(g, n, d, dtype, case["extra"], mean=0.25)
        x[:, ::97] *= 20.0  # a few columns far larger than the others
        s["x"] = x
        s["gamma"] = (1.0 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(DTYPES[case["param"]])
        s["beta"] = (0.1 * torch.randn(d, generator=g, device="cuda")).to(DTYPES[case["param"]])
        if op == "ln_grad":
            s["dy"] = _rows(g, n, d, dtype, case["extra"], std=0.01)
            s["mean"] = torch.empty(n, device="cuda")
            s["rstd"] = torch.empty(n, device="cuda")
            step = max(1, (1 << 26) // d)
            for a in range(0, n, step):
                c = x[a:a + step].float()
                m = c.mean(1)
                s["mean"][a:a + step] = m
                s["rstd"][a:a + step] = ((c - m[:, None]).square().mean(1) + EPS).rsqrt()
        return s
    s["scale"] = math.sqrt(d)
    s["ids"], s["pad"], masked = _ids(case, g)
    if op == "embed":
        s["weights"] = _rows(g, case["V"], d, dtype, case["extra"], std=0.02)
    else:
        s["grad"] = _rows(g, n, d, dtype, case["extra"], std=0.01)
        s["grad"][masked] = float("nan")
        if op == "grad_dense":
            s["out"] = torch.empty(case["V"], d, device="cuda")
    return s


def prepare(case, seed):
    s = _data(case, seed)
    if s["op"] == "clip":
        if case["pack"]:
            s["flat"] = torch.empty(case["total"], device="cuda")
            s["out"] = list(s["flat"].split([t.numel() for t in s["grads"]]))
        else:
            s["out"] = [torch.empty_like(t) for t in s["grads"]]
    if own:
        from paper_2205_11048_gb300 import binding as B
        s["worker"] = B.Worker()
        s["mode"] = B.MODULO if case.get("modulo") else B.DIRECT
        if s["op"] in ("norm", "clip"):  # the list of a program's gradient tensors
            s["parts"] = B.grad_parts(s["grads"], s.get("out"))
    return s


# ---- one pass -------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    w, op, c = s["worker"], s["op"], s["case"]
    if op == "embed":
        return w.embed(s["weights"], s["ids"], scale=s["scale"], pad_id=s["pad"],
                       dtype=DTYPES[c["out_type"]], id_mode=s["mode"])
    if op == "grad":
        ids, rows, count = w.embed_grad(s["ids"], s["grad"], c["V"], scale=s["scale"], pad_id=s["pad"],
                                        id_mode=s["mode"])
        return {"ids": ids, "rows": rows, "count": count}
    if op == "grad_dense":
        return w.embed_grad_dense(s["ids"], s["grad"], s["out"], scale=s["scale"], pad_id=s["pad"],
                                  id_mode=s["mode"])
    if op == "norm":
        return w.grad_norm(s["parts"])
    if op == "clip":
        norm = w.clip_grads(s["parts"], MAX_NORM)
        return {"norm": norm, "grads": s["flat"] if c["pack"] else s["out"]}
    if op == "ln":
        y, mean, rstd = w.layer_norm(s["x"], s["gamma"], s["beta"], EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dgamma, dbeta = w.layer_norm_grad(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _kept_rows(s):
    """The positions that are no padding, and the rows that their ids name."""
    kept = (s["ids"] != s["pad"]).nonzero().view(-1)
    ids = s["ids"][kept]
    return kept, (torch.remainder(ids, s["case"]["V"]) if s["case"]["modulo"] else ids)


def _run_plain(s):
    op, c = s["op"], s["case"]
    if op == "embed":
        ids = torch.remainder(s["ids"], c["V"])  # padding reads some row and is blanked
        y = s["weights"][ids].float() * s["scale"]
        return torch.where((s["ids"] != s["pad"])[:, None], y, 0.0).to(DTYPES[c["out_type"]])
    if op == "grad":
        kept, rows = _kept_rows(s)
        rows, order = torch.sort(rows, stable=True)
        first = torch.ones_like(rows, dtype=torch.bool)
        first[1:] = rows[1:] != rows[:-1]
        ids = torch.full_like(s["ids"], -1)
        sums = torch.zeros(c["n"], c["d"], device="cuda")
        if rows.numel():  # the slots that no row needs repeat the last one's id, with zeros
            ids[:] = rows[-1]
            slot = first.cumsum(0) - 1
            ids[slot] = rows
            sums.index_add_(0, slot, s["grad"][kept[order]].float())
        return {"ids": ids, "rows": sums * s["scale"], "count": first.sum()}
    if op == "grad_dense":
        kept, rows = _kept_rows(s)
        out = s["out"]
        out.zero_()
        out.index_add_(0, rows, s["grad"][kept].float() * s["scale"])
        return out
    if op in ("norm", "clip"):
        norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
        if op == "norm":
            return norm
        coef = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
        for t, o in zip(s["grads"], s["out"]):
            o.copy_(t.float() * coef)
        return {"norm": norm, "grads": s["flat"] if c["pack"] else s["out"]}
    x, gamma = s["x"].float(), s["gamma"].float()
    if op == "ln":
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = 1.0 / (x.square().mean(1) + EPS).sqrt()
        y = x * rstd[:, None] * gamma + s["beta"].float()
        return {"y": y.to(DTYPES[c["type"]]), "mean": mean, "rstd": rstd}
    dy = s["dy"].float()
    h = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * gamma
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return {"dx": dx.to(DTYPES[c["type"]]), "dgamma": (dy * h).sum(0), "dbeta": dy.sum(0)}


# ---- what a pass cannot do without ----------------------------------------------------

def work(case):
    op, b = case["op"], BYTES[case["type"]]
    if op in ("norm", "clip"):
        out = 0 if op == "norm" else 4 if case["pack"] else b
        return {"bytes": case["total"] * (b + out) + 4, "flops": case["total"] * (2 if op == "norm" else 3)}
    n, d = case["n"], case["d"]
    if op == "ln":
        return {"bytes": 2 * n * d * b + 8 * n + 2 * d * BYTES[case["param"]], "flops": 7 * n * d}
    if op == "ln_grad":
        return {"bytes": 3 * n * d * b + 8 * n + d * (BYTES[case["param"]] + 8), "flops": 13 * n * d}
    real = n * (1.0 - case["pad"])
    # the rows that n draws are expected to meet
    rows = float((-torch.expm1(real * torch.log1p(-_popularity(case).clamp(max=1 - 1e-12)))).sum())
    if op == "embed":
        return {"bytes": 8 * n + rows * d * b + n * d * BYTES[case["out_type"]], "flops": real * d}
    out = n * (8 + 4 * d) + 8 if op == "grad" else case["V"] * d * 4
    return {"bytes": 8 * n + real * d * b + out, "flops": real * d}


# ---- the definitions in 64 bits -------------------------------------------------------

def exact(case, seed):
    s = _data(case, seed)
    op = case["op"]
    if op in ("norm", "clip"):
        wide = torch.cat([t.double() for t in s["grads"]])
        norm = torch.dot(wide, wide).sqrt()
        if op == "norm":
            return norm
        wide *= min(1.0, MAX_NORM / (float(norm) + 1e-6))
        return {"norm": norm,
                "grads": wide if case["pack"] else list(wide.split([t.numel() for t in s["grads"]]))}
    if op in ("ln", "ln_grad"):
        x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
        d = x.shape[1]
        if op == "ln":
            mean = x.sum(1) / d
            var = (x - mean[:, None]).pow(2).sum(1) / d
            rstd = (var + EPS).pow(-0.5)
            return {"y": torch.addcmul(beta, (x - mean[:, None]) * rstd[:, None], gamma), "mean": mean,
                    "rstd": rstd}
        mean, rstd, dy = s["mean"].double(), s["rstd"].double(), s["dy"].double()
        h = (x - mean[:, None]) * rstd[:, None]
        along = (dy * h) @ gamma / d
        dx = rstd[:, None] * (dy * gamma - (dy @ gamma / d)[:, None] - h * along[:, None])
        return {"dx": dx, "dgamma": torch.einsum("nd,nd->d", dy, h), "dbeta": dy.sum(0)}
    ids, V = s["ids"].cpu(), case["V"]
    real = ids != s["pad"]
    at = (ids % V if case["modulo"] else ids)[real].cuda()
    real = real.cuda()
    if op == "embed":
        y = torch.zeros(case["n"], case["d"], dtype=torch.float64, device="cuda")
        y[real] = s["weights"].double().index_select(0, at) * s["scale"]
        return y
    sums = torch.zeros(V, case["d"], dtype=torch.float64, device="cuda")
    sums.index_add_(0, at, s["grad"][real].double())
    sums *= s["scale"]
    if op == "grad_dense":
        return sums
    met = torch.bincount(at, minlength=V).nonzero().view(-1)
    u, n = met.numel(), case["n"]
    ids = torch.cat([met, (met[-1:] if u else torch.tensor([-1], device="cuda")).expand(n - u)])
    return {"ids": ids, "rows": torch.cat([sums[met], sums.new_zeros(n - u, case["d"])]),
            "count": torch.tensor(u, device="cuda")}
