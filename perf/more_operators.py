"""The operators of a trainable block over tokens, as cases that can be timed and
compared: a block's output normalised, gated and added to the residual stream with
the norm before the next block, a gated linear recurrence over sequences, both in
both directions, and AdamW over many tensors at once.

A case is a dict of plain values:
  op        "norm", "norm_grad", "scan", "scan_grad" or "adamw"
  type      "f32", "bf16" or "f16", of x, the gate and the gradients
 norm, norm_grad:
  n, d      rows and width
  wide      type of the residual stream and the sum ("" without a residual)
  post, pre norm of the block's output and of the sum: "none", "rms" or "layer"
  gate      "none", "mul", "sigmoid" or "silu"
  param     type of the norms' weights and biases
 scan, scan_grad:
  layout    "equal" (sequences of one length), "padded" (of one length, but the rows
            behind each sequence's own length belong to none) or "packed" (one after
            another, of any length, with rows of none behind the last)
  n, rows   sequences, and rows of all of them together
  d         channels
  decay     "sigmoid" or "log": what the forget gate is given as
  tied      the input is weighted by one minus the decay
  state     each sequence starts from a state
  in_place  the last state replaces the first
 adamw:
  parts, total   tensors and their elements together
  weight    type of the weights
  copy      type of a second copy of the weights ("" for none)
  bits      of the states
"""
import math
import random

import torch

own = False

EPS = 1e-6
MAX_NORM = 0.5
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "": 0}

NORM = dict(type="bf16", wide="bf16", post="rms", pre="rms", gate="silu", param="f32")
SCAN = dict(type="bf16", layout="equal", decay="sigmoid", tied=True, state=False, in_place=False)
ADAMW = dict(op="adamw", type="bf16", weight="f32", copy="", bits=32)


def listed():
    return [
        # one new token of each of 64 sequences: the time is the call's and the launch's
        dict(NORM, name="norm-64x1024", op="norm", n=64, d=1024),
        # a long batch between two blocks, on a float32 residual stream
        dict(NORM, name="norm-32768x4096", op="norm", n=32_768, d=4096, wide="f32", post="none", gate="none",
             param="bf16"),
        # an odd width in float32, layer norms
        dict(NORM, name="norm-grad-5003x1001-f32", op="norm_grad", n=5_003, d=1_001, type="f32", wide="f32",
             post="layer", pre="layer", gate="sigmoid"),
        # a long batch, backwards
        dict(NORM, name="norm-grad-32768x2048", op="norm_grad", n=32_768, d=2048),
        # one new token of each of 256 sequences, with the states in place
        dict(SCAN, name="scan-step-256x1024", op="scan", n=256, rows=256, d=1024, state=True, in_place=True),
        # a training batch of equal sequences
        dict(SCAN, name="scan-16x4096x2048", op="scan", n=16, rows=65_536, d=2048),
        # one long prompt in few channels: the work is split over the length
        dict(SCAN, name="scan-1x262144x256", op="scan", n=1, rows=262_144, d=256, decay="log", tied=False,
             state=True),
        # a ragged batch of an odd width in float32, packed
        dict(SCAN, name="scan-grad-packed-61x20003x501-f32", op="scan_grad", n=61, rows=20_003, d=501, type="f32",
             layout="packed", state=True),
        # a padded training batch, backwards
        dict(SCAN, name="scan-grad-padded-32x2048x2048", op="scan_grad", n=32, rows=65_536, d=2048,
             layout="padded"),
        # the weights of a small model
        dict(ADAMW, name="adamw-306k", parts=7, total=306_496, type="f32"),
        # a large model's, with 16-bit gradients and a 16-bit copy for the next forward pass
        dict(ADAMW, name="adamw-64M", parts=148, total=64_000_000, copy="bf16"),
        # the same with states in 8 bits, and the states read out as a checkpoint takes them
        dict(ADAMW, name="adamw8-64M", parts=148, total=64_000_000, copy="bf16", bits=8),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi):
    d = _between(rng, 8, hi)
    if rng.random() < 0.6:  # most widths are multiples of eight, the others as they come
        d = max(8, d // 8 * 8)
    return d


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "scan", "scan_grad", "adamw"])
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    if op == "adamw":
        total = _between(rng, 1_000, 64_000_000)
        return dict(ADAMW, parts=min(_between(rng, 1, 200), total), total=total, type=kind,
                    weight=rng.choice(["f32", "f32", "bf16"]), copy=rng.choice(["", "bf16", "f16"]),
                    bits=rng.choice([32, 8]))
    if op in ("norm", "norm_grad"):
        d = _width(rng, 4096)
        norms = ["none", "rms", "layer"]
        return dict(NORM, op=op, n=_between(rng, 1, min(262_144, (1 << 26) // d)), d=d, type=kind,
                    wide=rng.choice(["f32", kind, kind, ""]), post=rng.choice(norms), pre=rng.choice(norms),
                    gate=rng.choice(["none", "mul", "sigmoid", "silu"]), param=rng.choice(["f32", kind]))
    d = _width(rng, 2048)
    layout = rng.choice(["equal", "padded", "packed"])
    rows = _between(rng, 1, min(262_144, (1 << 26) // d))
    n = _between(rng, 1, rows)
    if layout != "packed":
        rows -= rows % n
    return dict(SCAN, op=op, n=n, rows=rows, d=d, type=kind, layout=layout,
                decay=rng.choice(["sigmoid", "log"]), tied=rng.random() < 0.5, state=rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------

def _normal(g, *shape, dtype=torch.float32, mean=0.0, std=1.0):
    whole = torch.empty(shape, dtype=dtype, device="cuda")
    flat = whole.view(-1)
    for a in range(0, flat.numel(), 1 << 26):
        b = min(flat.numel(), a + (1 << 26))
        flat[a:b] = torch.randn(b - a, generator=g, device="cuda") * std + mean
    return whole


def _sequences(case):
    """The first row and the length of each sequence, as lists: the same for every seed."""
    n, rows, r = case["n"], case["rows"], random.Random(case["n"] * 31 + case["rows"])
    if case["layout"] == "packed":  # cuts at any place, twice at the same one too; a few rows behind
        used = rows - rows // 50
        cuts = [0] + sorted(r.randint(0, used) for _ in range(n - 1)) + [used]
        return cuts[:-1], [b - a for a, b in zip(cuts, cuts[1:])]
    each = rows // n
    first = [i * each for i in range(n)]
    if case["layout"] == "equal":
        return first, [each] * n
    return first, [r.randint(0, each) if i else each for i in range(n)]


def _parts(case):
    """The sizes of a few matrices and many small vectors, ragged, that sum to the total."""
    r = random.Random(case["parts"])
    share = [math.exp(r.uniform(0.0, 7.0)) for _ in range(case["parts"])]
    left = case["total"] - case["parts"]
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[0] += case["total"] - sum(sizes)
    return sizes


def _norm_data(case, g):
    n, d, kind, param = case["n"], case["d"], DTYPES[case["type"]], DTYPES[case["param"]]
    s = {"gate": None, "residual": None}
    s["x"] = _normal(g, n, d, dtype=kind, mean=0.25)
    s["x"][:, ::97] *= 20.0  # a few columns far larger than the others
    if case["gate"] != "none":
        s["gate"] = _normal(g, n, d, dtype=kind)
    if case["wide"]:
        s["residual"] = _normal(g, n, d, dtype=DTYPES[case["wide"]], std=2.0)
    for k, (mean, std) in {"post_weight": (1.0, 0.1), "post_bias": (0.0, 0.1), "pre_weight": (1.0, 0.1),
                           "pre_bias": (0.0, 0.1)}.items():
        s[k] = _normal(g, d, dtype=param, mean=mean, std=std)
    if case["post"] != "layer":
        s["post_bias"] = None
    if case["pre"] != "layer":
        s["pre_bias"] = None
    if case["pre"] == "none":
        s["pre_weight"] = None
    s["residual_scale"], s["block_scale"] = (1.25, 0.5) if case["wide"] else (1.0, 1.0)
    if case["op"] == "norm_grad":
        s["dy"] = _normal(g, n, d, dtype=kind, std=0.01) if case["pre"] != "none" else None
        wide = DTYPES[case["wide"] or case["type"]]
        s["dz"] = _normal(g, n, d, dtype=wide, std=0.01)
        s["z"] = torch.empty(n, d, dtype=wide, device="cuda")
        s["stats"] = torch.empty(n, 4, device="cuda")
        step = max(1, (1 << 25) // d)
        for a in range(0, n, step):  # as the forward pass leaves them
            rows = {k: s[k][a:a + step] if k in ("x", "gate", "residual") and s[k] is not None else s[k] for k in s}
            y, s["z"][a:a + step], s["stats"][a:a + step] = _norm_plain(case, rows)
    return s


def _scan_data(case, g):
    n, rows, d, kind = case["n"], case["rows"], case["d"], DTYPES[case["type"]]
    first, length = _sequences(case)
    s = {"state": None, "first": torch.tensor(first, device="cuda"), "length": torch.tensor(length, device="cuda")}
    s["offsets"] = torch.tensor(first + [first[-1] + length[-1]], device="cuda")
    s["x"] = _normal(g, rows, d, dtype=kind)
    s["f"] = _normal(g, rows, d, dtype=kind, mean=3.0, std=1.5)
    if case["decay"] == "log":  # from short memories to very long ones
        s["f"] = (s["f"].float().mul(-1.0).exp() * -1.0).to(kind)
    if case["layout"] != "equal":  # what rows of no sequence hold is never to be used
        none = ~_membership(s, rows)[0]
        s["x"][none] = float("nan")
        s["f"][none] = float("nan")
    if case["state"]:
        s["state"] = _normal(g, n, d)
    if case["op"] == "scan_grad":
        s["dy"] = _normal(g, rows, d, dtype=kind, std=0.01)
        s["dlast"] = _normal(g, n, d, std=0.01) if case["state"] else None
        s["y"] = _scan_plain(case, s)[0]
        if case["layout"] != "equal":
            s["dy"][none] = float("nan")
            s["y"][none] = float("nan")
    return s


def _adamw_data(case, g):
    """Tensors as parts of flat arrays, each from a multiple of BLOCK elements on; what lies
    between them is zero."""
    sizes = _parts(case)
    starts, at = [], 0
    for k in sizes:
        starts.append(at)
        at += -(-k // BLOCK) * BLOCK
    s = {"spans": [(a, k) for a, k in zip(starts, sizes)], "length": at}
    inside = torch.zeros(at, dtype=torch.bool, device="cuda")
    decays = torch.zeros(at, device="cuda")
    for i, (a, k) in enumerate(s["spans"]):
        inside[a:a + k] = True
        decays[a:a + k] = 0.0 if i % 3 == 2 else DECAY  # norms' weights and biases do not decay
    s["decays"] = decays
    s["w"] = torch.where(inside, _normal(g, at, std=0.02), 0.0).to(DTYPES[case["weight"]])
    s["grad"] = torch.where(inside, _normal(g, at, std=1e-4), 0.0).to(DTYPES[case["type"]])
    s["norm"] = s["grad"].double().square().sum().sqrt().float()
    # states of a run that has come some way: of different sizes from tensor to tensor
    size = torch.zeros(at, device="cuda")
    for a, k in s["spans"]:
        size[a:a + k] = 1e-4 * math.exp(3.0 * random.Random(a).uniform(-1.0, 1.0))
    s["m"] = _normal(g, at) * size * 0.3
    s["v"] = _normal(g, at).square() * size.square()
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to_m8(s["m"])
        s["v"], s["v_scale"] = _to_v8(s["v"])
    s["step"] = torch.full((), 1000, dtype=torch.int64, device="cuda")
    s["copy"] = torch.zeros(at, dtype=DTYPES[case["copy"]], device="cuda") if case["copy"] else None
    return s


def _data(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7_919 + 29)
    make = _norm_data if case["op"] in ("norm", "norm_grad") else _adamw_data if case["op"] == "adamw" else _scan_data
    return dict(make(case, g), case=case)


def prepare(case, seed):
    s = _data(case, seed)
    if own:
        from paper_2205_11048_gb300 import binding as B
        s["worker"] = B.Worker()
        if case["op"] in ("norm", "norm_grad"):
            s["block"] = B.residual_norm(
                post_norm=case["post"], pre_norm=case["pre"], gate=case["gate"], eps=EPS,
                residual_scale=s["residual_scale"], block_scale=s["block_scale"],
                **{k: s[k] for k in ("post_weight", "post_bias", "pre_weight", "pre_bias")})
        elif case["op"] == "adamw":  # the program's tensors, in the arrays that hold them
            cut = lambda t: [t[a:a + k] for a, k in s["spans"]]  # noqa: E731
            blocks = lambda t: [t[a // BLOCK:(a + k + BLOCK - 1) // BLOCK] for a, k in s["spans"]]  # noqa: E731
            scales = {k: blocks(s[k]) for k in ("m_scale", "v_scale") if k in s}
            states = B.adamw_states(cut(s["w"]), bits=case["bits"], betas=(BETA1, BETA2), eps=ADAM_EPS,
                                    weight_decay=[0.0 if i % 3 == 2 else DECAY for i in range(case["parts"])],
                                    copies=cut(s["copy"]) if case["copy"] else None,
                                    m=cut(s["m"]), v=cut(s["v"]), step=s["step"], **scales)
            s["parts"] = states.parts(cut(s["grad"]))
            if case["bits"] == 8:
                s["m_values"], s["v_values"] = torch.zeros(2, s["length"], device="cuda")
                s["values"] = cut(s["m_values"]), cut(s["v_values"])
        else:
            s["sequences"] = B.sequences(
                case["n"], offsets=s["offsets"] if case["layout"] == "packed" else None,
                lengths=s["length"] if case["layout"] == "padded" else None)
    return s


# ---- one pass -------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    w, c = s["worker"], s["case"]
    if c["op"] == "norm":
        y, z, stats = w.residual_norm(s["block"], s["x"], s["residual"], s["gate"])
        return {"y": y, "z": z, "stats": stats}
    if c["op"] == "norm_grad":
        return w.residual_norm_grad(s["block"], s["dy"], s["dz"], s["x"], s["z"], s["stats"], s["gate"],
                                    residual=bool(c["wide"]))
    if c["op"] == "scan":
        y, last = w.gated_scan(s["x"], s["f"], s["sequences"], decay=c["decay"], tied=c["tied"], state=s["state"],
                               state_out=s["state"] if c["in_place"] else None)
        return {"y": y, "state": last}
    if c["op"] == "scan_grad":
        dx, df, dstate = w.gated_scan_grad(s["dy"], s["x"], s["f"], s["y"], s["sequences"], decay=c["decay"],
                                           tied=c["tied"], state=s["state"], dstate=s["dlast"])
        return {"dx": dx, "df": df, "dstate": dstate}
    w.adamw(s["parts"], LR, norm=s["norm"], max_norm=MAX_NORM)
    out = {"w": s["w"], "copy": s["copy"], "step": s["step"]}
    if c["bits"] == 8:
        w.adamw_values(s["parts"], *s["values"])
        return dict(out, m=s["m_values"], v=s["v_values"])
    return dict(out, m=s["m"], v=s["v"])


def _run_plain(s):
    c = s["case"]
    if c["op"] == "norm":
        y, z, stats = _norm_plain(c, s)
        return {"y": y, "z": z, "stats": stats}
    if c["op"] == "norm_grad":
        return _norm_grad_plain(c, s)
    if c["op"] == "scan":
        y, last = _scan_plain(c, s)
        if c["in_place"]:
            s["state"].copy_(last)
            last = s["state"]
        return {"y": y, "state": last}
    if c["op"] == "scan_grad":
        return _scan_grad_plain(c, s)
    return _adamw_plain(c, s)


def _normed(x, kind):
    """The rows normalised, and the mean and the reciprocal deviation that did it."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    if kind == "none":
        return x, mean, torch.ones_like(mean)
    rstd = 1.0 / ((x - mean).square().mean(1, keepdim=True) + EPS).sqrt()
    return (x - mean) * rstd, mean, rstd


def _affine(x, weight, bias):
    if weight is not None:
        x = x * weight.float()
    return x if bias is None else x + bias.float()


def _norm_plain(c, s):
    x, mx, rx = _normed(s["x"].float(), c["post"])
    v = _affine(x, s["post_weight"], s["post_bias"])
    if c["gate"] != "none":
        g = s["gate"].float()
        v = v * (g if c["gate"] == "mul" else 1.0 / (1.0 + (-g).exp()) * (g if c["gate"] == "silu" else 1.0))
    z = v * s["block_scale"]
    if s["residual"] is not None:
        z = s["residual"].float() * s["residual_scale"] + z
    h, mz, rz = _normed(z, c["pre"])
    y = None if c["pre"] == "none" else _affine(h, s["pre_weight"], s["pre_bias"]).to(DTYPES[c["type"]])
    return y, z.to(DTYPES[c["wide"] or c["type"]]), torch.cat([mx, rx, mz, rz], 1)


def _back_through(g, h, rstd, kind):
    """The gradient of a normalised row's input from that of its output."""
    if kind == "none":
        return g
    along = h * (g * h).mean(1, keepdim=True)
    return rstd * (g - along - (g.mean(1, keepdim=True) if kind == "layer" else 0.0))


def _norm_grad_plain(c, s):
    kind, wide = DTYPES[c["type"]], DTYPES[c["wide"] or c["type"]]
    mx, rx, mz, rz = s["stats"].split(1, 1)
    dz, out = s["dz"].float(), {}
    if c["pre"] != "none":
        h, dy = (s["z"].float() - mz) * rz, s["dy"].float()
        dz = dz + _back_through(_affine(dy, s["pre_weight"], None), h, rz, c["pre"])
        out["dpre_weight"] = (dy * h).sum(0)
        if c["pre"] == "layer":
            out["dpre_bias"] = dy.sum(0)
    if c["wide"]:
        out["dresidual"] = (dz * s["residual_scale"]).to(wide)
    e = dz * s["block_scale"]
    h = (s["x"].float() - mx) * rx
    if c["gate"] != "none":
        g = s["gate"].float()
        sig = 1.0 / (1.0 + (-g).exp())
        act, slope = {"mul": (g, 1.0), "sigmoid": (sig, sig * (1.0 - sig)),
                      "silu": (g * sig, sig * (1.0 + g * (1.0 - sig)))}[c["gate"]]
        out["dgate"] = (e * _affine(h, s["post_weight"], s["post_bias"]) * slope).to(kind)
        e = e * act
    out["dpost_weight"] = (e * h).sum(0)
    if c["post"] == "layer":
        out["dpost_bias"] = e.sum(0)
    out["dx"] = _back_through(_affine(e, s["post_weight"], None), h, rx, c["post"]).to(kind)
    return out


def _membership(s, rows):
    """Which rows belong to a sequence, which are first and last in theirs, and whose they are."""
    t = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(s["first"], t, right=True) - 1  # of those that begin there, the last: it is not empty
    pos = t - s["first"][seq]
    return pos < s["length"][seq], pos == 0, pos == s["length"][seq] - 1, seq


def _combined(a, b, back=False):
    """All h_t = a_t h_(t-1) + b_t, or with t+1, by doubling: pairs of ever longer stretches are joined."""
    k, n = 1, a.shape[0]
    while k < n:
        here, there = (slice(0, n - k), slice(k, n)) if back else (slice(k, n), slice(0, n - k))
        b2, a2 = a[here] * b[there], a[here] * a[there]
        b, a = b.clone(), a.clone()
        b[here] += b2
        a[here] = a2
        k *= 2
    return b


def _gates(c, s, inside):
    """The decay, one minus it, and x, in 32 bits, with harmless values in rows of no sequence."""
    x = torch.where(inside, s["x"].float(), 0.0)
    f = torch.where(inside, s["f"].float(), 0.0)
    if c["decay"] == "log":
        f = f.clamp(max=0.0)
        return f.exp(), -torch.expm1(f), x
    return 1.0 / (1.0 + (-f).exp()), 1.0 / (1.0 + f.exp()), x


def _scan_plain(c, s):
    inside, first, _, seq = _membership(s, c["rows"])
    inside, first = inside[:, None], (first & inside)[:, None]
    a, rest, x = _gates(c, s, inside)
    b = rest * x if c["tied"] else x
    if s["state"] is not None:
        b = torch.where(first, b + a * s["state"][seq], b)
    h = _combined(torch.where(first | ~inside, 0.0, a), torch.where(inside, b, 0.0))
    at = (s["first"] + s["length"] - 1).clamp(min=0)
    none = torch.zeros_like(h[:1]) if s["state"] is None else s["state"]
    last = torch.where((s["length"] > 0)[:, None], h[at], none)
    return torch.where(inside, h, 0.0).to(DTYPES[c["type"]]), last


def _scan_grad_plain(c, s):
    kind = DTYPES[c["type"]]
    inside, first, last, seq = _membership(s, c["rows"])
    inside, first, last = inside[:, None], (first & inside)[:, None], (last & inside)[:, None]
    a, rest, x = _gates(c, s, inside)
    dy = torch.where(inside, s["dy"].float(), 0.0)
    if s["dlast"] is not None:
        dy = torch.where(last, dy + s["dlast"][seq], dy)
    after = torch.where(last, 0.0, torch.cat([a[1:], torch.zeros_like(a[:1])]))
    g = _combined(torch.where(inside, after, 0.0), dy, back=True)
    y = torch.where(inside, s["y"].float(), 0.0)
    h = torch.cat([torch.zeros_like(y[:1]), y[:-1]])
    h = torch.where(first, 0.0 if s["state"] is None else s["state"][seq], h)
    da = g * (h - x) if c["tied"] else g * h
    df = da * a * rest if c["decay"] == "sigmoid" else torch.where(s["f"].float() > 0, 0.0, da * a)
    dx = g * rest if c["tied"] else g
    out = {"dx": torch.where(inside, dx, 0.0).to(kind), "df": torch.where(inside, df, 0.0).to(kind)}
    out["dstate"] = None
    if c["state"]:
        at = s["first"].clamp(max=c["rows"] - 1)
        out["dstate"] = torch.where((s["length"] > 0)[:, None], a[at] * g[at], s["dlast"])
    return out


# States in 8 bits: blocks of BLOCK elements share a float32 scale. The first moment is held as
# an 8-bit float of 4 exponent and 3 mantissa bits, the largest of a block as 448; the second as
# one of 5 exponent and 3 mantissa bits without a sign, the largest as 1.875. The smallest code
# but zero stands for 1.125 * 2^-31, and what is not zero does not become zero.

def _to_m8(m):
    m = m.view(-1, BLOCK)
    scale = m.abs().amax(1, keepdim=True).clamp(min=2.0**-100) * (1.0 / 448.0)
    return (m * (torch.ones_like(scale) / scale)).to(torch.float8_e4m3fn).view(torch.uint8).view(-1), scale.view(-1)


def _to_v8(v):
    v = v.view(-1, BLOCK)
    scale = v.amax(1, keepdim=True).clamp(min=2.0**-100) * (1.0 / 1.875)
    bits = (v * (torch.ones_like(scale) / scale)).view(torch.int32)
    code = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - 768  # to the nearest, ties to the even code
    return torch.where(v > 0, code.clamp(1, 255), 0).to(torch.uint8).view(-1), scale.view(-1)


def _from_m8(codes, scale):
    return (codes.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * scale[:, None]).view(-1)


def _from_v8(codes, scale):
    code = codes.int()
    q = torch.where(code > 0, ((code + 768) << 20).view(torch.float32), 0.0)
    return (q.view(-1, BLOCK) * scale[:, None]).view(-1)


def _adamw_plain(c, s):
    g = s["grad"].float() * (torch.full_like(s["norm"], MAX_NORM) / (s["norm"] + 1e-6)).clamp(max=1.0)
    m, v = s["m"], s["v"]
    if c["bits"] == 8:
        m, v = _from_m8(m, s["m_scale"]), _from_v8(v, s["v_scale"])
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    s["step"] += 1
    t = s["step"].double()
    size = (LR / (1.0 - torch.pow(BETA1, t))).float()
    root = (1.0 / (1.0 - torch.pow(BETA2, t)).sqrt()).float()
    w = s["w"].float() * (1.0 - LR * s["decays"]) - size * (m / (v.sqrt() * root + ADAM_EPS))
    s["w"].copy_(w)
    if s["copy"] is not None:
        s["copy"].copy_(w)
    out = {"w": s["w"], "copy": s["copy"], "step": s["step"]}
    if c["bits"] == 8:
        s["m"], s["m_scale"] = _to_m8(m)
        s["v"], s["v_scale"] = _to_v8(v)
        return dict(out, m=_from_m8(s["m"], s["m_scale"]), v=_from_v8(s["v"], s["v_scale"]))
    s["m"].copy_(m)
    s["v"].copy_(v)
    return dict(out, m=s["m"], v=s["v"])


# ---- what a pass cannot do without ----------------------------------------------------

def work(case):
    op, b = case["op"], BYTES[case["type"]]
    if op == "adamw":
        each = b + 2 * BYTES[case["weight"]] + BYTES[case["copy"]]
        # 8-bit states go in and out with their scales, and out once more as float32 values
        each += 16 if case["bits"] == 32 else 4 + 16.0 / BLOCK + 8
        return {"bytes": case["total"] * each, "flops": case["total"] * 16}
    if op in ("scan", "scan_grad"):
        used, states = sum(_sequences(case)[1]), 4 * case["n"] * case["d"]
        if op == "scan":
            return {"bytes": (2 * used + case["rows"]) * case["d"] * b + states * (2 if case["state"] else 1),
                    "flops": used * case["d"] * 8}
        return {"bytes": (4 * used + 2 * case["rows"]) * case["d"] * b + states * (3 if case["state"] else 0),
                "flops": used * case["d"] * 14}
    n, d, wide, gate = case["n"], case["d"], BYTES[case["wide"]], case["gate"] != "none"
    pre, post = case["pre"] != "none", case["post"] != "none"
    sums = wide or b
    if op == "norm":
        return {"bytes": n * d * (b + wide + gate * b + sums + pre * b) + 16 * n, "flops": n * d * 18}
    return {"bytes": n * d * ((2 + 2 * gate + pre) * b + (1 + pre) * sums + wide) + 16 * n + 8 * d * (1 + pre),
            "flops": n * d * (20 + 8 * pre + 8 * post)}


# ---- the definitions in 64 bits -------------------------------------------------------

def exact(case, seed):
    s = _data(case, seed)
    if case["op"] == "norm":
        return _norm_exact(case, s)
    if case["op"] == "norm_grad":
        return _norm_grad_exact(case, s)
    if case["op"] == "adamw":
        return _adamw_exact(case, s)
    return _scan_exact(case, s) if case["op"] == "scan" else _scan_grad_exact(case, s)


def _statistics(x, kind):
    d = x.shape[1]
    mean = x.sum(1) / d if kind == "layer" else x.new_zeros(x.shape[0])
    var = torch.einsum("nd,nd->n", x, x) / d if kind == "rms" else (x - mean[:, None]).pow(2).sum(1) / d
    return mean, (x.new_ones(x.shape[0]) if kind == "none" else (var + EPS).pow(-0.5))


def _wide(t, like, fill):
    return like.new_full(like.shape[1:], fill) if t is None else t.double()


def _gate_exact(c, s):
    """The gate's factor and its derivative."""
    if c["gate"] == "none":
        return 1.0, 0.0
    g = s["gate"].double()
    sig = torch.sigmoid(g)
    if c["gate"] == "mul":
        return g, torch.ones_like(g)
    if c["gate"] == "sigmoid":
        return sig, sig - sig * sig
    return g * sig, sig + g * sig - g * sig * sig


def _norm_exact(c, s):
    x = s["x"].double()
    mx, rx = _statistics(x, c["post"])
    z = torch.addcmul(_wide(s["post_bias"], x, 0.0), (x - mx[:, None]) * rx[:, None], _wide(s["post_weight"], x, 1.0))
    z = s["block_scale"] * z * _gate_exact(c, s)[0]
    if s["residual"] is not None:
        z += s["residual_scale"] * s["residual"].double()
    mz, rz = _statistics(z, c["pre"])
    y = None
    if c["pre"] != "none":
        y = torch.addcmul(_wide(s["pre_bias"], x, 0.0), (z - mz[:, None]) * rz[:, None], _wide(s["pre_weight"], x, 1.0))
    return {"y": y, "z": z, "stats": torch.stack([mx, rx, mz, rz], 1)}


def _norm_grad_exact(c, s):
    st, out = s["stats"].double(), {}
    x = (s["x"].double() - st[:, :1]) * st[:, 1:2]
    d, D = x.shape[1], s["dz"].double()
    if c["pre"] != "none":
        z, dy, wp = (s["z"].double() - st[:, 2:3]) * st[:, 3:], s["dy"].double(), _wide(s["pre_weight"], x, 1.0)
        mean = (dy @ wp / d)[:, None] if c["pre"] == "layer" else 0.0
        D = D + st[:, 3:] * (dy * wp - mean - z * ((dy * z) @ wp / d)[:, None])
        out["dpre_weight"] = torch.einsum("nd,nd->d", dy, z)
        if c["pre"] == "layer":
            out["dpre_bias"] = dy.sum(0)
    if c["wide"]:
        out["dresidual"] = s["residual_scale"] * D
    wq = _wide(s["post_weight"], x, 1.0)
    act, slope = _gate_exact(c, s)
    if c["gate"] != "none":
        out["dgate"] = s["block_scale"] * D * slope * torch.addcmul(_wide(s["post_bias"], x, 0.0), x, wq)
    e = s["block_scale"] * D * act
    out["dpost_weight"] = torch.einsum("nd,nd->d", e, x)
    if c["post"] == "layer":
        out["dpost_bias"] = e.sum(0)
    dx = e * wq
    if c["post"] != "none":
        mean = (e @ wq / d)[:, None] if c["post"] == "layer" else 0.0
        dx = st[:, 1:2] * (dx - mean - x * ((e * x) @ wq / d)[:, None])
    out["dx"] = dx
    return out


def _walk(a, b):
    """All h_t = a_t h_(t-1) + b_t from h = 0: chunks of rows step by step side by side, then
    the chunks one after another."""
    n, d = a.shape
    size = max(1, int(math.isqrt(n)))
    many = -(-n // size)
    pad = (0, 0, 0, many * size - n)
    a = torch.nn.functional.pad(a, pad).view(many, size, d)
    h = torch.nn.functional.pad(b, pad).view(many, size, d)
    through = a.clone()
    for i in range(1, size):
        h[:, i] += a[:, i] * h[:, i - 1]
        through[:, i] *= through[:, i - 1]
    for j in range(1, many):
        h[j] += through[j] * h[j - 1, -1]
    return h.view(many * size, d)[:n]


def _rows_exact(c, s):
    """Sequence, place in it and membership of every row, by counting on the host."""
    seq, place = torch.zeros(c["rows"], dtype=torch.int64), torch.full((c["rows"],), -1)
    for i, (a, k) in enumerate(zip(*_sequences(c))):
        seq[a:a + k] = i
        place[a:a + k] = torch.arange(k)
    return seq.cuda(), place.cuda()


def _decay_exact(c, s, real):
    f = torch.where(real, s["f"].double(), 0.0)
    if c["decay"] == "log":
        f = torch.minimum(f, torch.zeros_like(f))
        return torch.exp(f), -torch.expm1(f)
    return torch.sigmoid(f), torch.sigmoid(-f)


def _scan_exact(c, s):
    seq, place = _rows_exact(c, s)
    real, first = (place >= 0)[:, None], (place == 0)[:, None]
    a, rest = _decay_exact(c, s, real)
    h = torch.where(real, s["x"].double(), 0.0)
    if c["tied"]:
        h = h * rest
    if s["state"] is not None:
        h = h + first * a * s["state"].double()[seq]
    h = _walk(a * (place > 0)[:, None], h) * real
    last = torch.zeros(c["n"], c["d"], dtype=torch.float64, device="cuda")
    if s["state"] is not None:
        last += s["state"]
    end = (s["length"] > 0).nonzero().view(-1)
    last[end] = h[(s["first"] + s["length"] - 1)[end]]
    return {"y": h, "state": last}


def _scan_grad_exact(c, s):
    seq, place = _rows_exact(c, s)
    real = (place >= 0)[:, None]
    a, rest = _decay_exact(c, s, real)
    g = torch.where(real, s["dy"].double(), 0.0)
    some = (s["length"] > 0).nonzero().view(-1)
    begin, end = s["first"][some], (s["first"] + s["length"] - 1)[some]
    if s["dlast"] is not None:
        g[end] += s["dlast"][some]
    flow = torch.roll(a, -1, 0)  # what carries the next row's gradient to this one
    flow[end] = 0.0
    g = _walk((flow * real).flip(0), g.flip(0)).flip(0)
    before = torch.roll(torch.where(real, s["y"].double(), 0.0), 1, 0)
    before[begin] = 0.0 if s["state"] is None else s["state"][some].double()
    if c["tied"]:
        before = before - torch.where(real, s["x"].double(), 0.0)
    df = g * before * a
    df = df * rest if c["decay"] == "sigmoid" else df * (s["f"].double() <= 0)
    out = {"dx": g * rest if c["tied"] else g, "df": torch.where(real, df, 0.0), "dstate": None}
    if c["state"]:
        out["dstate"] = s["dlast"].double()
        out["dstate"][some] = (a * g)[begin]
    return out


def _adamw_exact(c, s):
    g = s["grad"].double() * min(1.0, MAX_NORM / (float(s["norm"]) + 1e-6))
    m, v = s["m"], s["v"]
    if c["bits"] == 8:
        m, v = _from_m8(m, s["m_scale"]), _from_v8(v, s["v_scale"])
    m = torch.lerp(g, m.double(), BETA1)
    v = torch.lerp(g * g, v.double(), BETA2)
    t = int(s["step"]) + 1
    hat = (v / (1.0 - BETA2**t)).sqrt() + ADAM_EPS
    w = s["w"].double()
    w = w - LR * s["decays"].double() * w - LR * (m / (1.0 - BETA1**t)) / hat
    if c["bits"] == 8:  # the codes of the rounded moments; one next to a border may fall either way
        m, v = _from_m8(*_to_m8(m.float())), _from_v8(*_to_v8(v.float()))
    return {"w": w, "copy": w if c["copy"] else None, "step": s["step"] + 1, "m": m, "v": v}
