"""A block's operators against plain statements in 64 bits (needs a GPU).

Tolerances are bounds of the rounding, element by element, with U = 2^-24 the unit roundoff of
float32: beside each exact value goes a magnitude, the same formula of absolute values, and a
result that passes through at most k roundings is within k U of its magnitude of the exact one,
then rounded once more to its type (UNIT of itself).  k counts: a sum over a row of d columns at
most 32 additions in a thread, 5 in a warp and 5 across the warps (its mean and the root that
follow are within as many), a gate 12 (exp of up to 4 with arguments up to 4, and quotients)."""
import math

import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import IDS, TINY, TYPES, U, UNIT, gen, rand, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.fixture
def w():
    worker = B.Worker()
    yield worker
    worker.sync()
    worker.close()


def rounded(want, mag, k, dtype):
    return UNIT[dtype] * want.abs() * (1 + k * U) + k * U * mag + TINY[dtype]


# ---- norms with a gate and the residual -----------------------------------------------------

EPS = 1e-6


def stats_of(x, kind):
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    if kind == "none":
        return mean, torch.ones_like(mean)
    return mean, 1.0 / ((x - mean).square().mean(1, keepdim=True) + EPS).sqrt()


def act_of(gate, kind):
    sig = torch.sigmoid(gate)
    return {"mul": gate, "sigmoid": sig, "silu": gate * sig}[kind]


def formula(p, how):
    """(y, z) in 64 bits from the tensors of p, through autograd."""
    mx, rx = stats_of(p["x"], how["post_norm"])
    u = (p["x"] - mx) * rx
    if p.get("post_weight") is not None:
        u = u * p["post_weight"]
    if p.get("post_bias") is not None:
        u = u + p["post_bias"]
    if p.get("gate") is not None:
        u = u * act_of(p["gate"], how["gate"])
    z = how["block_scale"] * u
    if p.get("residual") is not None:
        z = z + how["residual_scale"] * p["residual"]
    if how["pre_norm"] == "none":
        return None, z
    mz, rz = stats_of(z, how["pre_norm"])
    y = (z - mz) * rz
    if p.get("pre_weight") is not None:
        y = y * p["pre_weight"]
    return (y if p.get("pre_bias") is None else y + p["pre_bias"]), z


def make(g, n, d, dtype, wide, post, pre, gate, ptype=torch.float32, extra=0, offset=0, weights=True, residual=True):
    t = {"x": rand(g, n, d, dtype=dtype, mean=0.3, extra=extra, offset=offset)}
    if residual:
        t["residual"] = rand(g, n, d, dtype=wide, std=1.5, extra=extra, offset=offset)
    if gate != "none":
        t["gate"] = rand(g, n, d, dtype=dtype, extra=extra, offset=offset).clamp_(-4, 4)
    if weights:
        t["post_weight"] = rand(g, d, dtype=ptype, mean=1.0, std=0.2)
        if post == "layer":
            t["post_bias"] = rand(g, d, dtype=ptype, std=0.3)
        if pre != "none":
            t["pre_weight"] = rand(g, d, dtype=ptype, mean=1.0, std=0.2)
        if pre == "layer":
            t["pre_bias"] = rand(g, d, dtype=ptype, std=0.3)
    how = dict(post_norm=post, pre_norm=pre, gate=gate, residual_scale=1.25, block_scale=0.5)
    block = B.residual_norm(eps=EPS, **how, **{k: t[k] for k in t if k.startswith(("post", "pre"))})
    return t, how, block


K = 160  # two norms of 42 and their quotients, a gate, scales, sums and products


def magnitudes(p, how, z):
    """Of z and y: the formulas of absolute values."""
    one = torch.ones_like(p["x"][:1])
    mx, rx = stats_of(p["x"], how["post_norm"])
    u = (p["x"].abs() + mx.abs()) * rx
    u = u * (1 + (u * rx).square().mean(1, keepdim=True) * 0) * p.get("post_weight", one).abs()
    u = u + p["post_bias"].abs() if "post_bias" in p else u
    if "gate" in p:
        u = u * act_of(p["gate"], how["gate"]).abs()
    mag = how["block_scale"] * u
    if "residual" in p:
        mag = mag + how["residual_scale"] * p["residual"].abs()
    if how["pre_norm"] == "none":
        return mag, None
    mz, rz = stats_of(z, how["pre_norm"])
    # a relative error of mag/sqrt(mean z^2) in z changes the deviation by as much
    spread = (mag.square().mean(1, keepdim=True)).sqrt() * rz
    my = (mag + mag.mean(1, keepdim=True)) * rz
    my = (my + spread * ((z - mz) * rz).abs()) * p.get("pre_weight", one).abs()
    return mag, (my + p["pre_bias"].abs() if "pre_bias" in p else my)


def check_forward(w, t, how, block, dtype, wide):
    p = {k: v.double() for k, v in t.items()}
    y, z, stats = w.residual_norm(block, t["x"], t.get("residual"), t.get("gate"))
    want_y, want_z = formula(p, how)
    mag_z, mag_y = magnitudes(p, how, want_z)
    assert z.dtype == wide
    within(z, want_z, rounded(want_z, mag_z, K, wide), "z")
    if want_y is None:
        assert y is None
    else:
        assert y.dtype == dtype
        within(y, want_y, rounded(want_y, mag_y, K, dtype), "y")
    mx, rx = stats_of(p["x"], how["post_norm"])
    mz, rz = stats_of(want_z, how["pre_norm"])
    want = torch.cat([mx, rx, mz, rz], 1)
    sx = p["x"].abs().mean(1, keepdim=True)
    sz = mag_z.mean(1, keepdim=True)
    ez = (mag_z.square().mean(1, keepdim=True)).sqrt() * rz  # relative, of the deviation
    ex = (p["x"].square().mean(1, keepdim=True)).sqrt() * rx
    within(stats, want, K * U * torch.cat([sx, rx * (1 + ex), sz, rz * (1 + ez)], 1), "stats")
    return y, z, stats


def check_gradient(w, t, how, block, dtype, wide, z, stats, g):
    """The gradient's formulas in 64 bits, from what the forward pass gave."""
    n, d = t["x"].shape
    dy = rand(g, n, d, dtype=dtype) if block.pre else None
    dz = rand(g, n, d, dtype=wide)
    got = w.residual_norm_grad(block, dy, dz, t["x"], z, stats, t.get("gate"), residual="residual" in t)
    st = stats.double()
    mx, rx, mz, rz = st.split(1, 1)
    one, zero = torch.ones(1, d, dtype=torch.float64, device="cuda"), torch.zeros(1, d, dtype=torch.float64, device="cuda")
    p = {k: v.double() for k, v in t.items()}
    D, mD = dz.double(), dz.double().abs()
    want, mag = {}, {}

    def through(gv, mg, h, r, kind):
        """A norm's gradient and its magnitude."""
        if kind == "none":
            return gv, mg
        a, ma = (gv * h).mean(1, keepdim=True), (mg * h.abs()).mean(1, keepdim=True)
        b, mb = (gv.mean(1, keepdim=True), mg.mean(1, keepdim=True)) if kind == "layer" else (0.0, 0.0)
        return r * (gv - b - h * a), r * (mg + mb + h.abs() * ma)

    if block.pre:
        zh = (z.double() - mz) * rz
        mzh = (z.double().abs() + mz.abs()) * rz
        gy = dy.double() * p.get("pre_weight", one)
        D2, m2 = through(gy, gy.abs() * (mzh / zh.abs().clamp(min=1e-30)).clamp(max=1.0) + gy.abs(), zh, rz, how["pre_norm"])
        # what (z - mz) loses by cancellation
        D, mD = D + D2, mD + m2 + rz * mzh * (gy * zh).abs().mean(1, keepdim=True) + rz * zh.abs() * (gy.abs() * mzh).mean(1, keepdim=True)
        if "pre_weight" in p:
            want["dpre_weight"], mag["dpre_weight"] = (dy.double() * zh).sum(0), (dy.double().abs() * mzh).sum(0)
        if "pre_bias" in p:
            want["dpre_bias"], mag["dpre_bias"] = dy.double().sum(0), dy.double().abs().sum(0)
    if "residual" in p:
        want["dresidual"], mag["dresidual"] = how["residual_scale"] * D, how["residual_scale"] * mD
    e, me = how["block_scale"] * D, how["block_scale"] * mD
    xh, mxh = (p["x"] - mx) * rx, (p["x"].abs() + mx.abs()) * rx
    if "gate" in p:
        gate = p["gate"].clone().requires_grad_()
        act = act_of(gate, how["gate"])
        slope, = torch.autograd.grad(act.sum(), gate)
        u = xh * p.get("post_weight", one) + p.get("post_bias", zero)
        mu = mxh * p.get("post_weight", one).abs() + p.get("post_bias", zero).abs()
        want["dgate"] = e * u * slope
        # silu's slope: sig (1 + g (1 - sig))
        mag["dgate"] = (me * u.abs() + e.abs() * mu) * (slope.abs() if how["gate"] != "silu" else 1 + gate.detach().abs())
        act = act.detach()
        e, me = e * act, me * act.abs()
    if "post_weight" in p:
        want["dpost_weight"], mag["dpost_weight"] = (e * xh).sum(0), (me * mxh).sum(0)
    if "post_bias" in p:
        want["dpost_bias"], mag["dpost_bias"] = e.sum(0), me.sum(0)
    wq = p.get("post_weight", one)
    want["dx"], mdx = through(e * wq, me * wq.abs(), xh, rx, how["post_norm"])
    if how["post_norm"] != "none":
        gu = (me * wq).abs()
        mdx = mdx + rx * mxh * (gu * xh.abs()).mean(1, keepdim=True) + rx * xh.abs() * (gu * mxh).mean(1, keepdim=True)
    mag["dx"] = mdx
    assert set(got) == set(want)
    for k in want:
        kind = got[k].dtype
        within(got[k], want[k], rounded(want[k], mag[k], (4 if k.startswith(("dpost", "dpre")) else 2) * K, kind), k)
    return got, dy, dz


SHAPES = [(1, 1, 0, 0), (3, 7, 0, 0), (5, 32, 0, 0), (2, 33, 3, 1), (64, 256, 0, 0), (17, 257, 0, 0), (40, 1001, 3, 1),
          (9, 1024, 8, 8), (700, 136, 0, 0), (5, 2056, 0, 0), (5, 4096, 0, 0), (3, 5001, 0, 0), (2, 8192, 0, 0),
          (3, 8200, 0, 0), (1, 16_384, 0, 0), (2, 20_011, 1, 0), (2, 20_016, 0, 0)]
HOWS = [("rms", "rms", "silu"), ("layer", "layer", "sigmoid"), ("none", "layer", "none"), ("rms", "none", "mul"),
        ("none", "rms", "none"), ("layer", "rms", "silu")]


@pytest.mark.parametrize("wide", ["same", "f32"])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d,extra,offset", SHAPES)
def test_residual_norm_and_its_gradient(w, dtype, wide, n, d, extra, offset):
    if wide == "f32" and dtype == torch.float32:
        pytest.skip("the same")
    wide = dtype if wide == "same" else torch.float32
    for i, (post, pre, gate) in enumerate(HOWS):
        if d == 1 and (post == "layer" or pre == "layer"):
            continue  # a row of one column minus its mean is nothing but rounding, 1/sqrt(eps) times
        g = gen(n * d + i)
        ptype = dtype if i % 2 else torch.float32
        t, how, block = make(g, n, d, dtype, wide, post, pre, gate, ptype, extra, offset, weights=i != 4,
                             residual=i not in (3,))
        if i == 3 and wide != dtype:
            continue  # without a residual the sum has x's type unless asked
        _, z, stats = check_forward(w, t, how, block, dtype, wide)
        check_gradient(w, t, how, block, dtype, wide, z, stats, g)


@pytest.mark.parametrize("n,d,dtype,post", [(100_000, 64, torch.bfloat16, "layer"), (30_000, 520, torch.bfloat16, "layer"),
                                            (20_000, 301, torch.float32, "layer"), (3_000_000, 8, torch.float32, "layer"),
                                            (9_000, 2048, torch.float16, "rms")])
def test_many_rows(w, n, d, dtype, post):
    """More rows than blocks, and (the last) more than a thread adds in one chain: the bounds of
    the parameters' gradients do not grow with the rows."""
    g = gen(d)
    t, how, block = make(g, n, d, dtype, dtype, post, "rms", "silu")
    _, z, stats = check_forward(w, t, how, block, dtype, dtype)
    check_gradient(w, t, how, block, dtype, dtype, z, stats, g)


def test_a_chain_of_equal_rows_keeps_its_digits(w):
    """6 10^6 equal rows: a plain chain of float32 sums would be off by far more than one of at
    most 512 rows, joined with compensation: 512 U + a few."""
    n, d = 6_000_000, 8
    x = torch.full((n, d), 1.1, device="cuda")
    dz = torch.full((n, d), 0.3, device="cuda")
    weight = torch.ones(d, device="cuda")
    block = B.residual_norm(post_weight=weight)
    _, z, stats = w.residual_norm(block, x)
    got = w.residual_norm_grad(block, None, dz, x, None, stats, residual=False)["dpost_weight"]
    want = x[0].double() * dz[0].double() * n
    within(got, want, (512 + 24) * U * want, "sum")


@pytest.mark.parametrize("d", [72, 1001, 4096, 9000])
def test_in_place_and_kept_or_not(w, d):
    """z in the residual, dresidual's z gone, no z at all: the same bits."""
    g = gen(d)
    t, how, block = make(g, 33, d, torch.bfloat16, torch.float32, "rms", "layer", "silu")
    y, z, stats = w.residual_norm(block, t["x"], t["residual"], t["gate"])
    y2, none, stats2 = w.residual_norm(block, t["x"], t["residual"], t["gate"], keep_sum=False)
    assert none is None and torch.equal(y, y2) and torch.equal(stats, stats2)
    stream = t["residual"].clone()
    y3, z3, _ = w.residual_norm(block, t["x"], stream, t["gate"], sum_out=stream)
    assert z3 is stream and torch.equal(y, y3) and torch.equal(z, stream)
    dy, dz = rand(g, 33, d, dtype=torch.bfloat16), rand(g, 33, d)
    a = w.residual_norm_grad(block, dy, dz, t["x"], z, stats, t["gate"])
    b = w.residual_norm_grad(block, dy, dz, t["x"], z, stats, t["gate"])
    c = w.residual_norm_grad(block, dy, dz, t["x"], z, stats, t["gate"], residual=False)
    assert all(torch.equal(a[k], b[k]) for k in a) and "dresidual" not in c
    assert all(torch.equal(a[k], c[k]) for k in c)
    # dresidual in dz's place, by the C call
    at = dz.clone()
    dx, dg = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    w._call("gba_residual_norm_grad", block.block, B._matrix(dy), B._matrix(at), B._matrix(t["x"]), B._matrix(z),
            B._matrix(t["gate"]), stats.data_ptr(), B._matrix(dx), B._matrix(at), B._matrix(dg), None)
    assert torch.equal(at, a["dresidual"]) and torch.equal(dx, a["dx"]) and torch.equal(dg, a["dgate"])


def test_shapes_types_and_no_rows(w):
    g = gen(1)
    x, r = rand(g, 12, 40, dtype=torch.bfloat16).view(3, 4, 40), rand(g, 12, 40).view(3, 4, 40)
    block = B.residual_norm(pre_norm="rms")
    y, z, stats = w.residual_norm(block, x, r)
    assert y.shape == z.shape == x.shape and z.dtype == torch.float32 and stats.shape == (12, 4)
    got = w.residual_norm_grad(block, y, None, x, z, stats)
    assert got["dx"].shape == x.shape and got["dresidual"].dtype == torch.float32
    assert w.residual_norm(B.residual_norm(), x, sum_dtype=torch.float32)[1].dtype == torch.float32
    wide = r.expand(3, 4, 40).transpose(0, 1)
    assert torch.equal(w.residual_norm(block, x.transpose(0, 1), wide)[0], y.transpose(0, 1))
    e = x[:0]
    y, z, stats = w.residual_norm(block, e, r[:0])
    weight = torch.ones(40, device="cuda")
    got = w.residual_norm_grad(B.residual_norm(pre_norm="rms", pre_weight=weight), y, z, e, z, stats)
    assert y.shape == z.shape == e.shape and not got["dpre_weight"].any()


@pytest.mark.parametrize("d", [24, 1003, 9001])
def test_infinities_and_nan_stay_in_their_rows(w, d):
    g = gen(d)
    t, how, block = make(g, 12, d, torch.float32, torch.float32, "layer", "rms", "silu")
    good = w.residual_norm(block, t["x"], t["residual"], t["gate"])
    dy, dz = rand(g, 12, d), rand(g, 12, d)
    back = w.residual_norm_grad(block, dy, dz, t["x"], good[1], good[2], t["gate"])
    for k, v in (("x", math.nan), ("residual", math.inf), ("gate", math.nan)):
        bad = {n: m.clone() for n, m in t.items()}
        bad[k][5, d // 2] = v
        y, z, stats = w.residual_norm(block, bad["x"], bad["residual"], bad["gate"])
        rest = torch.arange(12, device="cuda") != 5
        for a, b in zip((y, z, stats), good):
            assert torch.equal(a[rest], b[rest])
        assert not z[5, d // 2].isfinite() and y[5].isnan().any()
        got = w.residual_norm_grad(block, dy, dz, bad["x"], z, stats, bad["gate"])
        assert all(torch.equal(got[n][rest], back[n][rest]) for n in ("dx", "dresidual", "dgate"))
        assert got["dx"][5].isnan().any()


@pytest.mark.parametrize("gate", ["mul", "sigmoid", "silu"])
def test_gates_at_the_ends_of_their_range(w, gate):
    v = torch.tensor([[0.0, -0.0, 88.0, -88.0, 200.0, -200.0, 3e38, -3e38, 1e-30, math.inf, -math.inf, math.nan]],
                     device="cuda")
    x = torch.full_like(v, 2.0)
    block = B.residual_norm(gate=gate)
    z = w.residual_norm(block, x, gate=v)[1]
    want = 2.0 * act_of(v.double(), gate)
    finite = want.float().isfinite()
    assert torch.equal(z.isnan(), want.isnan())
    assert torch.equal(z[want.isinf()], want[want.isinf()].float())
    within(z[finite], want[finite], 16 * U * want[finite].abs() + 1e-37, "act")  # exp below 2^-126 is 0
    stats = torch.tensor([[0.0, 1.0, 0.0, 1.0]], device="cuda")
    got = w.residual_norm_grad(block, None, torch.ones_like(v), x, None, stats, gate=v, residual=False)
    gv = v[:, :9].double().requires_grad_()
    want, = torch.autograd.grad(2.0 * act_of(gv, gate).sum(), gv)
    within(got["dgate"][:, :9], want, 2e-35 + 16 * U * (1 + gv.detach().abs().clamp(max=100)), "slope")


def test_gradient_against_differences(w):
    """The loss <y, dy> + <z, dz> along a direction, by central differences of the forward pass:
    what they are off by their step is their own change from h to 2h, and rounding adds
    K U / h for each value of the sums."""
    g = gen(3)
    n, d = 6, 96
    t, how, block = make(g, n, d, torch.float32, torch.float32, "layer", "rms", "silu")
    dy, dz = rand(g, n, d), rand(g, n, d)
    y, z, stats = w.residual_norm(block, t["x"], t["residual"], t["gate"])
    got = w.residual_norm_grad(block, dy, dz, t["x"], z, stats, t["gate"])
    names = {"x": "dx", "residual": "dresidual", "gate": "dgate", "post_weight": "dpost_weight", "post_bias": "dpost_bias",
             "pre_weight": "dpre_weight"}

    def loss(at):
        b = B.residual_norm(eps=EPS, **how, **{k: at[k] for k in at if k.startswith(("post", "pre"))})
        y, z, _ = w.residual_norm(b, at["x"], at["residual"], at["gate"])
        return float((y.double() * dy.double()).sum() + (z.double() * dz.double()).sum())

    weight = float((y.abs() * dy.abs()).double().sum() + (z.abs() * dz.abs()).double().sum())
    for k, dk in names.items():
        way = torch.sign(rand(g, *t[k].shape)) if t[k].dim() == 2 else torch.sign(rand(g, t[k].shape[0]))
        slope = float((got[dk].double() * way.double()).sum())

        def difference(h):
            up, down = dict(t), dict(t)
            up[k], down[k] = t[k] + h * way, t[k] - h * way
            step = (up[k].double() - down[k].double()) * way.double()  # as it was rounded
            return (loss(up) - loss(down)) / float(step.mean())

        h = 2.0**-7
        one, two = difference(h), difference(2 * h)
        assert abs(one - slope) <= abs(two - one) + K * U * weight / h, k


# ---- gated scan ---------------------------------------------------------------------------

def lay_out(kind, n, rows, seed):
    """The first row and length of each sequence, and what sequences() takes."""
    cpu = torch.Generator().manual_seed(seed)
    if kind == "packed":
        used = rows - rows // 10
        cuts, _ = torch.sort(torch.randint(0, used + 1, (n - 1,), generator=cpu))
        cuts = [0] + cuts.tolist() + [used]
        return cuts[:-1], [b - a for a, b in zip(cuts, cuts[1:])], dict(offsets=torch.tensor(cuts, device="cuda"))
    each = rows // n
    first = [i * each for i in range(n)]
    if kind == "equal":
        return first, [each] * n, {}
    length = torch.randint(0, each + 1, (n,), generator=cpu).tolist()
    return first, length, dict(lengths=torch.tensor(length, device="cuda"))


def decays(f, decay):
    if decay == "log":
        f = f.clamp(max=0.0)
        return f.exp(), -torch.expm1(f)
    return torch.sigmoid(f), torch.sigmoid(-f)


def recurrence(a, b, entry, back=False):
    """v = a v + b along the rows (from the last with back), starting anew, from b, at an entry: by
    doubling, in 64 bits."""
    a, b = torch.where(entry[:, None], 0.0, a), b.clone()
    n, k = a.shape[0], 1
    while k < n:
        here, there = (slice(0, n - k), slice(k, n)) if back else (slice(k, n), slice(0, n - k))
        more, less = a[here] * b[there], a[here] * a[there]
        b[here] += more
        a[here] = less
        k *= 2
    return b


def where_rows(first, length, rows):
    """The rows that are first and last in a sequence that is not empty, those sequences, and
    which rows belong to one."""
    F, Ln = torch.tensor(first, device="cuda"), torch.tensor(length, device="cuda")
    on = (Ln > 0).nonzero().view(-1)
    inside = torch.zeros(rows + 1, dtype=torch.int64, device="cuda")
    inside.index_add_(0, F[on], torch.ones_like(on))
    inside.index_add_(0, F[on] + Ln[on], -torch.ones_like(on))
    return F[on], F[on] + Ln[on] - 1, on, inside.cumsum(0)[:-1] > 0


def flags(at, rows, inside):
    e = ~inside
    e[at] = True
    return e


def gate_units(f, a, rest, decay):
    """How far a gate's decay and one minus it may be off, of themselves, in units of U.  With
    t = exp(-f) from the hardware's power of two, which is off by 2^-22 of itself (4 U), and a
    rounded argument (|f| U): a = 1/(1+t) by t/(1+t) = 1-a times that, and t a by 1/(1+t) = a
    times it, with 4 for the sum, the quotient and the product; exp(f) by all of it, and
    1 - exp(f) by CUDA's expm1f within 2."""
    own = f.abs().clamp(max=100.0) + 4.0
    if decay == "log":
        return own + 1.0, torch.where(f < -0.69, own * a / rest + 1.0, 4.0)
    return own * rest + 4.0, own * a + 4.0


def plain_scan(x, f, first, length, decay, tied, state):
    """(y, last) in 64 bits, with the bound of their rounding in units of U: a step passes on what
    was off, times the decay, and adds what its gates are off and four roundings (of the input, of
    its own sum, and of the pairs that it is joined through)."""
    f = f.double()
    a, rest = decays(f, decay)
    ua, ub = gate_units(f, a, rest, decay)
    b = rest * x.double() if tied else x.double()
    rows, d = x.shape
    begin, end, on, inside = where_rows(first, length, rows)
    last = torch.zeros(len(first), d, dtype=torch.float64, device="cuda") if state is None else state.double().clone()
    b = torch.where(inside[:, None], b, 0.0)
    own = b.abs()
    mb = own.clone()
    b[begin] += a[begin] * last[on]
    mb[begin] += a[begin] * last[on].abs()
    entry = flags(begin, rows, inside)
    y, m = recurrence(a, b, entry), recurrence(a, mb, entry)
    more = ua * (m - own) + (ub * own if tied else 0.0) + 4.0 * m
    off = recurrence(a, torch.where(inside[:, None], more, 0.0), entry)
    last[on] = y[end]
    e = torch.zeros_like(last)
    e[on] = off[end]
    return y, last, off, e


def plain_scan_grad(dy, x, f, y, first, length, decay, tied, state, dlast):
    f = f.double()
    a, rest = decays(f, decay)
    ua, ub = gate_units(f, a, rest, decay)
    rows, d = x.shape
    begin, end, on, inside = where_rows(first, length, rows)
    own = inside[:, None]
    a, ua = torch.where(own, a, 0.0), torch.where(own, ua, 0.0)
    S = torch.zeros(len(first), d, dtype=torch.float64, device="cuda") if dlast is None else dlast.double().clone()
    G = torch.where(own, dy.double(), 0.0)
    mG = G.abs()
    G[end] += S[on]
    mG[end] += S[on].abs()
    entry = flags(end, rows, inside)
    # what the next row's gradient comes here through
    nothing = torch.zeros_like(a[:1])
    after, uafter = torch.cat([a[1:], nothing]), torch.cat([ua[1:], nothing])
    G, mG = recurrence(after, G, entry, True), recurrence(after, mG, entry, True)
    passed = torch.where(entry[:, None], 0.0, after * torch.cat([mG[1:], nothing]))
    eG = recurrence(after, uafter * passed + 4.0 * mG, entry, True)
    h = torch.cat([nothing, y[:-1].double()])
    h[begin] = 0.0 if state is None else state.double()[on]
    mh = h.abs()
    if tied:
        h, mh = h - x.double(), mh + x.double().abs()
    s = a * rest if decay == "sigmoid" else torch.where(f > 0, 0.0, a)
    us = ua + ub if decay == "sigmoid" else ua
    r, ur = (rest, ub) if tied else (torch.ones_like(G), 0.0)
    out = {"dx": G * r, "ex": eG * r + (ur + 2.0) * mG * r, "df": G * h * s, "ef": eG * h.abs() * s + (us + 5.0) * mG * mh * s}
    out = {k: torch.where(own, v, 0.0) for k, v in out.items()}
    e = torch.zeros_like(S)
    S[on] = (a * G)[begin]
    e[on] = (a * eG + (ua + 2.0) * a * mG)[begin]
    return out, S, e


def check_scan(w, kind, n, rows, d, dtype, decay, tied, with_state, out=None, extra=0, offset=0, mean=2.0, grad=True):
    g = gen(n * 7 + rows + d)
    first, length, how = lay_out(kind, n, rows, rows + n)
    seq = B.sequences(n, **how)
    x = rand(g, rows, d, dtype=dtype, extra=extra, offset=offset)
    f = rand(g, rows, d, dtype=dtype, std=2.0, mean=mean if decay == "sigmoid" else -1.0, extra=extra, offset=offset)
    state = rand(g, n, d) if with_state else None
    inside = torch.zeros(rows, dtype=torch.bool)
    for a, k in zip(first, length):
        inside[a:a + k] = True
    inside = inside.cuda()
    x[~inside], f[~inside] = math.nan, math.nan
    out = out or dtype
    y, last = w.gated_scan(x, f, seq, decay=decay, tied=tied, state=state, dtype=out)
    want, h, off, e = plain_scan(torch.where(inside[:, None], x, 0), torch.where(inside[:, None], f, 0), first, length,
                                 decay, tied, state)
    assert y.dtype == out and not y[~inside].any()
    within(y, want, UNIT[out] * want.abs() * (1 + 64 * U) + U * off + TINY[out], "y")
    within(last, h, U * h.abs() + U * e, "last")
    again = w.gated_scan(x, f, seq, decay=decay, tied=tied, state=state, dtype=out)
    assert torch.equal(y, again[0]) and torch.equal(last, again[1])
    if not grad:
        return
    dy = rand(g, rows, d, dtype=out)
    dlast = rand(g, n, d) if with_state or n % 2 else None
    dy[~inside] = math.nan
    y[~inside] = math.nan
    got = w.gated_scan_grad(dy, x, f, y, seq, decay=decay, tied=tied, state=state, dstate=dlast)
    z = {k: torch.where(inside[:, None], v, 0) for k, v in dict(dy=dy, x=x, f=f, y=y).items()}
    want, S, e = plain_scan_grad(z["dy"], z["x"], z["f"], z["y"], first, length, decay, tied, state, dlast)
    for k, ek, v in (("dx", "ex", got[0]), ("df", "ef", got[1])):
        assert v.dtype == dtype and not v[~inside].any()
        within(v, want[k], UNIT[dtype] * want[k].abs() * (1 + 64 * U) + U * want[ek] + TINY[dtype], k)
    if state is None:
        assert got[2] is None
    else:
        within(got[2], S, U * S.abs() + U * e, "dstate")
    again = w.gated_scan_grad(dy, x, f, y, seq, decay=decay, tied=tied, state=state, dstate=dlast)
    assert all(a is b or torch.equal(a, b) for a, b in zip(got, again))


LAYOUTS = [("equal", 1, 1), ("equal", 5, 5), ("equal", 300, 300), ("equal", 3, 21), ("equal", 1, 64), ("equal", 2, 130),
           ("equal", 1, 2047), ("equal", 33, 33 * 64), ("equal", 7, 7 * 65), ("padded", 1, 9), ("padded", 6, 6 * 50),
           ("padded", 40, 40 * 33), ("packed", 1, 12), ("packed", 9, 200), ("packed", 60, 1500), ("packed", 700, 650)]
GATES = [("sigmoid", True, False), ("sigmoid", False, True), ("log", True, True), ("log", False, False)]


@pytest.mark.parametrize("d", [1, 3, 8, 20, 64, 132, 33, 200])
@pytest.mark.parametrize("kind,n,rows", LAYOUTS)
def test_gated_scan_and_its_gradient(w, kind, n, rows, d):
    for i, (decay, tied, state) in enumerate(GATES):
        check_scan(w, kind, n, rows, d, TYPES[(i + d) % 3], decay, tied, state)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("d,extra,offset", [(40, 0, 0), (40, 8, 8), (40, 3, 0), (40, 0, 1), (41, 0, 0), (7, 1, 2)])
def test_rows_anywhere_and_float32_outputs(w, dtype, d, extra, offset):
    check_scan(w, "packed", 11, 400, d, dtype, "sigmoid", True, True, out=torch.float32, extra=extra, offset=offset)
    check_scan(w, "equal", 4, 400, d, dtype, "log", False, True, extra=extra, offset=offset)


@pytest.mark.parametrize("kind,n,rows,d", [("equal", 1, 40_000, 8), ("equal", 1, 9_000, 132), ("packed", 3, 70_000, 4),
                                           ("padded", 2, 50_000, 12), ("equal", 1, 12_000, 1), ("packed", 500, 20_000, 136)])
def test_long_sequences(w, kind, n, rows, d):
    """Over groups of tiles, groups of groups and those one after another."""
    check_scan(w, kind, n, rows, d, torch.float32, "sigmoid", True, True, mean=5.0)
    check_scan(w, kind, n, rows, d, torch.bfloat16, "log", False, False)


@pytest.mark.parametrize("kind,n,rows,d", [("equal", 2, 60_000, 1024), ("packed", 100, 50_000, 1020),
                                           ("equal", 16, 16 * 1001, 2044), ("equal", 300, 300 * 130, 132)])
def test_many_tiles(w, kind, n, rows, d):
    check_scan(w, kind, n, rows, d, torch.bfloat16, "sigmoid", True, True, mean=4.0)


@pytest.mark.parametrize("kind,n,rows,d", [("equal", 64, 64 * 70, 1024), ("packed", 40, 9000, 501), ("padded", 20, 20 * 150, 516)])
def test_many_sequences_in_float32(w, kind, n, rows, d):
    for dtype, out in ((torch.float32, None), (torch.bfloat16, torch.float32)):
        check_scan(w, kind, n, rows, d, dtype, "sigmoid", True, True, out=out, mean=4.0)


@pytest.mark.parametrize("n,d", [(1, 64), (33, 1024), (256, 77)])
def test_steps_with_the_state_in_place_follow_the_sequence(w, n, d):
    """A sequence a row at a time gives what it gives at once, within the rounding of both."""
    g, rows = gen(n), 12
    x, f, s0 = rand(g, n * rows, d).view(n, rows, d), rand(g, n * rows, d, mean=1.0).view(n, rows, d), rand(g, n, d)
    seq, one = B.sequences(n), B.sequences(n)
    y, last = w.gated_scan(x, f, seq, state=s0)
    state = s0.clone()
    _, _, off, e = plain_scan(x.reshape(-1, d), f.reshape(-1, d), [i * rows for i in range(n)], [rows] * n, "sigmoid", True, s0)
    for t in range(rows):
        yt, st = w.gated_scan(x[:, t:t + 1], f[:, t:t + 1], one, state=state, state_out=state)
        assert st is state and yt.shape == (n, 1, d)
        within(yt[:, 0], y[:, t], 2 * U * off.view(n, rows, d)[:, t], "step")
    within(state, last, 2 * U * e, "state")
    # and through a longer call, in place
    state = s0.clone()
    w.gated_scan(x, f, seq, state=state, state_out=state)
    assert torch.equal(state, last)
    ds = rand(g, n, d)
    dy = rand(g, n * rows, d).view(n, rows, d)
    dx, df, dstate = w.gated_scan_grad(dy, x, f, y, seq, state=s0, dstate=ds)
    at = ds.clone()
    dx2, df2 = torch.empty_like(dx), torch.empty_like(df)
    m = lambda t: B._matrix(t.view(-1, d))  # noqa: E731
    w._call("gba_gated_scan_grad", B.gba_scan(0, 1, n, None, None), m(dy), m(at), m(x), m(f), m(s0), m(y), m(dx2), m(df2),
            m(at))
    assert torch.equal(at, dstate) and torch.equal(dx, dx2) and torch.equal(df, df2)


@pytest.mark.parametrize("d", [64, 513])
@pytest.mark.parametrize("n,rows,kind", [(1, 60_000, "equal"), (2, 30_001, "packed"), (700, 5, "equal"), (300, 40, "packed")])
def test_states_in_place_of_split_and_of_short_sequences(w, n, rows, kind, d):
    """A sequence whose rows several blocks, or several warps of one, go through: the state that one of them
    writes is not read by another."""
    g = gen(d + n)
    total = n * rows
    x, f, dy = rand(g, total, d), rand(g, total, d, mean=2.0), rand(g, total, d)
    s0, ds = rand(g, n, d), rand(g, n, d)
    if kind == "equal":
        seq, x, f, dy = B.sequences(n), x.view(n, rows, d), f.view(n, rows, d), dy.view(n, rows, d)
        offsets = None
    else:
        offsets = torch.tensor([0] + [i * rows + (i * 7) % rows for i in range(1, n)] + [total], device="cuda")
        seq = B.sequences(n, offsets=offsets)
    y, last = w.gated_scan(x, f, seq, state=s0)
    dx, df, dstate = w.gated_scan_grad(dy, x, f, y, seq, state=s0, dstate=ds)
    m = lambda t: B._matrix(t.view(-1, d))  # noqa: E731
    for _ in range(3):
        state = s0.clone()
        y2, st = w.gated_scan(x, f, seq, state=state, state_out=state)
        assert st is state and torch.equal(state, last) and torch.equal(y, y2)
        at = ds.clone()
        dx2, df2 = torch.empty_like(dx), torch.empty_like(df)
        w._call("gba_gated_scan_grad", B.gba_scan(0, 1, n, None, None if offsets is None else offsets.data_ptr()), m(dy),
                m(at), m(x), m(f), m(s0), m(y), m(dx2), m(df2), m(at))
        assert torch.equal(at, dstate) and torch.equal(dx, dx2) and torch.equal(df, df2)


@pytest.mark.parametrize("d", [8, 33])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_infinities_and_nan_stay_in_their_sequence(w, d, value):
    g = gen(d)
    n, each = 9, 300
    x, f = rand(g, n * each, d), rand(g, n * each, d, mean=2.0)
    s0, dy = rand(g, n, d), rand(g, n * each, d)
    seq = B.sequences(n)
    y, last = w.gated_scan(x, f, seq, state=s0)
    grads = w.gated_scan_grad(dy, x, f, y, seq, state=s0, dstate=s0)
    row, col = 4 * each + 170, d // 2
    touched = torch.zeros(n * each, d, dtype=torch.bool, device="cuda")
    touched[row:5 * each, col] = True
    for into in ("x", "state", "dy"):
        bx, bs, bd = x.clone(), s0.clone(), dy.clone()
        where = touched.clone()
        if into == "x":
            bx[row, col] = value
        elif into == "state":
            bs[4, col] = value
            where[4 * each:5 * each, col] = True
        if into != "dy":
            y2, last2 = w.gated_scan(bx, f, seq, state=bs)
            assert torch.equal(y2[~where], y[~where])
            assert not y2[where].isfinite().any()
            keep = torch.ones_like(last, dtype=torch.bool)
            keep[4, col] = False
            assert torch.equal(last2[keep], last[keep]) and not last2[~keep].isfinite().any()
        else:
            bd[row, col] = value
            dx, df, ds = w.gated_scan_grad(bd, x, f, y, seq, state=s0, dstate=s0)
            where = torch.zeros_like(touched)
            where[4 * each:row + 1, col] = True
            assert torch.equal(dx[~where], grads[0][~where]) and torch.equal(df[~where], grads[1][~where])
            assert not dx[where].isfinite().any() and not ds[4, col].isfinite()


def test_gates_of_the_scan_at_the_ends_of_their_range(w):
    v = [0.0, -0.0, 100.0, -100.0, 3e38, -3e38, math.inf, -math.inf, 20.0, -20.0]
    f = torch.tensor([v, v], device="cuda").t().contiguous().t()
    x = torch.ones_like(f)
    s0 = torch.full((1, len(v)), 3.0, device="cuda")
    for decay in ("sigmoid", "log"):
        for tied in (True, False):
            y, last = w.gated_scan(x, f, B.sequences(1), decay=decay, tied=tied, state=s0)
            want, h, off, e = plain_scan(x, f, [0], [2], decay, tied, s0)
            within(y, want, U * (want.abs() + off) + 1e-36, "y")
            dx, df, ds = w.gated_scan_grad(x, x, f, y, B.sequences(1), decay=decay, tied=tied, state=s0, dstate=s0)
            want, S, e = plain_scan_grad(x, x, f, y, [0], [2], decay, tied, s0, s0)
            within(dx, want["dx"], U * (want["dx"].abs() + want["ex"]) + 1e-36, "dx")
            within(df, want["df"], U * (want["df"].abs() + want["ef"]) + 1e-36, "df")
            within(ds, S, U * (S.abs() + e) + 1e-36, "ds")


def test_no_rows_and_no_sequences(w):
    e = torch.empty(0, 8, device="cuda")
    y, last = w.gated_scan(e, e, B.sequences(0))
    assert y.shape == (0, 8) and last.shape == (0, 8)
    s0 = rand(gen(1), 3, 8)
    assert torch.equal(w.gated_scan(e, e, B.sequences(3), state=s0)[1], s0)
    assert not w.gated_scan(e, e, B.sequences(3))[1].any()
    assert torch.equal(w.gated_scan_grad(e, e, e, e, B.sequences(3), state=s0, dstate=s0)[2], s0)
    x = rand(gen(2), 5, 8)
    none = torch.zeros(4, dtype=torch.int64, device="cuda")
    y, last = w.gated_scan(x, x, B.sequences(3, offsets=none), state=s0)
    assert not y.any() and torch.equal(last, s0)


@pytest.mark.parametrize("bad", [dict(offsets=[0, 6, 4, 12]), dict(offsets=[-1, 2, 4, 12]), dict(offsets=[0, 2, 4, 13]),
                                 dict(offsets=[9, 6, 3, 0]), dict(lengths=[1, -1, 2]), dict(lengths=[1, 5, 2]),
                                 dict(offsets=[0, 2**62, 2**62, 2**62])])
def test_bad_offsets_and_lengths_are_reported_once(bad):
    w = B.Worker()
    x = rand(gen(1), 12, 8)
    s0 = rand(gen(2), 3, 8)
    how = {k: torch.tensor(v, device="cuda") for k, v in bad.items()}
    y, _ = w.gated_scan(x, x, B.sequences(3, **how), state=s0)
    w.gated_scan_grad(y, x, x, y, B.sequences(3, **how), state=s0, dstate=s0)
    with pytest.raises(B.GBAError) as e:
        w.sync()
    assert e.value.status == B.GBA_E_ARG and "offsets" in str(e.value)
    w.sync()
    good, _ = w.gated_scan(x, x, B.sequences(3), state=s0)
    w.sync()
    assert good.isfinite().all()
    w.close()


def test_scan_gradient_against_differences(w):
    """As for the norms: the loss <y, dy> + <last, dlast> along directions."""
    g = gen(5)
    n, each, d = 3, 50, 24
    seq = B.sequences(n)
    for decay, tied in (("sigmoid", True), ("log", False)):
        t = {"x": rand(g, n * each, d), "f": rand(g, n * each, d, mean=1.0 if decay == "sigmoid" else -2.0, std=0.5), "state": rand(g, n, d)}
        dy, dl = rand(g, n * each, d), rand(g, n, d)

        def run(at):
            return w.gated_scan(at["x"], at["f"], seq, decay=decay, tied=tied, state=at["state"])

        y, last = run(t)
        got = dict(zip(("x", "f", "state"), w.gated_scan_grad(dy, t["x"], t["f"], y, seq, decay=decay, tied=tied,
                                                              state=t["state"], dstate=dl)))
        _, _, off, e = plain_scan(t["x"], t["f"], [i * each for i in range(n)], [each] * n, decay, tied, t["state"])
        weight = float((off * dy.abs()).sum() + (e * dl.abs()).sum())

        def loss(at):
            y, last = run(at)
            return float((y.double() * dy.double()).sum() + (last.double() * dl.double()).sum())

        for k in t:
            way = torch.sign(rand(g, *t[k].shape))
            slope = float((got[k].double() * way.double()).sum())

            def difference(h):
                up, down = dict(t), dict(t)
                up[k], down[k] = t[k] + h * way, t[k] - h * way
                return (loss(up) - loss(down)) / float(((up[k].double() - down[k].double()) * way.double()).mean())

            h = 2.0**-6
            one, two = difference(h), difference(2 * h)
            assert abs(one - slope) <= abs(two - one) + U * weight / h, k


# ---- AdamW --------------------------------------------------------------------------------

LR, BETAS, AEPS = 2e-3, (0.9, 0.98), 1e-8


def to_m8(m):
    scale = m.abs().amax().clamp(min=2.0**-100) * (1.0 / 448.0)
    return (m * (1.0 / scale)).to(torch.float8_e4m3fn).view(torch.uint8), scale


def to_v8(v):
    scale = v.amax().clamp(min=2.0**-100) * (1.0 / 1.875)
    bits = (v * (1.0 / scale)).view(torch.int32)
    code = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - 768
    return torch.where(v > 0, code.clamp(1, 255), 0).to(torch.uint8), scale


def of_m8(c, scale):
    return c.view(torch.float8_e4m3fn).float() * scale


def of_v8(c, scale):
    return torch.where(c > 0, ((c.int() + 768) << 20).view(torch.float32), 0.0) * scale


def by_blocks(fn, *ts):
    """fn of each 256 elements; its results joined, scales as one value each."""
    outs = [fn(*p) for p in zip(*[t.split(256) if t.numel() else [t] for t in ts])]
    return [torch.cat([o[i].view(-1) for o in outs]) for i in range(len(outs[0]))] if outs else []


def read8(st, i):
    m, v = [], []
    for j, (cm, cv) in enumerate(zip(st.m[i].split(256), st.v[i].split(256))):
        m.append(of_m8(cm, st.m_scale[i][j]))
        v.append(of_v8(cv, st.v_scale[i][j]))
    return torch.cat(m), torch.cat(v)


def tensors(g, sizes, dtype, offset, std):
    out = []
    for i, k in enumerate(sizes):
        flat = torch.full((k + offset + 3,), math.nan, dtype=dtype, device="cuda")
        t = flat[offset:offset + k]
        t.copy_(torch.randn(k, generator=g, device="cuda") * std)
        out.append(t)
    return out


def check_adamw(w, sizes, wt, gt, ct, bits, offset=0, steps=3, clip=None, decay=0.1):
    g = gen(sum(sizes) + bits)
    weights = tensors(g, sizes, wt, offset, 0.05)
    copies = tensors(g, sizes, ct, offset, 0.0) if ct else None
    decays = [decay * (i % 2) for i in range(len(sizes))]
    st = B.adamw_states(weights, bits=bits, betas=BETAS, eps=AEPS, weight_decay=decays, copies=copies)
    for step in range(1, steps + 1):
        grads = tensors(g, sizes, gt, offset, 0.01)
        norm = None if clip is None else torch.tensor(2.0, device="cuda")
        c = torch.ones((), device="cuda") if clip is None else torch.tensor(clip, device="cuda") / (norm + 1e-6)
        before = [(t.clone(), *([a.clone() for a in read8(st, i)] if bits == 8 else [st.m[i].clone(), st.v[i].clone()]))
                  for i, t in enumerate(weights)]
        w.adamw(st.parts(grads), LR, norm=norm, max_norm=clip)
        values = w.adamw_values(st.parts(grads))
        assert int(st.step) == step
        for i, (w0, m, v) in enumerate(before):
            gr = grads[i].float() * c.clamp(max=1.0)
            m = m * BETAS[0] + gr * (1.0 - BETAS[0])
            v = v * BETAS[1] + gr * gr * (1.0 - BETAS[1])
            if bits == 32:
                assert torch.equal(st.m[i], m) and torch.equal(st.v[i], v)
                now = m, v
            else:
                cm, ms = by_blocks(to_m8, m)
                cv, vs = by_blocks(to_v8, v)
                assert torch.equal(st.m[i], cm) and torch.equal(st.m_scale[i], ms)
                assert torch.equal(st.v[i], cv) and torch.equal(st.v_scale[i], vs)
                assert not (cv == 0)[v > 0].any()
                now = read8(st, i)
            assert torch.equal(values[0][i], now[0]) and torch.equal(values[1][i], now[1])
            m, v = m.double(), v.double()
            move = LR * (m / (1 - BETAS[0]**step)) / ((v / (1 - BETAS[1]**step)).sqrt() + AEPS)
            want = w0.double() * (1 - LR * decays[i]) - move
            # the step size and the root's factor 6 each (their exponentials, logarithms' products
            # and quotients), the root, the denominator, the quotient and the product one each
            bound = 16 * U * move.abs() + 2 * U * w0.double().abs()
            within(weights[i], want, UNIT[wt] * want.abs() + 2 * bound + TINY[wt], "weight")
            if copies:
                within(copies[i], want, UNIT[ct] * want.abs() + 2 * bound + TINY[ct], "copy")


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("wt,gt,ct,offset,clip", [
    (torch.float32, torch.float32, None, 0, None), (torch.float32, torch.bfloat16, torch.bfloat16, 0, 0.7),
    (torch.bfloat16, torch.bfloat16, None, 1, 5.0), (torch.float16, torch.float32, torch.float32, 3, 0.0),
    (torch.float32, torch.float16, torch.float16, 2, 0.25)])
def test_adamw(w, bits, wt, gt, ct, offset, clip):
    check_adamw(w, [1, 7, 255, 256, 257, 2048, 5000, 70_001, 512], wt, gt, ct, bits, offset, clip=clip)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("many", [1, 17, 161, 900])
def test_adamw_of_many_tensors(w, bits, many):
    check_adamw(w, [1 + (37 * i) % 600 for i in range(many)], torch.float32, torch.float32, None, bits, steps=1)


def test_adamw_of_more_elements_than_blocks(w):
    check_adamw(w, [1_500_001, 1_000_000], torch.float32, torch.bfloat16, torch.bfloat16, 32, steps=1)
    check_adamw(w, [1_500_001, 1_000_000], torch.float32, torch.bfloat16, torch.bfloat16, 8, steps=1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("norm", [math.nan, math.inf])
def test_a_norm_that_is_not_finite_changes_nothing(w, bits, norm):
    g = gen(2)
    weights, grads = tensors(g, [300, 5], torch.float32, 0, 1.0), tensors(g, [300, 5], torch.float32, 0, 1.0)
    copies = tensors(g, [300, 5], torch.bfloat16, 0, 1.0)
    st = B.adamw_states(weights, bits=bits, copies=copies)
    parts = st.parts(grads)
    w.adamw(parts, LR)
    held = [t.clone() for t in (*weights, *copies, *st.m, *st.v, *(st.m_scale or []), *(st.v_scale or []), st.step)]
    w.adamw(parts, LR, norm=torch.tensor(norm, device="cuda"), max_norm=1.0)
    now = [*weights, *copies, *st.m, *st.v, *(st.m_scale or []), *(st.v_scale or []), st.step]
    assert all(torch.equal(a, b) for a, b in zip(held, now)) and int(st.step) == 1
    w.adamw(parts, LR, norm=torch.tensor(1.0, device="cuda"), max_norm=1.0)
    assert int(st.step) == 2 and not torch.equal(held[0], weights[0])


def test_states_of_both_kinds_in_one_call_and_an_empty_one(w):
    g = gen(4)
    a, b = tensors(g, [500], torch.float32, 0, 1.0), tensors(g, [700], torch.float32, 0, 1.0)
    ga, gb = tensors(g, [500], torch.float32, 0, 1.0), tensors(g, [700], torch.float32, 0, 1.0)
    alone = [[t.clone() for t in a], [t.clone() for t in b]]
    for ts, gs, bits in ((alone[0], ga, 32), (alone[1], gb, 8)):
        w.adamw(B.adamw_states(ts, bits=bits).parts(gs), LR)
    s32, s8 = B.adamw_states(a, bits=32), B.adamw_states(b, bits=8)
    p32, p8 = s32.parts(ga), s8.parts(gb)
    both = (B.gba_adamw_part * 3)(p8.array[0], B.gba_adamw_part(n=0, bits=32), p32.array[0])
    desc = B.gba_adamw_desc(LR, 0.9, 0.999, 1e-8, None, None, 0.0)
    w._call("gba_adamw", both, 3, desc, s32.step.data_ptr())
    assert torch.equal(a[0], alone[0][0]) and torch.equal(b[0], alone[1][0]) and int(s32.step) == 1
    w._call("gba_adamw", both, 0, desc, s32.step.data_ptr())
    assert int(s32.step) == 2


def test_rates_from_the_device_and_long_runs(w):
    """A learning rate read from the device is the same as the number; far steps have no
    correction left."""
    g = gen(6)
    a = tensors(g, [1000], torch.float32, 0, 1.0)
    b = [t.clone() for t in a]
    grads = tensors(g, [1000], torch.float32, 0, 1.0)
    far = torch.tensor(2**40, device="cuda")
    sa, sb = B.adamw_states(a, step=far.clone()), B.adamw_states(b, step=far.clone())
    w.adamw(sa.parts(grads), 0.25)
    w.adamw(sb.parts(grads), torch.tensor(0.25, device="cuda"))
    assert torch.equal(a[0], b[0]) and int(sa.step) == 2**40 + 1


def test_8_bit_states_over_their_whole_range(w):
    """Elements from the largest to far below what a block resolves, a block of zeros, and one of
    tiny values."""
    g = gen(8)
    size = torch.cat([2.0 ** -torch.arange(256, device="cuda").float().div(4), torch.zeros(256, device="cuda"),
                      torch.full((256,), 1e-19, device="cuda"), torch.full((100,), 1e18, device="cuda")])
    sign = torch.sign(torch.randn(size.numel(), generator=g, device="cuda"))
    weights = [torch.zeros_like(size)]
    st = B.adamw_states(weights, bits=8, betas=BETAS)
    grads = [size * sign]
    w.adamw(st.parts(grads), LR)
    m = torch.zeros_like(size) * BETAS[0] + grads[0] * (1.0 - BETAS[0])  # 0 + -0 is 0, not -0
    v = torch.zeros_like(size) * BETAS[1] + grads[0] * grads[0] * (1.0 - BETAS[1])
    for fn, x, codes, scales in ((to_m8, m, st.m[0], st.m_scale[0]), (to_v8, v, st.v[0], st.v_scale[0])):
        c, s = by_blocks(fn, x)
        assert torch.equal(codes, c) and torch.equal(scales, s)
    got_m, got_v = [t[0] for t in w.adamw_values(st.parts(grads))]
    top = slice(0, 40)  # within 2^10 of the largest: m to 2^-4 of itself, v to 2^-4
    assert float(((got_m - m).abs() / m.abs())[top].max()) <= 2.0**-4 * (1 + 1e-6)
    assert float(((got_v - v).abs() / v)[top].max()) <= 2.0**-4 * (1 + 1e-6)
    assert not got_m[256:512].any() and not got_v[256:512].any()
    assert weights[0].isfinite().all()


# ---- together -------------------------------------------------------------------------------

def one_step(w, t, block, seq, parts, lr):
    y, last = w.gated_scan(t["x"], t["f"], seq, state=t["state"])
    out, z, stats = w.residual_norm(block, y, t["residual"], t["gate"])
    back = w.residual_norm_grad(block, out, z, y, z, stats, t["gate"])
    dx, df, ds = w.gated_scan_grad(back["dx"], t["x"], t["f"], y, seq, state=t["state"], dstate=last)
    for p, k in zip(t["grads"], ("dpost_weight", "dpre_weight")):
        p.copy_(back[k])
    norm = w.grad_norm([dx, df, *t["grads"]])
    w.adamw(parts, lr, norm=norm, max_norm=1.0)
    return out, z, dx, df, ds, norm


@pytest.mark.parametrize("n,each,d", [(3, 200, 64), (40, 64, 520), (2, 3000, 33)])
def test_a_captured_block_replays_and_outlives_a_larger_call(n, each, d):
    """Forward, backward and update captured, a larger batch run (and memory of the old workspace's
    size used by others), the first replayed on new data: the bits of direct calls."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        w = B.Worker()

        def data(seed, each=each):
            g = gen(seed)
            t = {k: rand(g, n * each, d, dtype=torch.bfloat16) for k in ("x", "f", "gate")}
            t["residual"], t["state"] = rand(g, n * each, d), rand(g, n, d)
            return t

        def made():
            weights = [torch.ones(d, device="cuda"), torch.ones(d, device="cuda")]
            st = B.adamw_states(weights, bits=8)
            block = B.residual_norm(post_norm="rms", pre_norm="rms", gate="silu", post_weight=weights[0],
                                    pre_weight=weights[1])
            grads = [torch.empty(d, device="cuda") for _ in weights]
            return weights, block, st, grads

        lengths = torch.randint(0, each + 1, (n,), device="cuda")
        seq = B.sequences(n, lengths=lengths)
        lr = torch.tensor(1e-2, device="cuda")
        weights, block, st, grads = made()
        weights2, block2, st2, grads2 = made()
        t, t2 = dict(data(1), grads=grads), dict(data(1), grads=grads2)
        parts, parts2 = st.parts(grads), st2.parts(grads2)
        one_step(w, t, block, seq, parts, lr)
        one_step(w, t2, block2, seq, parts2, lr)
        w.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = one_step(w, t, block, seq, parts, lr)
        big = dict(data(2, 8 * each), grads=[torch.empty(d, device="cuda") for _ in range(2)])
        w3, b3, s3, _ = made()
        one_step(w, big, b3, B.sequences(n, lengths=8 * lengths), s3.parts(big["grads"]), lr)
        w.sync()
        others = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(32)]
        for seed in (3, 4):
            new = data(seed)
            lengths.copy_(torch.randint(0, each + 1, (n,), device="cuda"))
            lr.mul_(0.5)
            for k in new:
                t[k].copy_(new[k])
                t2[k].copy_(new[k])
            graph.replay()
            got = [v.clone() for v in out]
            for a, b in zip(got, one_step(w, t2, block2, seq, parts2, lr)):
                assert torch.equal(a, b)
            assert all(torch.equal(a, b) for a, b in zip(weights, weights2))
            assert all(torch.equal(a, b) for a, b in zip((*st.m, *st.v, st.step), (*st2.m, *st2.v, st2.step)))
        assert all(bool(o.isnan().all()) for o in others)
        w.sync()
        del graph
    w.close()


def test_calls_under_another_stream_are_ordered_with_it():
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    w = B.Worker(own)
    n, d = 4, 2048
    with torch.cuda.stream(other):
        x, f = rand(gen(1), 20_000, d, dtype=torch.bfloat16), rand(gen(2), 20_000, d, dtype=torch.bfloat16)
        seq = B.sequences(n)
        want = w.gated_scan(x, f, seq)[0].clone()
        for _ in range(5):
            late = torch.zeros_like(x)
            late.copy_(x)
            assert torch.equal(w.gated_scan(late, f, seq)[0], want)
    other.synchronize()
    w.close()
