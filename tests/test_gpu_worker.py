"""The worker's operators against plain statements in 64 bits (needs a GPU).

Tolerances are bounds of the rounding, element by element, with U = 2^-24 the unit
roundoff of float32: a sum of terms t_i in which each passes through at most k additions is
within k U sum |t_i| of the exact one (first order; k is raised by a few for the terms' own
roundings), and a result of type T is rounded once more, by at most UNIT[T] of itself."""
import math

import numpy as np
import pytest
import torch

from paper_2205_11048_gb300 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0**-24
UNIT = {torch.float32: U, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
TINY = {torch.float32: 2.0**-149, torch.bfloat16: 2.0**-133, torch.float16: 2.0**-24}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.fixture
def w():
    worker = B.Worker()
    yield worker
    worker.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rand(g, *shape, dtype=torch.float32, std=1.0, mean=0.0, extra=0, offset=0):
    """Rows with `extra` columns between them, starting `offset` elements into an allocation."""
    rows, cols = (1, shape[0]) if len(shape) == 1 else shape
    flat = torch.full((offset + rows * (cols + extra),), float("nan"), dtype=dtype, device="cuda")
    m = flat[offset:].view(rows, cols + extra)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=g, device="cuda") * std + mean)
    return m if len(shape) == 2 else m.reshape(-1)


def within(got, want, bound, what):
    got, want, bound = got.double(), want.double(), torch.as_tensor(bound, device=got.device).double()
    assert got.shape == want.shape, what
    off = (got - want).abs() - bound
    assert not torch.isnan(got).any(), what
    assert float(off.max() if off.numel() else 0.0) <= 0.0, (what, float(off.max()))


# ---- lookup ------------------------------------------------------------------------------

def plain_embed(weights, rows, scale, zero, dtype):
    """The exact product of two float32 numbers, rounded to float32 and then to dtype."""
    x = (weights.double()[rows] * float(np.float32(scale))).float()
    x[zero] = 0.0
    return x.to(dtype)


@pytest.mark.parametrize("out", TYPES, ids=IDS.get)
@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d,extra,offset", [
    (1, 1, 0, 0), (1, 1024, 0, 0), (3, 7, 0, 0), (65, 64, 0, 0), (33, 12, 4, 4), (17, 1001, 3, 1),
    (5, 4098, 0, 2), (700, 130, 6, 0), (20_000, 264, 0, 0)])
def test_embed(w, dtype, out, n, d, extra, offset):
    if dtype != torch.float32 and out not in (torch.float32, dtype):
        pytest.skip("refused (see the test of refusals)")
    g = gen(n + d)
    V = 501
    weights = rand(g, V, d, dtype=dtype, extra=extra, offset=offset)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    ids[torch.rand(n, generator=g, device="cuda") < 0.2] = -7
    to = rand(g, n, d, dtype=out, extra=extra, offset=offset)
    before = to.as_strided((n, d + extra), (d + extra, 1), max(0, offset)).clone() if n > 1 and extra else None
    w.embed(weights, ids, scale=1.7, pad_id=-7, out=to)
    w.sync()
    want = plain_embed(weights, ids.clamp(min=0), 1.7, ids == -7, out)
    assert torch.equal(to, want)
    if before is not None:  # what lies between the rows is not touched
        after = to.as_strided((n, d + extra), (d + extra, 1), max(0, offset))
        assert torch.equal(after[:-1, d:].isnan(), before[:-1, d:].isnan())


def test_embed_folds_hashed_ids_and_keeps_shapes(w):
    g = gen(1)
    weights = rand(g, 1009, 48)
    ids = torch.randint(-2**63, 2**63 - 1, (4, 5, 6), generator=g, device="cuda")
    y = w.embed(weights, ids, id_mode=B.MODULO, dtype=torch.float16)
    rows = torch.tensor([int(i) % 2**64 % 1009 for i in ids.flatten().tolist()], device="cuda")
    assert y.shape == (4, 5, 6, 48)
    assert torch.equal(y.view(-1, 48), plain_embed(weights, rows, 1.0, rows < 0, torch.float16))


def test_embed_keeps_infinities_and_nan_where_they_are(w):
    weights = torch.ones(4, 24, device="cuda")
    weights[1, 3], weights[2, 5] = float("inf"), float("nan")
    y = w.embed(weights, torch.tensor([0, 1, 2, 3, 9], device="cuda"), scale=-2.0, pad_id=9)
    want = weights * -2.0
    assert torch.equal(torch.nan_to_num(y[:4], nan=7.0), torch.nan_to_num(want, nan=7.0))
    assert torch.equal(y[4], torch.zeros(24, device="cuda"))


@pytest.mark.parametrize("bad", [-1, 10, 2**40])
def test_an_id_out_of_range_is_reported_once_and_gives_zeros(w, bad):
    weights = rand(gen(2), 10, 16)
    y = w.embed(weights, torch.tensor([3, bad, 4], device="cuda"))
    with pytest.raises(B.GBAError) as e:
        w.sync()
    assert e.value.status == B.GBA_E_ID_RANGE
    assert torch.equal(y[1], torch.zeros(16, device="cuda"))
    assert torch.equal(y[::2], weights[3:5])
    w.sync()  # and the worker goes on
    assert torch.equal(w.embed(weights, torch.tensor([bad], device="cuda"), pad_id=bad), torch.zeros(1, 16, device="cuda"))
    w.sync()


def test_rows_past_the_reach_of_32_bits(w):
    """2^22 + 3 rows of 1,024 bf16: the last rows start beyond 2^32 elements' bytes."""
    V, d = 2**22 + 3, 1024
    weights = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 2**21, 2**22, V - 1], device="cuda")
    weights[rows] = rand(gen(3), 4, d, dtype=torch.bfloat16)
    assert torch.equal(w.embed(weights, rows, scale=2.0), (weights[rows].float() * 2.0).to(torch.bfloat16))
    grad = rand(gen(4), 4, d, dtype=torch.bfloat16)
    out = torch.empty(V, d, device="cuda")
    w.embed_grad_dense(rows, grad, out)
    assert torch.equal(out[rows], grad.float())
    out[rows] = 0.0
    assert not bool(out.any())


def server(mode, rows=2003, dim=20, kind=B.ADAGRAD):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        return B.GBA([(rows, dim, mode, 4096, B.opt_desc(kind, 0.05))], 0, None, 1, 4, seed=11)


@pytest.mark.parametrize("overlap", [False, True])
@pytest.mark.parametrize("mode", [B.DIRECT, B.MODULO, B.HASH])
def test_embed_table_sees_every_step_before_it_and_none_after(w, mode, overlap):
    """The worker's stream is not the server's: the lookup takes the rows as the steps before
    left them, and a step that follows does not reach into it."""
    g = gen(5)
    srv = server(mode)
    srv.set_overlap(overlap)
    n, d = 3000, 20
    ids = torch.randint(0, 2003, (n,), generator=g, device="cuda")
    if mode != B.DIRECT:
        ids = ids * 7_777_777_777 - 2**40
    asked = torch.cat([ids[:500], ids[:1] + 1 if mode == B.HASH else ids[:1], ids[:1]])
    for step in range(4):
        rows = rand(g, n, d, std=0.1)
        torch.cuda.synchronize()
        srv.push(step, [ids], [rows], torch.empty(0, device="cuda"), 1)
        assert srv.try_apply() == 1
        y = w.embed_table(srv, 0, asked, scale=3.0, pad_id=int(ids[0]))
        srv.push(step, [ids], [rows], torch.empty(0, device="cuda"), 1)
        if step == 3:  # the last lookup is followed by a step of its own
            before = y.clone()
            assert srv.try_apply() == 1
            srv.sync()
            torch.cuda.synchronize()
            assert torch.equal(y, before)
            break
        now = srv.pull(0, asked)
        srv.sync()
        torch.cuda.synchronize()
        want = (now.double() * 3.0).float()
        want[asked == ids[0]] = 0.0
        assert torch.equal(y, want)
        assert srv.try_apply() == 1
    w.sync()
    srv.close()


def test_embed_table_refuses_the_reserved_id_and_an_id_out_of_range(w):
    for mode, bad in ((B.HASH, -2**63), (B.DIRECT, 2003), (B.DIRECT, -1)):
        srv = server(mode)
        y = w.embed_table(srv, 0, torch.tensor([5, bad], device="cuda"))
        with pytest.raises(B.GBAError) as e:
            w.sync()
        assert e.value.status == B.GBA_E_ID_RANGE
        assert torch.equal(y[1], torch.zeros(20, device="cuda")) and bool(y[0].any())
        srv.sync()  # the server is not concerned
        with pytest.raises(B.GBAError):
            w.embed_table(srv, 1, torch.tensor([5], device="cuda"))
        srv.close()


# ---- its gradient ---------------------------------------------------------------------------

def plain_grad(ids, grad, scale, pad, V):
    """(rows that occur, their sums, the sums of the absolute values, tokens of each) in 64 bits."""
    keep = ids != pad if pad is not None else torch.ones_like(ids, dtype=torch.bool)
    rows, inverse = torch.unique(ids[keep], return_inverse=True)
    x = grad[keep].double()
    sums = torch.zeros(rows.numel(), grad.shape[1], dtype=torch.float64, device="cuda")
    mags = torch.zeros_like(sums)
    sums.index_add_(0, inverse, x)
    mags.index_add_(0, inverse, x.abs())
    s = float(np.float32(scale))
    return rows, sums * s, mags * abs(s)


# a token passes through at most 127 additions in its item, and is merged with compensation
GRAD_ADDS = 127 + 4


def check_message(got, want, n):
    ids, rows, count = got
    uniq, sums, mags = want
    u = uniq.numel()
    assert int(count) == u
    assert torch.equal(ids[:u], uniq)
    within(rows[:u], sums, GRAD_ADDS * U * mags, "rows")
    assert torch.equal(ids[u:], (uniq[-1] if u else torch.tensor(-1, device="cuda")).expand(n - u))
    assert not bool(rows[u:].any())


def tokens(g, n, V, kind, pad):
    if kind == "one":
        ids = torch.full((n,), V // 2, device="cuda")
    elif kind == "distinct":
        ids = torch.randperm(max(n, V), generator=g, device="cuda")[:n] % V
    elif kind == "runs":  # sorted runs of 1 .. 200: cuts at every place of a run
        ids = torch.repeat_interleave(torch.arange(V, device="cuda"),
                                      torch.randint(1, 201, (V,), generator=g, device="cuda"))[:n]
        ids = torch.cat([ids, torch.zeros(n - ids.numel(), dtype=torch.int64, device="cuda")])
        ids = ids[torch.randperm(n, generator=g, device="cuda")]
    else:
        ids = (torch.rand(n, generator=g, device="cuda") ** 6 * V).long().clamp_(max=V - 1)
    if pad:
        ids[torch.rand(n, generator=g, device="cuda") < pad] = -1
    return ids


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d,V,kind,pad,extra,offset", [
    (1, 1, 1, "one", 0, 0, 0), (1, 64, 100, "distinct", 0, 0, 0), (2, 5, 7, "one", 0, 0, 0),
    (63, 16, 9, "skew", 0, 0, 0), (64, 16, 1, "one", 0, 0, 0), (65, 16, 1, "one", 0, 0, 0),
    (129, 24, 3, "skew", 0.3, 0, 0), (1000, 33, 50, "runs", 0, 1, 1), (2048, 8, 2, "skew", 0, 0, 0),
    (2049, 12, 40, "runs", 0.1, 4, 4), (5000, 40, 70, "runs", 0, 0, 2), (6656, 16, 100_000, "skew", 0.05, 0, 0),
    (4097, 130, 300_000, "distinct", 0, 0, 0), (20_000, 3, 1, "one", 0.5, 0, 0),
    (100_000, 20, 1000, "skew", 0, 0, 0), (300, 4104, 37, "skew", 0.2, 8, 0), (500, 16, 10, "one", 1.1, 0, 0)])
def test_embed_grad(w, dtype, n, d, V, kind, pad, extra, offset):
    check_embed_grad(w, dtype, n, d, V, kind, pad, extra, offset)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d,V,kind,pad,extra", [
    (16_000, 1024, 500, "skew", 0.1, 0), (15_001, 2056, 3000, "runs", 0, 8), (14_600, 4096, 9, "one", 0.3, 0),
    (20_000, 1536, 40_000, "distinct", 0.9, 0), (14_592, 8192, 300, "skew", 0, 0), (30_000, 528, 200, "skew", 0, 0),
    (16_000, 1024, 10, "one", 1.1, 0)])
def test_embed_grad_of_many_wide_rows(w, dtype, n, d, V, kind, pad, extra):
    """Tokens enough for every SM to take many, of rows of several slabs."""
    check_embed_grad(w, dtype, n, d, V, kind, pad, extra, 0)


def check_embed_grad(w, dtype, n, d, V, kind, pad, extra, offset):
    g = gen(n + 3 * d)
    ids = tokens(g, n, V, kind, pad)
    grad = rand(g, n, d, dtype=dtype, extra=extra, offset=offset)
    grad[ids == -1] = float("nan")  # what stands at padding is never read
    got = w.embed_grad(ids, grad, V, scale=2.5, pad_id=-1)
    want = plain_grad(ids, grad, 2.5, -1, V)
    w.sync()
    check_message(got, want, n)
    again = w.embed_grad(ids, grad, V, scale=2.5, pad_id=-1)
    for a, b in zip(got, again):
        assert torch.equal(a, b)
    out = rand(g, V, d, extra=extra, offset=offset)
    w.embed_grad_dense(ids, grad, out, scale=2.5, pad_id=-1)
    uniq, sums, mags = want
    within(out[uniq], sums, GRAD_ADDS * U * mags, "dense")
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[uniq] = False
    assert not bool(out[rest].any())
    base = rand(g, V, d)
    more = base.clone()
    w.embed_grad_dense(ids, grad, more, scale=2.5, pad_id=-1, accumulate=True)
    within(more[uniq], base.double()[uniq] + sums,
           GRAD_ADDS * U * mags + U * (base.double()[uniq].abs() + mags), "accumulated")
    assert torch.equal(more[rest], base[rest])
    w.sync()


def test_embed_grad_of_a_million_tokens_of_one_row(w):
    """Sums of 2^20 equal and of alternating gradients: many items of one run."""
    n, d = 1 << 20, 8
    ids = torch.full((n,), 3, device="cuda")
    grad = torch.full((n, d), 0.3, device="cuda")
    grad[:, 1] = 0.3 * (1 - 2 * (torch.arange(n, device="cuda") % 2))
    got = w.embed_grad(ids, grad, 5)
    check_message(got, plain_grad(ids, grad, 1.0, None, 5), n)
    w.sync()


def test_embed_grad_folds_hashed_ids(w):
    g = gen(8)
    V, n = 997, 3000
    ids = torch.randint(-2**63, 2**63 - 1, (n,), generator=g, device="cuda")
    ids[::5] = ids[0]
    ids[3::50] = -2**62
    grad = rand(g, n, 24, dtype=torch.bfloat16)
    rows = torch.tensor([int(i) % 2**64 % V for i in ids.tolist()], device="cuda")
    rows[ids == -2**62] = -1
    got = w.embed_grad(ids, grad, V, pad_id=-2**62, id_mode=B.MODULO)
    check_message(got, plain_grad(rows, grad, 1.0, -1, V), n)


@pytest.mark.parametrize("bad", [-1, 100, 2**33])
def test_embed_grad_with_an_id_out_of_range_gives_nothing(w, bad):
    ids = torch.tensor([5, bad, 7, 5], device="cuda")
    grad = torch.ones(4, 8, device="cuda")
    got, rows, count = w.embed_grad(ids, grad, 100)
    out = torch.ones(100, 8, device="cuda")
    w.embed_grad_dense(ids, grad, out, accumulate=True)
    with pytest.raises(B.GBAError) as e:
        w.sync()
    assert e.value.status == B.GBA_E_ID_RANGE
    assert int(count) == 0 and bool((got == -1).all()) and not bool(rows.any())
    assert bool((out == 1.0).all())
    check_message(w.embed_grad(ids, grad, 100, pad_id=bad), plain_grad(ids, grad, 1.0, bad, 100), 4)
    w.sync()


def test_embed_grad_keeps_infinities_and_nan_in_their_rows(w):
    ids = torch.tensor([2, 1, 2, 0, 3], device="cuda")
    grad = torch.ones(5, 16, device="cuda")
    grad[0, 3], grad[2, 3], grad[1, 5], grad[3, 0] = float("inf"), float("-inf"), float("nan"), float("inf")
    _, rows, _ = w.embed_grad(ids, grad, 4)
    want = torch.tensor([1.0, 1.0, 2.0, 1.0], device="cuda")[:, None].repeat(1, 16)
    want[0, 0], want[1, 5], want[2, 3] = float("inf"), float("nan"), float("nan")
    assert torch.equal(torch.nan_to_num(rows[:4], nan=9.0, posinf=8.0), torch.nan_to_num(want, nan=9.0, posinf=8.0))
    assert not bool(rows[4].any())


def test_embed_grad_is_the_difference_of_the_lookup(w):
    """L = sum(out * G) is linear in the weights: a step of 1 in one weight changes it by the
    gradient, up to the rounding of the two sums."""
    g = gen(9)
    V, d, n = 6, 8, 40
    weights, G = rand(g, V, d), rand(g, n, d)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda")
    out = torch.empty(V, d, device="cuda")
    w.embed_grad_dense(ids, G, out, scale=1.5, pad_id=2)
    for r in range(V):
        for c in (0, 5):
            up = weights.clone()
            up[r, c] += 1.0
            a, b = (w.embed(x, ids, scale=1.5, pad_id=2).double() for x in (up, weights))
            got = float(((a - b) * G.double()).sum())
            # each output of the row carries the rounding of the weight's step and its product
            mag = float((G.double()[(ids == r) & (ids != 2), c].abs()).sum()) * 1.5 * (1 + abs(float(up[r, c])) * 2)
            assert abs(got - float(out[r, c])) <= (GRAD_ADDS + 4) * U * mag + 1e-12


@pytest.mark.parametrize("mode", [B.DIRECT, B.MODULO])
def test_a_message_of_summed_rows_gives_the_servers_step(w, mode):
    """The n single rows, the distinct rows and all n slots are the same message."""
    g = gen(10)
    V, d, n = 2003, 20, 3000
    ids = tokens(g, n, V, "skew", 0)
    if mode == B.MODULO:
        ids = ids + V * torch.randint(0, 2**40, (n,), generator=g, device="cuda")
    rows = rand(g, n, d, std=0.1)
    sids, srows, count = w.embed_grad(ids, rows, V, id_mode=mode)
    u = int(count)
    torch.cuda.synchronize()
    tables = []
    for i, r in ((ids, rows), (sids[:u], srows[:u]), (sids, srows)):
        srv = server(mode, V, d)
        srv.push(0, [i.contiguous()], [r.contiguous()], torch.empty(0, device="cuda"), 1)
        assert srv.try_apply() == 1
        tables.append(srv.table(0))
        srv.close()
    for t in tables[1:]:
        assert torch.equal(t[3], tables[0][3])
        # Adagrad's step is at most lr = 0.05, and moves with the sum's relative error
        assert float((t[0] - tables[0][0]).abs().max()) <= 1e-5
    assert torch.equal(tables[1][0], tables[2][0])


# ---- norm and clipping -----------------------------------------------------------------------

SIZES = [[1], [0], [], [5, 0, 3], [1000], [2047, 2048, 2049], [100_003, 7, 1], [33] * 16, [9] * 17,
         [1001] * 130, [65] * 250, [3] * 2100, [3_000_001, 500]]
# 32 squares, then a square root's half, and the result's rounding
NORM_BOUND = (32 / 2 + 2) * U


def gradients(g, sizes, types, offset=0, std=0.01):
    return [rand(g, k, dtype=types[i % len(types)], std=std, offset=(offset * (i + 1)) % 8) if k
            else torch.empty(0, dtype=types[i % len(types)], device="cuda") for i, k in enumerate(sizes)]


def exact_norm(grads):
    return math.sqrt(sum(float(t.double().square().sum()) for t in grads))


@pytest.mark.parametrize("types", [[torch.float32], [torch.bfloat16], [torch.float16], TYPES],
                         ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s, default=0)}")
def test_norm_and_clipping(w, sizes, types):
    g = gen(len(sizes))
    for offset in (0, 1):
        grads = gradients(g, sizes, types, offset)
        want = exact_norm(grads)
        norm = w.grad_norm(grads)
        assert abs(float(norm) - want) <= NORM_BOUND * want
        most = 0.5 * want if want > 0 else 1.0
        coef = min(1.0, most / (want + 1e-6))
        out = [torch.full((t.numel() + offset,), 7.0, device="cuda")[offset:] for t in grads]
        same = [torch.full_like(t, 7.0) for t in grads]
        for to in (out, same):
            assert torch.equal(w.clip_grads(B.grad_parts(grads, to), most), norm)
        for t, a, b in zip(grads, out, same):
            want_t = t.double() * coef
            tol = (NORM_BOUND + 4 * U) * want_t.abs()
            within(a, want_t, tol + TINY[torch.float32], "float32 output")
            within(b, want_t, tol * 1.01 + UNIT[t.dtype] * want_t.abs() + TINY[t.dtype], "own type")
        assert torch.equal(w.clip_grads(grads, most), norm)  # in place, the same numbers
        for t, b in zip(grads, same):
            assert torch.equal(t, b)
    w.sync()


def test_gradients_within_the_norm_are_copied_or_left(w):
    grads = gradients(gen(1), [1000, 77], TYPES)
    before = [t.clone() for t in grads]
    out = [torch.zeros_like(t) for t in grads]
    w.clip_grads(B.grad_parts(grads, out), 1e9)
    w.clip_grads(grads, 1e9)
    for t, b, o in zip(grads, before, out):
        assert torch.equal(t, b) and torch.equal(o, b)
    w.clip_grads(grads, 0.0)
    assert not any(bool(t.any()) for t in grads)


@pytest.mark.parametrize("size", [3, 40, 5000])
@pytest.mark.parametrize("value", [1e-38, 1e-30, 3e-20, 1e18, 1e25, 3e35])
def test_the_norm_neither_overflows_nor_vanishes(w, value, size):
    t = rand(gen(2), size, std=1.0) * value
    t[size // 2] = value
    want = exact_norm([t])
    assert abs(float(w.grad_norm([t, torch.zeros(100, device="cuda")])) - want) <= NORM_BOUND * want + 2.0**-150


@pytest.mark.parametrize("at", [0, 7, 4099])
def test_infinities_and_nan_show_in_the_norm(w, at):
    for bad in (float("inf"), float("-inf"), float("nan")):
        t = rand(gen(3), 4100, dtype=torch.bfloat16)
        t[at] = bad
        out = torch.zeros_like(t)
        norm = float(w.clip_grads(B.grad_parts([t], [out]), 1.0))
        if math.isnan(bad):
            assert math.isnan(norm) and bool(out.isnan().all())
        else:
            assert norm == math.inf and bool(out[at].isnan())
            out[at] = 0.0
            assert not bool(out.any())


def test_two_calls_of_a_norm_give_the_same_bits(w):
    grads = gradients(gen(4), [1_000_003, 501, 77_777], TYPES)
    assert len({float(w.grad_norm(grads)) for _ in range(5)}) == 1


# ---- layer norm ---------------------------------------------------------------------------------

def depth(d):
    """Additions a column's term passes through: 16 (or its share of a wide row) in its thread,
    5 between lanes, up to 32 between warps; a few more for the terms' own roundings."""
    return 16 + d // 1024 + 5 + 32 + 4


def plain_norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    var = (x - mean).square().mean(1, keepdim=True)
    rstd = 1.0 / (var + eps).sqrt()
    h = (x - mean) * rstd
    g = 1.0 if gamma is None else gamma.double()
    b = 0.0 if beta is None else beta.double()
    return h * g + b, mean, rstd, var, g, b


WIDTHS = [(1, 1), (5, 2), (3, 16), (9, 17), (300, 64), (130, 100), (7, 1001), (33, 1024), (5, 4096), (3, 4098),
          (4, 8200), (3, 16384), (3, 16392), (2, 20_001), (1, 70_000), (5000, 24)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d", WIDTHS)
@pytest.mark.parametrize("extra,offset,own_params", [(0, 0, False), (8, 8, True), (3, 1, False)])
def test_layer_norm_and_its_gradient(w, dtype, n, d, extra, offset, own_params):
    check_layer_norm(w, dtype, n, d, extra, offset, own_params)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d,extra", [(7400, 1040, 0), (8001, 1536, 8), (5003, 2056, 0), (3700, 4096, 16), (1300, 8192, 0),
                                       (700, 16384, 0)])
def test_layer_norm_of_many_wide_rows(w, dtype, n, d, extra):
    """Rows enough for every SM to take several: they come through shared memory."""
    check_layer_norm(w, dtype, n, d, extra, extra, False)


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d", [(50, 136), (41, 150), (40, 392), (700, 432), (9, 512), (33, 600), (21, 776), (5, 78),
                                 (6, 260), (3, 1030)])
def test_layer_norm_of_rows_about_a_warp_wide(w, dtype, n, d):
    check_layer_norm(w, dtype, n, d, 0, 0, True)


def check_layer_norm(w, dtype, n, d, extra, offset, own_params):
    g = gen(n + d)
    eps = 1e-5
    x = rand(g, n, d, dtype=dtype, extra=extra, offset=offset, mean=0.5)
    x[:, ::7] *= 10.0
    ptype = dtype if own_params else torch.float32
    gamma, beta = rand(g, d, dtype=ptype, std=0.5, mean=1.0), rand(g, d, dtype=ptype)
    y, mean, rstd = w.layer_norm(x, gamma, beta, eps)
    wy, wm, wr, wv, wg, wb = plain_norm(x, gamma, beta, eps)
    k = depth(d)
    xa = x.double().abs().mean(1, keepdim=True)
    dm = (k + 2) * U * xa  # of the mean
    dr = (k / 2 + 4) * U + 0.5 * dm.square() / (wv + eps) + 2 * U * xa * wv.sqrt() / (wv + eps)  # of rstd, relative
    within(mean, wm.view(-1), dm.view(-1) + 1e-30, "mean")
    within(rstd, wr.view(-1), (dr * wr).view(-1), "rstd")
    core = (wy - wb).abs()
    tol = wg.abs() * wr * (dm + 2 * U * (x.double().abs() + wm.abs())) + (dr + 3 * U) * core + 2 * U * (core + wb.abs())
    within(y, wy, tol * 1.01 + UNIT[dtype] * wy.abs() + TINY[dtype], "y")

    # the gradient, of these means and deviations
    dy = rand(g, n, d, dtype=dtype, extra=extra, offset=offset)
    dx, dgamma, dbeta = w.layer_norm_grad(dy, x, gamma, mean, rstd)
    m, r, e = mean.double()[:, None], rstd.double()[:, None], dy.double()
    h, gg = (x.double() - m) * r, dy.double() * wg
    dh = 3 * U * r * (x.double().abs() + m.abs())
    mg, mgh = gg.mean(1, keepdim=True), (gg * h).mean(1, keepdim=True)
    want = r * (gg - mg - h * mgh)
    e_mg = (k + 2) * U * gg.abs().mean(1, keepdim=True)
    e_mgh = (k + 3) * U * (gg * h).abs().mean(1, keepdim=True) + (gg.abs() * dh).mean(1, keepdim=True)
    tol = r * (e_mg + h.abs() * e_mgh + dh * mgh.abs() + 5 * U * (gg.abs() + mg.abs() + (h * mgh).abs()))
    within(dx, want, tol * 1.01 + UNIT[dtype] * want.abs() + TINY[dtype], "dx")
    within(dbeta, e.sum(0), (n + 8) * U * e.abs().sum(0), "dbeta")
    within(dgamma, (e * h).sum(0), (n + 8) * U * (e * h).abs().sum(0) + (e.abs() * dh).sum(0), "dgamma")
    again = w.layer_norm_grad(dy, x, gamma, mean, rstd)
    for a, b in zip((dx, dgamma, dbeta), again):
        assert torch.equal(a, b)
    w.sync()


@pytest.mark.parametrize("d", [40, 1024, 9000, 20_000])
def test_layer_norm_in_place_and_without_parameters(w, d):
    x = rand(gen(d), 6, d)
    y, mean, rstd = w.layer_norm(x)
    one, zero = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")
    assert torch.equal(y, w.layer_norm(x, one, zero)[0])
    m = B._matrix(x.clone())
    check = x.clone()
    B.check(w.L.gba_layer_norm(w.h, B._matrix(check), None, None, 0, 1e-5, B._matrix(check), None, None))
    assert torch.equal(check, y) and m.rows == 6
    dy = rand(gen(d + 1), 6, d)
    dx, dgamma, dbeta = w.layer_norm_grad(dy, x, None, mean, rstd)
    dg = torch.empty(d, device="cuda")
    B.check(w.L.gba_layer_norm_grad(w.h, B._matrix(dy), B._matrix(x), None, 0, mean.data_ptr(), rstd.data_ptr(),
                                    B._matrix(dy), dg.data_ptr(), None))
    assert torch.equal(dy, dx) and torch.equal(dg, dgamma)


@pytest.mark.parametrize("mean", [0.0, 100.0, -3000.0])
def test_layer_norm_of_a_large_mean_keeps_its_digits(w, mean):
    """The squares are those of the differences: their error does not grow with mean^2."""
    x = rand(gen(6), 20, 1024, mean=mean)
    _, _, rstd = w.layer_norm(x)
    _, _, wr, wv, _, _ = plain_norm(x, None, None, 1e-5)
    xa = x.double().abs().mean(1, keepdim=True)
    dm = (depth(1024) + 2) * U * xa
    bound = ((depth(1024) / 2 + 4) * U + 0.5 * dm.square() / wv + 2 * U * xa / wv.sqrt()) * wr
    within(rstd, wr.view(-1), bound.view(-1), "rstd")


def test_layer_norm_of_equal_columns_and_of_nan(w):
    x = torch.full((3, 96), 2.5, device="cuda")
    x[1, 7], x[2, 9] = float("nan"), float("inf")
    y, mean, rstd = w.layer_norm(x, eps=1e-5)
    assert not bool(y[0].any()) and float(mean[0]) == 2.5
    assert abs(float(rstd[0]) - 1e-5**-0.5) <= 4 * U * 1e-5**-0.5 + 1e-5**-1.5 * U * 1e-5
    assert bool(y[1:].isnan().all())


def test_layer_norm_gradient_against_differences(w):
    """Central differences of step s of L = sum(y * G): the forward's rounding gives an error of
    at most (tolerance of y, about 70 U |G| per column) / s, the third derivative s^2 / 6 of it;
    for unit rows of 24 columns and s = 2^-6 both are below 1e-2."""
    g = gen(7)
    n, d, s = 3, 24, 2.0**-6
    x, G = rand(g, n, d), rand(g, n, d)
    gamma, beta = rand(g, d, std=0.2, mean=1.0), rand(g, d)

    def loss(x, gamma, beta):
        return float((w.layer_norm(x, gamma, beta)[0].double() * G.double()).sum())

    _, mean, rstd = w.layer_norm(x, gamma, beta)
    dx, dgamma, dbeta = w.layer_norm_grad(G, x, gamma, mean, rstd)
    for which, grad, at in ([(0, dx, (i, j)) for i in range(n) for j in (0, 11, 23)] +
                            [(1, dgamma, (j,)) for j in (0, 5, 23)] + [(2, dbeta, (j,)) for j in (0, 5, 23)]):
        sides = []
        for sign in (1, -1):
            args = [x.clone(), gamma.clone(), beta.clone()]
            args[which][at] += sign * s
            sides.append(loss(*args))
        assert abs((sides[0] - sides[1]) / (2 * s) - float(grad[at])) <= 1e-2


# ---- calls, streams, captures ---------------------------------------------------------------------

def test_expanded_and_transposed_gradients_are_taken(w):
    ids = torch.tensor([1, 0, 1], device="cuda")
    _, rows, count = w.embed_grad(ids, torch.ones(1, 8, device="cuda").expand(3, 8), 2)
    assert int(count) == 2 and torch.equal(rows[:2, 0], torch.tensor([1.0, 2.0], device="cuda"))
    t = rand(gen(1), 8, 3)
    out = torch.empty(2, 8, device="cuda")
    w.embed_grad_dense(ids, t.t(), out)
    assert torch.equal(out[0], t[:, 1])
    x = rand(gen(2), 16, 6)
    assert torch.equal(w.layer_norm(x.t())[0], w.layer_norm(x.t().contiguous())[0])


def test_no_tokens_and_no_rows(w):
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    W, g = torch.ones(4, 8, device="cuda"), torch.empty(0, 8, device="cuda")
    assert w.embed(W, none).shape == (0, 8) and w.embed(W, none.view(0, 5)).shape == (0, 5, 8)
    ids, rows, count = w.embed_grad(none, g, 4)
    assert ids.numel() == rows.numel() == int(count) == 0
    strided = torch.ones(4, 10, device="cuda")
    for out in (W.clone(), strided[:, :8]):
        w.embed_grad_dense(none, g, out, accumulate=True)
        assert bool((out == 1.0).all())
        w.embed_grad_dense(none, g, out)
        assert not bool(out.any())
    assert bool((strided[:, 8:] == 1.0).all())
    y, mean, rstd = w.layer_norm(g)
    dx, dgamma, dbeta = w.layer_norm_grad(g, g, None, mean, rstd)
    assert y.shape == dx.shape == (0, 8) and not bool(dgamma.any()) and not bool(dbeta.any())
    assert float(w.grad_norm([])) == 0.0 and float(w.clip_grads([g], 1.0)) == 0.0
    w.sync()


def test_bad_tensors_are_refused(w):
    ids = torch.tensor([1, 0], device="cuda")
    W = torch.ones(4, 8, device="cuda")
    bad = [lambda: w.embed(W, ids.int()), lambda: w.embed(W.cpu(), ids), lambda: w.embed(W, ids.cpu()),
           lambda: w.embed(W.double(), ids), lambda: w.embed(W.half(), ids, dtype=torch.bfloat16),
           lambda: w.embed(W.t(), ids), lambda: w.embed(W, ids, id_mode=B.HASH),
           lambda: w.embed(W, ids, out=torch.empty(3, 8, device="cuda")),
           lambda: w.embed_grad(ids, W, 4), lambda: w.embed_grad(ids, W[:2], 0),
           lambda: w.embed_grad_dense(ids, W[:2], W.half()), lambda: w.embed_grad_dense(ids, W[:2], W),
           lambda: w.grad_norm([W.t()]), lambda: w.grad_norm([W.cpu()]), lambda: w.clip_grads([W], -1.0),
           lambda: B.grad_parts([W], [W[:2]]), lambda: B.grad_parts([W], []),
           lambda: w.clip_grads(B.grad_parts([W.view(-1)[:16]], [W.view(-1)[8:24]]), 1.0),
           lambda: w.layer_norm(W, W[0], W[0].half()), lambda: w.layer_norm(W, W[0, :3]),
           lambda: w.layer_norm(W, eps=-1.0), lambda: w.layer_norm(W.long()),
           lambda: w.layer_norm_grad(W[:3], W, None, W[:, 0], W[:, 0]),
           lambda: w.layer_norm_grad(W, W, None, W[0, :3], W[:, 0])]
    for i, call in enumerate(bad):
        with pytest.raises(B.GBAError) as e:
            call()
        assert e.value.status == B.GBA_E_ARG, i
    w.sync()


def test_calls_under_another_stream_are_ordered_with_it():
    """Tensors made and used on a stream that is not the worker's."""
    w = B.Worker()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for i in range(20):
            g = gen(i)
            weights = rand(g, 5000, 256)
            ids = torch.randint(0, 5000, (20_000,), generator=g, device="cuda")
            y = w.embed(weights, ids, scale=2.0)
            z, _, _ = w.layer_norm(y)
            ok = torch.equal(y, weights[ids] * 2.0) and bool(z.isfinite().all())
            del y, z, weights
            assert ok
    w.sync()
    w.close()


@pytest.mark.parametrize("n", [5000, 20_000])
def test_a_captured_sequence_replays(n):
    """After a first run at the size, the calls allocate nothing and can be captured."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        w = B.Worker()
        g = gen(11)
        V, d = 700, 64
        weights, G = rand(g, V, d), rand(g, n, d)
        gamma = rand(g, d)
        ids = torch.randint(0, V, (n,), generator=g, device="cuda")

        def step():
            y = w.embed(weights, ids, scale=8.0)
            z, mean, rstd = w.layer_norm(y, gamma)
            dx, dgamma, dbeta = w.layer_norm_grad(G, y, gamma, mean, rstd)
            i, r, c = w.embed_grad(ids, dx, V, scale=8.0)
            norm = w.clip_grads([r, dgamma, dbeta], 1.0)
            return z, i, r, c, dgamma, dbeta, norm

        step()
        w.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = step()
        for seed in (12, 13):
            ids.copy_(tokens(gen(seed), n, V, "skew", 0))
            G.copy_(rand(gen(seed), n, d))
            graph.replay()
            got = [t.clone() for t in out]
            for a, b in zip(got, step()):
                assert torch.equal(a, b)
        w.sync()
        del graph
    w.close()
