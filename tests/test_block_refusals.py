"""More of what the entry points of a block's operators refuse and take, without a GPU (see
test_block_host.py, whose library it uses)."""
import pytest

from paper_2205_11048_gb300 import binding as B
from tests.test_block_host import AT, F, T, adamw, mat, narrow, norm, norm_grad, part, place, scan, scan_grad, scan_of, w  # noqa: F401


@pytest.mark.parametrize("eps,status", [(2.0**-126, B.GBA_OK), (2.0**-127, B.GBA_E_ARG), (1e-44, B.GBA_E_ARG)])
def test_an_eps_is_a_normal_number(F, w, eps, status):  # noqa: F811
    assert adamw(F, w, eps=eps) == status


@pytest.mark.parametrize("rounding,status", [(0, B.GBA_OK), (1, B.GBA_OK), (2, B.GBA_E_ARG), (-1, B.GBA_E_ARG)])
def test_a_rounding_is_known(F, w, rounding, status):  # noqa: F811
    for p in (part(), narrow()):
        d = B.gba_adamw_desc(1e-3, 0.9, 0.999, 1e-8, None, None, 0.0, rounding)
        assert F.gba_adamw(w, (B.gba_adamw_part * 1)(p), 1, d, place(30)) == status


@pytest.mark.parametrize("how", [dict(bits=8, rounding="up"), dict(bits=32, rounding="chance"), dict(bits=8, rounding=1)])
def test_a_rounding_is_one_of_states_in_8_bits(how):
    with pytest.raises(B.GBAError) as e:
        B.adamw_states([T(8)], **how)
    assert e.value.status == B.GBA_E_ARG


WIDE = AT + 41 * 4096  # a matrix of 3 x 8 columns, and one a little wider


def column(i, stride=24, **k):
    return mat(0, stride=stride, data=WIDE + 4 * i, **k)


@pytest.mark.parametrize("a,b,apart", [
    (column(0), column(8), True), (column(8), column(0), True), (column(16), column(0), True),
    (column(0), column(16), True), (column(0), column(7), False), (column(7), column(0), False),
    (column(16), column(9), False), (column(0), column(8, stride=25), False), (column(0, stride=25), column(8), False),
    (column(0), column(24 + 8), True), (column(24 + 8), column(0), True), (column(24 + 17), column(0), False),
    (column(17), column(24), False), (column(0), column(0), False), (column(0), column(48), False),
    (column(0, type=B.F32), column(8, stride=48, type=B.BF16), True),
    (column(0, type=B.F32), column(7, stride=48, type=B.BF16), False),
    (column(12, stride=48, type=B.BF16), column(0, type=B.F32), True),
    (column(21, stride=48, type=B.BF16), column(0, type=B.F32), False)])
def test_columns_of_one_matrix_are_apart(F, w, a, b, apart):  # noqa: F811
    """Outputs beside one another and beside inputs, and those that touch."""
    want = B.GBA_OK if apart else B.GBA_E_ARG
    if a.type == b.type:
        assert norm_grad(F, w, dx=a, dg=b) == norm_grad(F, w, dx=a, x=b) == norm_grad(F, w, dg=b, dz=a) == want
        assert norm(F, w, z=a, y=b) == norm(F, w, y=b, g=a) == norm(F, w, z=a, x=b) == want
        assert scan_grad(F, w, dx=a, df=b) == scan_grad(F, w, f=a, df=b) == want
        assert scan(F, w, y=a, f=b) == want
    else:  # a residual stream in 32 bits beside 16-bit matrices
        x, y, g = [mat(i, type=B.BF16) for i in (0, 4, 2)]
        wide, half = (a, b) if a.type == B.F32 else (b, a)
        assert norm(F, w, x=x, g=g, r=mat(1), z=wide, y=half) == norm(F, w, x=half, g=g, r=mat(1), z=wide, y=y) == want


def test_columns_are_not_apart_from_arrays(F, w):  # noqa: F811
    assert norm_grad(F, w, dx=column(0), sums=(WIDE + 32, None, None, None)) == B.GBA_E_ARG
    assert norm(F, w, y=column(0), stats=WIDE + 32) == B.GBA_E_ARG


def test_the_sequences_of_a_call_without_rows_are_looked_at(F, w):  # noqa: F811
    """Their offsets and lengths may be bad all the same, which only a kernel can see."""
    e = dict(rows=0, data=None)
    rows = {k: mat(0, **e) for k in ("x", "f", "y")}
    back = {**rows, **{k: mat(0, **e) for k in ("dy", "dx", "df")}}
    n = F.fake_block_launches()
    for i, how in enumerate((dict(offsets=place(50)), dict(lengths=place(50)))):
        assert scan(F, w, scan_of(**how), **rows, state=None, out=None) == B.GBA_OK
        assert scan_grad(F, w, scan_of(**how), **back, ds=None, state=None, out=None) == B.GBA_OK
        assert F.fake_block_launches() == n + 2 * i + 2
    assert scan(F, w, scan_of(), **rows, state=None, out=None) == B.GBA_OK  # nothing to see and nothing to write
    assert F.fake_block_launches() == n + 4
