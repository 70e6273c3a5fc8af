"""More of what the entry points of a block's operators refuse and take, without a GPU (see
test_block_host.py, whose library it uses)."""
import pytest

from paper_2205_11048_gb300 import binding as B
from tests.test_block_host import F, T, adamw, narrow, part, place, w  # noqa: F401


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
