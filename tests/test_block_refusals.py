"""More of what the entry points of a block's operators refuse and take, without a GPU (see
test_block_host.py, whose library it uses)."""
import pytest

from paper_2205_11048_gb300 import binding as B
from tests.test_block_host import F, adamw, w  # noqa: F401


@pytest.mark.parametrize("eps,status", [(2.0**-126, B.GBA_OK), (2.0**-127, B.GBA_E_ARG), (1e-44, B.GBA_E_ARG)])
def test_an_eps_is_a_normal_number(F, w, eps, status):  # noqa: F811
    assert adamw(F, w, eps=eps) == status
