"""sv_rope3d_rotate takes anything that int() takes for `inverse`, through the module and through ctypes.  Every call ends before a launch."""
import numpy as np
import pytest

import paper_2509_24695_amd as sv
from tests.test_host_entry import FAKE, _desc, _rope, _status, route  # noqa: F401


@pytest.mark.parametrize("inverse", [0, 1, True, np.True_, np.int64(1), 1.0, np.float32(0.0)])
def test_inverse(route, inverse):                                     # noqa: F811
    wrong_place = FAKE + 8
    assert _status(sv.sv_rope3d_rotate, wrong_place, None, _desc(), _rope(), None, inverse, FAKE, None, _desc()) == 4


def test_no_flag(route):                                              # noqa: F811
    with pytest.raises((TypeError, ValueError)):
        sv.sv_rope3d_rotate(FAKE + 8, None, _desc(), _rope(), None, "inverse", FAKE, None, _desc())
