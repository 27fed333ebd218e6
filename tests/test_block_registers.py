"""The kernels of a block's operators keep what they hold in registers: none
spills, but for the gradients of the norms over rows beyond 8192 elements, of
odd lengths most (and of bf16 rows beyond 4096, a few).  In the projections a spill would be wrong,
not slow alone: their waits count the loads between them, and a spilled
register's store would be one more.  The counts come from the metadata of the
code objects in libhla.so.  CPU only.
"""
import os
import re

import pytest

from tests.test_register_spills import READELF, _spilled
from tests.test_store_data_hazard import LIB

# mangled: the kernels, and the shapes of a row held by 512 and 1024 threads
KERNELS = r"k_gated_norm|k_residual_norm|k_column_sums|k_glr|k_glu|k_product|k_joined|k_packed"
WIDE = {r"norm_back.*RowShapeILi2ELi1024E": 256, r"k_gated_norm_back.*RowShapeILi2ELi512E": 16}


@pytest.mark.skipif(not os.path.exists(LIB), reason="libhla.so is not built")
@pytest.mark.skipif(not os.path.exists(READELF), reason="llvm-readelf is not installed")
def test_nothing_spills(tmp_path):
    counts = {s: n for s, n in _spilled(tmp_path).items() if re.search(KERNELS, s)}
    for name in KERNELS.split("|"):
        assert any(name in s for s in counts), name
    over = {s: n for s, n in counts.items()
            if n > next((most for shape, most in WIDE.items() if re.search(shape, s)), 0)}
    assert not over, over
