"""What the compiler has allotted to the kernels of latent caches: no scratch memory, and where loads to LDS are counted by hand no
accumulation registers to hold what does not fit (a spilt register's accesses would be counted among the loads)."""
import re

import pytest

from test_kernel_resources import kernels  # noqa: F401

COUNTED = ("latent_attend_kernel", "latent_project_kernel", "latent_prompt_kernel")


@pytest.mark.parametrize("kernel,count", [("latent_append_kernel", 4), ("latent_read_kernel", 4), ("latent_absorb_kernel", 4),
                                          ("latent_attend_kernel", 16), ("latent_join_kernel", 2), ("latent_values_kernel", 4),
                                          ("latent_table_kernel", 1), ("latent_gather_kernel", 4), ("latent_project_kernel", 2),
                                          ("latent_prompt_kernel", 8)])
def test_latent_kernels_do_not_spill(kernels, kernel, count):  # noqa: F811
    mine = {n: k for n, k in kernels.items() if re.search(r"\d%s[IE]" % kernel, n)}
    assert len(mine) == count, sorted(mine)
    for name, k in mine.items():
        fields = ("private_segment_fixed_size", "vgpr_spill_count") + (("agpr_count",) if kernel in COUNTED else ())
        spilt = {f: k[f] for f in fields}
        assert not any(spilt.values()), (name, spilt)
