"""The restated plan of the linear layers' products against the library's, as far as it shows without a device: workspace sizes."""
import random

import pytest

import paper_2501_09849_b200 as cdl
from linear_plan import workspace_bytes
from paper_2501_09849_b200 import build as cdl_build


@pytest.mark.parametrize("seed", range(8))
def test_workspace_sizes_agree(seed):
    cdl_build.build()
    rng = random.Random(seed)
    for _ in range(250):
        M, N, K = (int(round(2 ** rng.uniform(0, 14.5))) for _ in range(3))
        assert cdl.cdl_linear_workspace_bytes(M, N, K) == workspace_bytes(M, N, K), (M, N, K)
