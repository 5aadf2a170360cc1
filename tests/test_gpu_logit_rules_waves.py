"""Rules in blocks of four waves: more blocks than compute units, several rows a wave, every token against the definition."""
import numpy as np
import pytest

import test_gpu_logit_rules as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("in_place", [True, False])
def test_blocks_of_four_waves_with_rows_to_spare(gpu, bf16, in_place):
    """320 blocks of 14 rows: four waves with three or four rows each.  Tokens of the rows' paths and new ones lie in every block."""
    c = T.case(61, 64, 14, 8, 2500, 3)
    rng = np.random.default_rng(62)
    c["tokens"] = rng.integers(0, 2500, (64, 8)).astype(np.int32)
    c["tokens"][:, 5] = c["tokens"][:, 3]                            # (some twice on a path)
    c["new"] = rng.integers(-1, 2500, (64, 3)).astype(np.int32)
    T.run(gpu, c, bf16, in_place=in_place)
