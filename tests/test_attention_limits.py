"""Launch sizes of attention, without a GPU: the parts that a setting asks for stay within what a launch counts."""
import numpy as np
import pytest

from paper_2008_01425_amd import binding as B
from parity_util import env_settings


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("sequences,heads,rows", [(1 << 14, 32, 1 << 15), (1 << 10, 512, 1 << 15), (1 << 15, 16, 1 << 14), (1, 1 << 14, 1 << 16)])
def test_forced_parts_leave_a_launch_countable(sequences, heads, rows, backward):
    """Parts are floats of the workspace: [part][sequence][row][head][width], forward two more for each head, backward those of two gradients behind a float for each head."""
    shape = B.pg_attention_shape(sequences, rows, rows, heads, heads, 1, 1.0, None, None, None)
    tiles = sequences * heads * (rows // 128)
    for splits in (1, 3, 64):
        with env_settings(dict(PG_ATTENTION_SPLITS=splits)):
            c = B.pg_init(1, np.zeros((0, 2), np.int32), np.zeros(0, np.float32), [4], [4], 1, 1)
            size = B.pg_attention_workspace_bytes(c, shape, B.PG_BF16, backward)
            B.pg_destroy(c)
        floats = sequences * rows * heads
        parts = (size // 4 - floats) / (2 * floats) if backward else size / 4 / (3 * floats)
        assert parts == int(parts) and parts <= splits
        assert max(parts, 1) * tiles < 1 << 30
        assert max(parts, 1) == max(1, min(splits, ((1 << 30) - 1) // tiles))


# Bytes of scratch a lane of the kernels that do not fit their registers has at most: (kernel, arithmetic, width filled up to): bytes.  All others have none.
SCRATCH = {("", 0, 256): 600, ("", 1, 128): 32, ("", 1, 256): 128, ("", 2, 64): 352, ("", 2, 96): 320, ("dq_", 0, 192): 240, ("dq_", 0, 256): 860, ("dq_", 2, 64): 160,
           ("dq_", 2, 128): 192, ("dkv_", 0, 192): 128, ("dkv_", 0, 256): 880, ("dkv_", 1, 128): 96, ("dkv_", 2, 128): 420}


def test_what_goes_through_scratch():
    import re

    import code_objects
    found = 0
    for name, kernel in code_objects.kernels(B.LIB_PATH).items():
        m = re.match(r"pg::attention_(|dq_|dkv_)kernel<(\d), (\d+), ", name)
        if m:
            found += 1
            assert kernel[".private_segment_fixed_size"] <= SCRATCH.get((m.group(1), int(m.group(2)), int(m.group(3))), 0), name
    assert found >= 90
