"""What the entry points around the layers say of sizes at their limits, on the CPU: a workspace's size, or the refusal
that the call itself would give."""
import os

import pytest

import paper_2401_13660_amd as mb
from paper_2401_13660_amd import _binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libmbscan.so not built")


@pytest.mark.parametrize("V,d", [(1, 1 << 34), (1, (1 << 34) - 1), (1, 1 << 45), (130000, 1 << 28)])
def test_no_tokens_and_wide_rows(V, d):
    """A workgroup per token and tile of columns (no workspace) counts a row's spans in 32 bits, so it takes no rows of this
    width: without tokens either, the table is set to zero by the launch that sorts them, which has a workspace."""
    assert mb.load_library().mb_embedding_bwd_workspace(0, V, d) > 0


def test_no_tokens_and_ordinary_rows():
    for V, d in ((1, 1), (256, 1792), (131072, 2304), (1, 1 << 19)):
        assert mb.load_library().mb_embedding_bwd_workspace(0, V, d) == 0
