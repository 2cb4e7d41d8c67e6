"""Host-side checks of the training operators at the ends of their ranges that need no GPU."""
import pytest

import paper_2110_14895_b200 as vit
from paper_2110_14895_b200 import build as vit_build


@pytest.fixture(scope="module", autouse=True)
def built():
    vit_build.build()
    vit.lib()


def test_clip_scratch_of_the_longest_lists():
    """960 tensors to a launch: the scratch grows by the same for each, up to the last count that there is."""
    one = vit.vit_grad_clip_bytes(960)
    for count in (961, 10 ** 6, 2 ** 31 - 960, 2 ** 31 - 959, 2 ** 31 - 1):
        assert vit.vit_grad_clip_bytes(count) == -(-count // 960) * one
