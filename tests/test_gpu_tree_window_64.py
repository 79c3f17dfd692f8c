"""Windows about as long as a tree is deep: a draft with an empty mask stands one position in front of the tree, one that sees all 64 drafts 64 behind it."""
import random

import pytest

from paper_2609_04774_b200 import binding
from tests.tree_util import TreeStep, tree_seen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mx4"])
@pytest.mark.parametrize("Hq", [2, 8])
@pytest.mark.parametrize("window", [62, 63, 64, 65, 66])
@pytest.mark.parametrize("sinks", [0, 100])
def test_a_draft_64_positions_back(ctx, kind, Hq, window, sinks):
    rng = random.Random(window)
    full = (1 << 64) - 1
    masks = [[0] + [rng.getrandbits(64) | 1 for _ in range(62)] + [full], [rng.choice([0, full, 1, full - 1]) for _ in range(64)]]
    s = TreeStep(Hq, [300, 40], masks, Hq, 2, 32, kind)
    # the rule itself: the last row sees the first draft from a window of 65 on, or where the sinks reach that far
    assert [bool(tree_seen(base, m, window, sinks)[63, base]) for base, m in zip(s.bases, masks)][0] == (window > 64)
    s.check(ctx, window, sinks)
