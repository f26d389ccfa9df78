"""CPU checks of the drafts example: what it refuses, before anything is launched, and that a refusal changes nothing."""
import pytest

from paper_2603_08727_amd.paged_drafts_example import DraftedLayer

TREES = [[-1, 0, 0, 1, 2], [-1, -1]]


def layer(window=256):
    x = DraftedLayer.__new__(DraftedLayer)             # (without the pages, which are on the GPU)
    x.have, x.window, x.rows, x.max_tokens, x.device = [40, 7], window, 100, 64, "cpu"
    x.drafted = (None, None, TREES)
    return x


@pytest.mark.parametrize("paths", [[[0, 1]], [[0], [], []], [], [[1], []], [[0, 3], []], [[0, 1, 4], []], [[0, 0], []], [[5], []], [[0], [2]], [[-1], []], [[], [0, 1]]])
def test_paths_that_are_none_of_the_trees_are_refused(paths):
    """Another number of requests; a path that does not begin at the accepted rows, leaves out or repeats a draft, or names one that is not there."""
    x = layer()
    with pytest.raises(ValueError, match="path"):
        x.accept(paths)
    assert x.have == [40, 7] and x.drafted is not None


def test_drafts_are_accepted_once():
    x = layer()
    x.accept([[], []])
    assert x.have == [40, 7]
    with pytest.raises(ValueError, match="drafted"):
        x.accept([[], []])


def test_trees_that_reach_behind_the_window_are_refused():
    """A window takes no drafts away: a draft at its depth would see a first one, which decoding would not."""
    x = layer(window=3)
    with pytest.raises(ValueError, match="window"):
        x.draft(None, [[-1, 0, 1, 2], [-1]])
    assert x.have == [40, 7] and x.drafted is not None
