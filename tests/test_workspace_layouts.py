"""Where the workspaces' parts lie: what is read 16 bytes at a time starts at a
multiple of 16."""
import pytest

from paper_2609_27233_amd import lib as sm


@pytest.mark.parametrize("vocab", [1, 1000, 128256, 1 << 19])
def test_every_row_of_the_sampling_workspace_is_aligned(vocab):
    L = sm.load()
    one = L.sm_sample_workspace_bytes(1, vocab)
    assert one > 0 and one % 16 == 0
    for rows in (2, 3, 1024):
        assert L.sm_sample_workspace_bytes(rows, vocab) == rows * one
