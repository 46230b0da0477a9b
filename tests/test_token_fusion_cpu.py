"""The token-fusion example's arguments and sizes, without a GPU."""
import pytest

from paper_2608_08330_gb300 import token_fusion as F


def test_head_layout():
    assert F.head_layout(384) == (6, 64) and F.head_layout(96) == (3, 32) and F.head_layout(32) == (1, 32)
    for channels in (0, 16, 48, 100):
        with pytest.raises(ValueError):
            F.head_layout(channels)


@pytest.mark.parametrize("absent", [["0"], ["-1"], ["1", "99"]])
def test_absent_agents_are_checked(absent, capsys):
    with pytest.raises(SystemExit):
        F.main(["--workload", "tiny", "--absent", *absent])
    assert "agent 0 is the ego" in capsys.readouterr().err


def test_the_ego_is_needed():
    for maps in ([], [None, 1]):
        with pytest.raises(ValueError):
            F.fuse(maps, "fp16", 4, 4, 0.8)


def test_workspace_has_a_part_per_65536_keys():
    part = 35200 * 6 * 66 * 4
    assert F.workspace_bytes(35200, 176000, 6, 64) == 4 * part
    assert F.workspace_bytes(1, 65536, 1, 32) == 2 * 34 * 4 and F.workspace_bytes(1, 65537, 1, 32) == 3 * 34 * 4
