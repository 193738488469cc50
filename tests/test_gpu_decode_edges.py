"""The command of paper_1901_10008_amd.decode with more tenants than its usual ones."""
import pytest

from paper_1901_10008_amd import decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [0, 40])
def test_command_with_a_dozen_tenants(vocab, capsys):
    """Each one's prompt is longer than that of the one before: the last one's has to find room too."""
    decode.main(["--tenants", "13", "--layers", "1", "--prompt", "16", "--children", "1", "--steps", "1", "--drafts", "2", "--vocab", str(vocab)])
    assert "13 " in capsys.readouterr().out
