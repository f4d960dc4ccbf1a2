"""The decoding example with a window and no word about pages: a token attends to its window, not to pages ranked over everything."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_window_by_itself_is_attended_to(capsys):
    """The prompt is 19 windows long.  The cache's attention is as near to attention over the unquantised window as without a window (8 bits: 0.06)."""
    from paper_2110_08919_amd import decode
    r = decode.main(["--prompt", "1900", "--conversations", "2", "--steps", "3", "--layers", "2", "--window", "100"])
    assert "tokens/s" in capsys.readouterr().out
    assert set(r) == {"all_pages"} and max(r["all_pages"]) < 0.06
