"""What the decoding example refuses before it needs a device."""
from types import SimpleNamespace

import pytest

from paper_2110_08919_amd import decode


def test_selected_pages_with_a_window_are_refused(capsys):
    with pytest.raises(SystemExit) as e:
        decode.main(["--pages", "16", "--window", "100"])
    assert e.value.code == 2 and "--pages with --window" in capsys.readouterr().err
    with pytest.raises(AssertionError, match="window"):
        decode.Decoder.step(SimpleNamespace(shape=decode.Shape(window=100), kept=None), 4)
