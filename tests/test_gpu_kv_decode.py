"""The decoding example: a stack of attention layers that generates tokens from quantised caches."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_decoder_generates_from_quantised_caches():
    from paper_2110_08919_amd import decode
    shape = decode.Shape(layers=2, width=256, heads=6, kv_heads=2, dim=48, vocabulary=500, page=16)
    g = torch.Generator().manual_seed(0)
    prompts = [torch.randint(500, (n,), generator=g).tolist() for n in (150, 1, 37)]
    # 8 bits over +-4 sigma: a step of sigma / 32; keys off by 0.009 sigma a feature and values by as much move an average by
    # a few hundredths of it, 2.5 sigma in 16 steps by ten times that
    for packed, bound in ((False, 0.06), (True, 0.6)):
        d = decode.Decoder(shape, prompts, 12, packed=packed)
        assert max(d.errors(0)) < bound
        assert max(d.errors(12)) < bound                   # 12 pages of 16 tokens: all there are
        tokens = [d.step(3).tolist() for _ in range(5)]
        assert all(0 <= t < 500 for row in tokens for t in row)
        assert d.lengths.tolist() == [157, 8, 44]


def test_command_prints_errors_and_speed(capsys):
    from paper_2110_08919_amd import decode
    r = decode.main(["--prompt", "600", "--conversations", "2", "--steps", "3", "--pages", "4", "--layers", "2"])
    out = capsys.readouterr().out
    assert "tokens/s" in out and set(r) == {"all_pages", "selected_pages"}
    assert max(r["all_pages"]) < 0.06


def test_errors_are_compared_with_every_token_so_far():
    """A step in between leaves its keys and values out of what the errors are measured against: that is refused."""
    from paper_2110_08919_amd import decode
    shape = decode.Shape(layers=1, width=128, heads=2, kv_heads=1, dim=32, vocabulary=100, page=16)
    d = decode.Decoder(shape, [[1, 2, 3], list(range(40))], 8)
    assert max(d.errors(0)) < 0.06 and max(d.errors(0)) < 0.06
    d.step(0)
    with pytest.raises(AssertionError):
        d.errors(0)
