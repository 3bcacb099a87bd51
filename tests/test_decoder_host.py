"""What the decoder refuses before anything reaches the device."""
import pytest
import torch

from paper_1809_02697_amd import decoder


def _decoder(vocab=20, pages=4, page_size=4):
    """A decoder without layers on the host: enough for the checks of a step."""
    d = decoder.Decoder.__new__(decoder.Decoder)
    d.embed, d.layers, d.caches, d.page_size, d.device = torch.zeros(vocab, 8), [], [], page_size, "cpu"
    d.free, d.pages, d.lengths = list(range(pages))[::-1], [[], []], [0, 0]
    return d


@pytest.mark.parametrize("tokens,error", [([[20], []], ValueError), ([[3, -1], [0]], ValueError), ([[], [0, 1 << 40]], ValueError),
                                          ([[1]], ValueError), ([[], []], ValueError), ([[1] * 9, [1] * 8], RuntimeError)])
def test_refused_steps_leave_the_decoder_as_it_was(tokens, error):
    d = _decoder()
    with pytest.raises(error):
        d.step(tokens)
    assert d.free == [3, 2, 1, 0] and d.pages == [[], []] and d.lengths == [0, 0]
