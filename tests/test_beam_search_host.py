"""CPU: searches that Decoder.beam_search cannot make are refused before any cache is forked."""
import pytest

from paper_2509_24381_amd.binding import RsError
from paper_2509_24381_amd.decode import Decoder


class Forked(Exception):
    pass


class Prompt:
    def length(self, layer=0):
        return 100

    def fork(self, n=None):
        raise Forked


def search(n_tokens, beams, end=None):
    Decoder.beam_search(None, [Prompt()], None, None, None, None, n_tokens, beams, end=end)


@pytest.mark.parametrize("n_tokens, beams, end", [(0, 4, None), (-1, 4, None), (0, 4, 2), (5, 0, None), (5, -1, 3), (5, 65, None), (5, 33, 2), (5, 64, 0)])
def test_refusals(n_tokens, beams, end):
    with pytest.raises(RsError, match="n_tokens >= 1") as e:
        search(n_tokens, beams, end)
    assert e.value.status_name == "RS_EINVAL" and str(beams) in str(e.value)


@pytest.mark.parametrize("n_tokens, beams, end", [(1, 1, None), (5, 64, None), (5, 32, 2), (5, 1, 0)])
def test_the_largest_and_smallest_are_made(n_tokens, beams, end):
    with pytest.raises(Forked):
        search(n_tokens, beams, end)
