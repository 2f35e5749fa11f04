"""CPU-only: windows, first tokens and an eps that their 32 bits do not hold are refused as other arguments are."""
import pytest

from paper_2604_08077_b200 import binding
from test_more_text_host import INVALID, append, chunk, code, decode, handle, rotate  # noqa: F401


@pytest.mark.parametrize("call", [chunk, decode])
@pytest.mark.parametrize("bad", [dict(window=2 ** 31), dict(window=2 ** 64), dict(sinks=2 ** 31), dict(window=-2 ** 31 - 1), dict(window=16.0), dict(sinks=None)])
def test_windows_that_are_no_32_bits(handle, call, bad):                                   # noqa: F811
    assert code(lambda: call(handle, **bad)) == INVALID


@pytest.mark.parametrize("call", [rotate, append])
@pytest.mark.parametrize("eps", [1e39, -1e39, None, "1e-6"])
def test_eps_that_is_no_32_bit_number(handle, call, eps):                                  # noqa: F811
    assert code(lambda: call(handle, eps=eps)) == INVALID
    with pytest.raises(binding.AdasparkError):
        call(handle, eps=eps)
