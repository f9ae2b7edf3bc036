"""A top_k that the C struct cannot hold is refused, not cut to its low 32 bits (no GPU)."""
import pytest

from paper_2505_14260_amd import msd


@pytest.mark.parametrize("top_k", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, -2 ** 32 + 5])
def test_top_k_past_32_bits_is_refused(top_k):
    with pytest.raises(ValueError, match="top_k"):
        msd.Sampling(1.0, 1.0, 0.0, top_k)
    with pytest.raises(ValueError, match="top_k"):
        msd.Sampling(1.0, 1.0, top_k=top_k)


def test_settings_keep_their_values():
    s = msd.Sampling(0.7, 0.9, 0.01, 2 ** 31 - 1)
    assert (s.temperature, s.top_p, s.min_p, s.top_k) == (0.7, 0.9, 0.01, 2 ** 31 - 1)
    assert msd.Sampling(1.0, 1.0, 0.0, -1).top_k == -1      # the library refuses it
    assert (msd.Sampling().temperature, msd.Sampling().top_k) == (0.0, 0)
