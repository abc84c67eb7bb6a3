"""The largest and smallest calls of the operators around a decoding step, as the host sees them: what no launch can hold is refused as such."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2103_00130_amd import binding
    return binding


def logprobs(b, rows=3, vocab=100, scale=1.0):
    d = ctypes.c_void_p(0x1000)
    return b.lib.abft_logprobs(d, vocab, 2, rows, vocab, scale, d, d, d, d, d, 0, None, None, None, 0, None)


def test_rows_of_logits_beyond_a_launch(b):
    # 2^24 workgroups of 256 threads are 2^32 threads
    for rows in (2 ** 24, 2 ** 24 + 1, 2 ** 31 - 1, 2 ** 31, 2 ** 40):
        assert logprobs(b, rows=rows) == b.ABFT_EUNSUPPORTED and b"too large" in b.lib.abft_last_error(), rows
        assert b.lib.abft_logprobs_workspace_bytes(rows, 100000, 5) == 0
    assert b.lib.abft_logprobs_workspace_bytes(2 ** 24 - 1, 100000, 5) > 0


def test_scales_under_which_differences_that_32_bits_do_not_hold_would_count(b):
    for scale in (2.0 ** -121, 1e-38, 2.0 ** -140):
        assert logprobs(b, scale=scale) == b.ABFT_EINVAL and b"scale" in b.lib.abft_last_error(), scale
    assert logprobs(b, rows=0, scale=2.0 ** -120) == b.ABFT_OK
