"""Streams that the feed-forward calls take (no GPU needed)."""
from types import SimpleNamespace

import pytest

from paper_2309_17224_amd import fp8lin as F


def test_a_stream_of_another_gpu_is_refused():
    """The kernels of a call run on its tensors' GPU; a stream of another would take them there."""
    stream = lambda gpu: SimpleNamespace(cuda_stream=77, device_index=gpu)  # noqa: E731
    assert F._stream_on(stream(0), 0) == 77 and F._stream_on(stream(3), 3) == 77
    with pytest.raises(ValueError, match="stream"):
        F._stream_on(stream(1), 0)
