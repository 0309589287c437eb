"""How far gamma may go: what the fp32 arithmetic can still hold, refused beyond."""
import pytest

from test_launches_cpu import A, BF16, F32, launches, recorder   # noqa: F401 (a fixture)

SHAPE = 2
TINY, LARGE = 2.0 ** -126, 2.0 ** 120


def calls(gamma, dt):
    return {
        "forward": lambda lib: lib.laser_history_attention_forward(A, 32, A, 16, A, 16, A, 2, 10, 5, 4, 2, 8, gamma, dt, A, A, None),
        "cache": lambda lib: lib.laser_cache_attention_forward(A, 32, A, A, A, A, A, 2, 4, 3, 8, 16, 4, 50, 4, 2, 8, gamma, 1, dt, A, A, A, 1 << 30, None),
        "weights": lambda lib: lib.laser_cache_weights(A, 32, A, A, A, A, A, 2, 4, 3, 8, 16, 4, 50, 4, 2, 8, gamma, 1, 1, dt, A, None)}


def backward(gamma, dt):
    return lambda lib: lib.laser_history_attention_backward(A, 32, A, 16, A, 16, A, A, A, A, 2, 10, 5, 4, 2, 8, gamma, dt, A, 32, A, 16, A, 16, A, 1 << 20,
                                                            None)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_gamma_at_its_limits(recorder, dt):
    every = lambda gamma: {**calls(gamma, dt), "backward": backward(gamma, dt)}
    for gamma in (TINY, 1.0, LARGE):
        for name, call in every(gamma).items():
            assert launches(recorder, call), (name, gamma)
    for name, call in every(TINY / 2).items():    # (log2(e) / gamma leaves fp32 a little further down)
        assert call(recorder) == SHAPE, name
    for gamma in (2.0 * LARGE, 3e38):       # (the backward pass starts its scores at -gamma lse)
        for name, call in every(gamma).items():
            assert call(recorder) == (SHAPE if name == "backward" else 0), (name, gamma)
