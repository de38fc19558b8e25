"""The example that runs the sequence operators together: it trains, and its stream gives what the whole pass gives."""
import pytest

pytestmark = pytest.mark.gpu


def test_stream_model_learns_and_streams():
    from examples.stream_model import run
    losses, off = run(batch=8, segments=160, channels=48, steps=25, log=lambda *_: None)
    assert losses[-1] < 0.5 * losses[0], losses
    assert off <= 1e-4           # sums of some 50 float32 terms in another order, a carried state of float32
