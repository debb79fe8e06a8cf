"""GPU: the example of recover.py -- a quantized model, adapters, distillation -- learns."""
import pytest

from paper_2512_02010_amd import recover

pytestmark = pytest.mark.gpu


def test_adapters_learn_what_quantization_lost():
    losses, adapted, plain = recover.run(steps=60)
    assert all(v == v and v < 1e3 for v in losses)
    first, last = sum(losses[:5]) / 5, sum(losses[-5:]) / 5
    assert last < 0.8 * first, (first, last)
    assert adapted < 0.8 * plain, (adapted, plain)
