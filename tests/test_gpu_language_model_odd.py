"""examples/language_model.py with a vocabulary that is no multiple of eight."""
import pytest

from test_gpu_language_model import example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [4099, 5003])
def test_a_step_with_an_odd_vocabulary(example, vocab):  # noqa: F811
    """As near the model in 64 bits as with a round one."""
    errors = example.main(256, 512, 1024, vocab)
    assert errors["loss"] < 0.05
    for name, off in errors.items():
        assert off < 0.4, (name, errors)
