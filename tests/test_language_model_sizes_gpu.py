"""GPU test: the small language model on a single token, which has no successor and so no loss."""
import pytest

from paper_2009_12263_amd.language_model import main

pytestmark = pytest.mark.gpu


def test_one_token():
    assert main(["--steps", "2", "--tokens", "1", "--vocab", "50", "--dim", "16"]) == 0.0
