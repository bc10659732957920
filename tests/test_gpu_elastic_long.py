"""The example's job with a batch of thousands of tokens, whose gradients are summed in several launches."""
import pytest

import test_gpu_elastic_step as short
from gpu_util import say

pytestmark = pytest.mark.gpu
example = short.example


def test_resharded_job_of_long_batches(example, monkeypatch):
    say("example: 20 sequences")
    monkeypatch.setattr(example, "SEQUENCES", 20)
    short.test_resharded_job_equals_the_one_that_stays(example)
