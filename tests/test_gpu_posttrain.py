"""The post-training example: the operators together with the compressed step."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_policy_raises_the_reward():
    import posttrain
    h = posttrain.train(posttrain.parse(["--loss", "policy", "--steps", "60"]))
    assert abs(sum(h[:3]) / 3 - 1 / posttrain.CLASSES) < 0.05
    assert sum(h[-5:]) / 5 > 0.3


def test_preference_lowers_the_loss():
    import posttrain
    h = posttrain.train(posttrain.parse(["--loss", "preference", "--steps", "60"]))
    assert abs(h[0] - math.log(2)) < 0.1      # the reference without dropout: not exactly log 2
    assert sum(h[-5:]) / 5 < 0.4


def test_same_seed_same_run():
    import posttrain
    a = posttrain.train(posttrain.parse(["--loss", "preference", "--steps", "3", "--seed", "5"]))
    b = posttrain.train(posttrain.parse(["--loss", "preference", "--steps", "3", "--seed", "5"]))
    assert a[0] == b[0]      # later steps: torch's index_add_ adds in any order
