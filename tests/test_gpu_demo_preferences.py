"""The operators for language models together, as a decentralised training run uses them."""
import pytest

pytestmark = pytest.mark.gpu


def test_workers_learn_from_pairs_and_rewards():
    from paper_2009_05766_amd.demo_preferences import main
    seen, rewards = main(["--workers", "4", "--steps", "14"])
    # pairs start undecided (loss log 2) and end in the teacher's order; rewards rise by more than their noise (4 x 384 tokens: 0.013)
    assert 0.6 < seen[0][0] < 0.8 and seen[-1][0] < 0.2 and seen[-1][1] > 0.95
    assert rewards[-1] > rewards[0] + 0.05
