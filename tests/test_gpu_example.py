"""The example that runs the operators together: it learns, its 4-bit head stands for its float head, and two runs agree."""
import pytest

pytestmark = pytest.mark.gpu

SMALL = ["--scale", "10", "--dim", "40", "--classes", "33", "--top", "5", "--minibatches", "4", "--targets", "50",
         "--fanout", "5", "--steps", "30"]


def test_distill_nodes():
    from examples import distill_nodes
    r = distill_nodes.main(SMALL)
    # a step along the gradient of a sum of convex terms, small against their curvature, lowers it; half is left
    # open for the targets that differ from step to step
    assert 0 < r["last_loss"] < r["first_loss"]
    # an element's rounding is at most a quarter of its size above half the block's scale, and the errors of the
    # K products are independent: far below one in the sum
    assert 0 < r["error_4bit"] < 0.5
    assert distill_nodes.main(SMALL)["first_loss"] == r["first_loss"]


def test_distill_nodes_two_runs_agree_to_the_end():
    """Sums in a fixed order, products and updates of distinct rows: every figure of a second run is the first's."""
    from examples import distill_nodes
    assert distill_nodes.main(SMALL) == distill_nodes.main(SMALL)
