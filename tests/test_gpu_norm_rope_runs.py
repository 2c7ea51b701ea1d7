"""Head norms of sizes that have no kernel of their own, with so many tokens that a warp works
through several tasks: parts of one token, and several tokens one after another."""
import pytest

from test_gpu_norm_rope import Step, ppas  # noqa: F401

pytestmark = pytest.mark.gpu


# 152 SMs hold 3648 warps; a token's 24 head rows are 3, 5 and 12 passes of 32 lanes
@pytest.mark.parametrize("D,rotary", [(64, 64), (80, 32), (256, 128)])
@pytest.mark.parametrize("T", [1601, 4100, 8001])
@pytest.mark.parametrize("inter", [False, True])
def test_more_tasks_than_warps(ppas, D, rotary, T, inter):  # noqa: F811
    s = Step(T, 16, 4, D, rotary, inter, seed=D + T, gap=8)
    ppas.ppas_norm_rope_append(**s.args())
    s.check()
