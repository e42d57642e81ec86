"""Groups of experts whose values leave fp32's range when they are added: a group is left out for having no expert left, never
for what its sum rounds to."""
import numpy as np
import pytest

from tests.test_gpu_route import INF, _run

pytestmark = pytest.mark.gpu
LOWEST = float(np.finfo(np.float32).min)


# groups of 2^i whole lanes and others; one launch (up to 16 rows) and two
SIZES = [(8, 4, 3, 6), (32, 8, 5, 20), (64, 8, 3, 24), (256, 8, 4, 32), (512, 16, 5, 32), (60, 4, 3, 32), (90, 6, 4, 32),
         (510, 30, 29, 32)]


@pytest.mark.parametrize("experts,groups,top_groups,k", SIZES)
@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("rows", [3, 40])
def test_groups_masked_by_the_lowest_number(experts, groups, top_groups, k, sigmoid, rows):
    """Two masked experts' values add up to less than any fp32 number: their group comes last, but it has experts."""
    rng = np.random.default_rng(experts + rows)
    l = rng.standard_normal((rows, experts))
    each = experts // groups
    masked = np.zeros(groups, bool)
    masked[rng.permutation(groups)[:groups - top_groups + 1]] = True        # one of them stays
    _run(l, k, sigmoid=sigmoid, bias=np.where(np.repeat(masked, each), LOWEST, 0.0), groups=groups, top_groups=top_groups)
    one = np.repeat(masked, each) & (np.arange(experts) % each > 0)         # a masked group's first expert is not
    _run(l, k, sigmoid=sigmoid, bias=np.where(one, LOWEST, 0.0), groups=groups, top_groups=top_groups)
    _run(l, k, sigmoid=sigmoid, bias=np.full(experts, LOWEST), groups=groups, top_groups=top_groups)


@pytest.mark.parametrize("experts,groups,top_groups,k", SIZES)
@pytest.mark.parametrize("sigmoid", [True, False])
@pytest.mark.parametrize("rows", [3, 40])
def test_groups_whose_sums_pass_the_range(experts, groups, top_groups, k, sigmoid, rows):
    """Biases of both signs and of sizes whose sums overflow, ruled-out experts and infinite biases among them: the groups'
    order is that of the exact sums."""
    rng = np.random.default_rng(experts * 3 + rows)
    l = rng.standard_normal((rows, experts))
    l[rng.random(l.shape) < 0.1] = -INF
    sizes = np.array([LOWEST, -2.5e38, -1.8e38, 0.0, 1.8e38, 2.5e38, -LOWEST])
    _run(l, k, sigmoid=sigmoid, bias=rng.choice(sizes, experts), groups=groups, top_groups=top_groups)
    _run(l, k, sigmoid=sigmoid, bias=rng.choice(sizes[:3], experts), groups=groups, top_groups=top_groups)
    _run(l, k, sigmoid=sigmoid, bias=rng.choice(sizes[4:], experts), groups=groups, top_groups=top_groups)
    _run(l, k, sigmoid=sigmoid, bias=rng.choice(np.append(sizes, [-INF, INF]), experts), groups=groups, top_groups=top_groups)
