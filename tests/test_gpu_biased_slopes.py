"""Distance biases of any size and sign on every kernel, against a bound of each
slot's own: the score of a row's own slot has nothing to round."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

from tests.test_gpu_biased import BF16, F16, Cache, Case, _built, ctx, masks  # noqa: E402,F401
from tests.test_gpu_biased_far_scores import check  # noqa: E402

SLOPES = {"usual": [0.7, 2.0 ** -8, 0.1, 1.0], "steep": [100.0, 1e4, 1e6, 1e9], "rising": [-0.5, -100.0, -1e4, -2.0 ** -9],
          "mixed": [1e3, 0.0, -3.0, 1e-30]}


@pytest.mark.parametrize("slopes", sorted(SLOPES))
@pytest.mark.parametrize("form", [dict(), dict(cap=30.0), dict(docs=50), dict(frame=40), dict(window=90, sinks=5, docs=200)])
@pytest.mark.parametrize("news", [[130, 33, 300], [2, 1, 3]])
@pytest.mark.parametrize("dtype,dim,page", [(BF16, 128, 64), (F16, 64, 16), (BF16, 64, 5), (F16, 64, 5)])
def test_slopes_of_any_size(ctx, slopes, form, news, dtype, dim, page):   # noqa: F811
    lens = [150, 700, 300]
    f = dict(form)
    first, until = masks(lens, news, f.pop("docs", 0), f.pop("frame", 0), 3)
    case = Case(Cache(lens, 2, dim, page, dtype, 5, junk=0.0), news, 4, first=first, until=until, seed=5, **f)
    case.slope = torch.tensor(SLOPES[slopes])
    check(ctx, case)


@pytest.mark.parametrize("news", [[130, 33, 300], [2, 1, 3]])
@pytest.mark.parametrize("cap,frame", [(0.0, 0), (30.0, 0), (0.0, 40)])
@pytest.mark.parametrize("dtype,page", [(BF16, 64), (F16, 16), (F16, 5)])
def test_slopes_that_leave_a_row_its_own_slot(ctx, news, cap, frame, dtype, page):   # noqa: F811
    """Biases past 32 bits' range take every other slot's weight, and nothing from the row's own."""
    lens = [150, 700, 300]
    first, until = masks(lens, news, 0, frame, 3)
    case = Case(Cache(lens, 2, 64, page, dtype, 5, junk=0.0), news, 4, cap=cap, until=until, seed=5)
    case.slope = torch.tensor([3e36, 1e38, 3e38, 2e36])
    check(ctx, case)
