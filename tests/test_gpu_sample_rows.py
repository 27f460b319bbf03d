"""celty_sample on rows that the choice of a token must not be sensitive to:
logits with an offset, filters at the ends of their ranges.  The definition is
that of tests/test_gpu_sample.py."""
import pytest

from tests.test_gpu_sample import _rows, _sample, _want, env  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("p", [float("-inf"), -3.0e38, -1.0, -0.0, 0.0, 1e-45])
def test_top_p_that_keeps_the_first_token_alone(env, p):  # noqa: F811
    """Also beside a top-k whose bin is the largest logit's."""
    torch, _ = env
    for dtype in ("float16", "float32"):
        logits, noise = _rows(torch, 6, 5003, dtype, 41)
        flat, _ = _rows(torch, 6, 5003, dtype, 42, sharp=False)
        for x in (logits, flat, torch.zeros_like(logits)):
            for f in (dict(p=p), dict(p=p, k=1), dict(p=p, k=7), dict(p=p, k=3000), dict(p=p, k=9000), dict(p=p, m=0.2, k=50)):
                got = _sample(env, x, noise, **f)
                assert (got == x.float().cpu().numpy().argmax(1)).all(), (dtype, f)
                assert (got == _want(x, noise, **f)).all()
