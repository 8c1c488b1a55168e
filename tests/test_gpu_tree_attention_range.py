"""Values near the ends of fp32's range: a row's weights are at most 1, so they overflow nowhere that the formula's weights would not."""
import numpy as np
import pytest

from test_gpu_tree_attention import Case, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40, 130])
@pytest.mark.parametrize("ctx", [220, 9000])
@pytest.mark.parametrize("top", [124, -80])
def test_large_and_small_values(kind, n, ctx, top):
    """Scores (base 2) are 0, but for one of 7.5 behind the first blocks that a wavefront goes through: below the factor that an accumulator's reference may lag
    behind by.  Values are up to 2^top; the sums of products with weights of at most 1 stay below 2^top (1 + T 2^-7.5) in magnitude, and far below
    with their random signs.  Once the late score is a cached token's, once it comes in pieces of 2.5."""
    for steps in ((7.5,), (2.5, 5.0, 7.5)):
        def edit(k, v, at):
            k.zero_()
            for i, s in enumerate(steps):
                k[ctx - 40 - 36 * (len(steps) - 1 - i), :, 0] = s
            v.copy_((v.float() / v.float().abs().amax(dim=-1, keepdim=True) * 2.0 ** top).to(v.dtype))
        c = Case(kind, 2, 1, 64, 64, [ctx], [n], trees([n]), edit=edit, seed=n)
        c.q.zero_()
        c.q[:, :, 0] = 1.0
        got = c.run(scale=float(np.log(2.0)))
        assert np.isfinite(got.float().cpu().numpy()).all()
        c.check(got, scale=float(np.log(2.0)))
