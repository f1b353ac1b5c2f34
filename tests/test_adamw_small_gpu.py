"""8-bit moments of gradients whose squares float32 hardly holds."""
import pytest
import torch

from paper_2608_05088_amd import libmalt as lm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lm.lib()
    from paper_2608_05088_amd import ops as module
    return module


def test_first_moments_go_with_the_second(ops):
    """Gradients of 1e-15 to 2e-15: second moments (at most 0.05 x 4e-30) below 2^-100, a block of zeros.  A first moment
    that stayed would be divided by eps alone in a step without a gradient.  Without either a step is
    |m| / sqrt(v) with m = 0.1 g, v = 0.05 g^2 and their bias corrections (1 - 0.9^t, 1 - 0.95^t): 1 at
    t = 1 and less later."""
    n, lr = 600, 1e-3
    g = (1.0 + torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))) * 1e-15
    p = [torch.zeros(n, device="cuda")]
    st = [ops.adamw_state(p[0], 8)]
    for t in range(1, 30):
        before = p[0].clone()
        ops.adamw_step(p, [g if t < 6 else torch.zeros_like(g)], st, lr=lr, betas=(0.9, 0.95), eps=1e-20, weight_decay=0.0,
                       step=t, seed=t)
        # Rounded: the update by 12 2^-24 of itself, the sum by half a step of p (below 8 lr).
        assert float((p[0] - before).abs().max()) <= lr * (1 + 1e-5)
        m, v = ops.adamw_moments(p, st)[0]
        assert bool((m == 0).all()) and bool((v == 0).all())


def test_other_blocks_keep_their_first_moments(ops):
    """A block beside it, whose second moments are 2^-99 and more, keeps both."""
    g = torch.full((512,), 1e-15, device="cuda")
    g[256:] = 1e-14
    p = [torch.zeros(512, device="cuda")]
    st = [ops.adamw_state(p[0], 8)]
    ops.adamw_step(p, [g], st, lr=1e-3, betas=(0.9, 0.95), eps=1e-20, weight_decay=0.0, step=1, seed=1)
    m, v = ops.adamw_moments(p, st)[0]
    assert bool((m[:256] == 0).all()) and bool((v[:256] == 0).all())
    # All equal, so each is its block's largest: its code is the largest, and the scale holds it to float32.
    assert bool(((m[256:] - 1e-15).abs() <= 1e-21).all()) and bool(((v[256:] / (0.05 * 1e-28) - 1).abs() <= 1e-6).all())
