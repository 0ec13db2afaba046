"""GPU tests of the shared-prefix serving operators at the edges of what they accept: values near
the largest of their type.  Oracle and tolerances are those of test_gpu_serve.py.
"""
import pytest
import torch

from test_gpu_serve import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,T", [([1, 1, 1], 50), ([1, 1, 1], 700), ([40, 2, 37], 700)])
def test_large_values_under_rising_scores(dtype, new, T):
    """Values up to 3e38 whose scores rise along the prefix: every output is a mean of them and
    finite, also where weights against an early maximum would sum past fp32."""
    for mag in (1e35, 1e37, 2e38):
        b = Batch(dtype, T, [60, 5, 17], new, 2, 4, 64, 16)

        def limit(x):
            return (x.double().clamp(-1.5, 1.5) * mag).to(x.dtype)
        for x in (b.V, b.Vp):
            x.copy_(limit(x))
        b.tv = [limit(v) for v in b.tv]
        u = torch.randn(64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        b.K[1] = u * torch.linspace(0.05, 2.5, T, device="cuda")[None, :, None] + 0.02 * b.K[1].float()
        b.Q.copy_(u + 0.1 * b.Q.float())
        b.check(b.run(max_new=max(new)), b.want())
