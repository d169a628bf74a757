"""The README's training example, run as it stands: the norm and both steps read the gradients of
the present step."""
import os
import re

import pytest
import torch

from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_training_example():
    need_gpu()
    from paper_2607_04422_amd import fp4root as F
    code = [b for b in re.findall(r"```python\n(.*?)```", open(README).read(), re.S) if "GradClipper" in b]
    assert len(code) == 1
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")      # noqa: E731
    w, dw, gain = rnd(64, 256).bfloat16(), rnd(64, 256), (1 + 0.1 * rnd(256)).bfloat16()
    seen = []

    class Root(F.RootStep):
        def __call__(self, step, grad_scale):
            torch.cuda.synchronize()
            dy, o = env["dy"].float(), env["o"]
            want = (dy * (o.h.float() * o.rstd[:, None])).sum(0)
            norm = (want.double().square().sum() + dw.double().square().sum()).sqrt()
            seen.append((float(env["clip"].total_norm), float(norm)))
            assert torch.allclose(env["dgain"], want, rtol=1e-4, atol=1e-4)
            super().__call__(step, grad_scale=grad_scale)
            env["dy"].mul_(2.0)                        # the next step's gradients are others
            dw.mul_(0.5)
    env = {"F": F, "torch": torch, "x": rnd(48, 256).bfloat16(), "residual": rnd(48, 256).bfloat16(), "gain": gain,
           "dy": rnd(48, 256).bfloat16(), "dh": rnd(48, 256).bfloat16(), "dw": dw, "root": Root([w], [dw], 0.02),
           "state": F.QAdamWState(256), "steps": 3, "step": 0}
    exec(code[0], env)
    # dgain's sum of 48 products in binary32 on either side: 2 48 2^-24 at most of their magnitudes,
    # far below the factors of 2 between the steps
    assert len(seen) == 3 and all(abs(a - b) <= 1e-4 * b for a, b in seen), seen
