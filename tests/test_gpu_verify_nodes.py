"""readme_verify_drafts on the GPU: nodes with many drafts."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1100, 9001])
@pytest.mark.parametrize("kind", ["given", "distinct", "certain"])
def test_hundreds_of_refusals_at_a_node(kind, V, dtype):
    """Up to 1000 drafts of one node, refused one after the other, many of them of a
    token refused up to 500 drafts before; the first two requests take their last."""
    new = [1001, 400, 700, 131]
    c = Case(new, V, 1, kind, dtype, seed=V, sharp=1.0)
    rng, o = np.random.default_rng(V), 0
    c.parent[:] = 0
    c.u[:] = 1.0 - 2.0 ** -24
    for r, n in enumerate(new):
        if c.q is not None:
            c.q[o, V - V // 8:] = 0.0  # what is left of p in the end
        p = c.p[o].double().cpu().numpy()
        q = p * 0 + 1.0 if c.q is None else c.q[o].double().cpu().numpy()
        # Refused by the first draft's factor, so that nothing is left of p there; of
        # certain drafts, entries far below what is left
        low = np.nonzero(q > 2 * p)[0] if c.q is not None else np.nonzero(p < 4.0 / V)[0]
        low = rng.permutation(low)[:n // 2]
        assert len(low) > 60
        c.tokens[o + 1:o + n] = np.concatenate([low, rng.choice(low, n)])[:n - 1]
        c.u[o] = (0.3, 0.7, 0.001, 0.9)[r]
        if r < 2:
            c.tokens[o + n - 1] = V - 1 - r
            c.u[o + n - 1] = 0.0
        o += n
    acc, tok = c.check()
    assert (acc == [1, 1, 0, 0]).all() and (tok >= 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("held", [[5, 6, 7], [5, 20000, 69999], [4607, 4608, 70000], [0, 70000], [35000]])
def test_drafts_that_held_all_of_q(held, dtype):
    """Without replacement, all of q lies on the tokens that are refused first: what
    later drafts are tried with is 0, so one is taken if anything is left of its token,
    and refused, with nothing changed, if not."""
    V, n = 70001, 10
    c = Case([n] * 3, V, 1, "distinct", dtype, seed=21)
    c.parent[:] = 0
    c.q[:] = 0.0
    k = len(held)
    behind = ([held[0], 12, 13, held[-1], 14], [12, held[0], 13, 12, 13], [12, 13, 900, 12, 13])
    for r in range(3):
        o = r * n
        c.q[o, held] = torch.tensor([0.5, 0.3, 0.2][:k]).to(dtype).cuda()
        c.p[o, held] = 1e-3
        c.p[o, 12:14] = 0.0
        c.tokens[o + 1:o + 1 + k] = held
        c.tokens[o + 1 + k:o + 6 + k] = behind[r]
        c.tokens[o + 6 + k:o + n] = 12
        c.u[o:o + n] = [0.5] + [0.9] * (n - 1)
    acc, tok = c.check(safe=False)
    assert (acc == [1, 0, 1]).all() and (tok >= 0).all()
