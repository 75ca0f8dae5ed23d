"""readme_verify_drafts on the GPU: what its results depend on."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["given", "distinct", "certain"])
def test_rows_off_the_path_mean_nothing(kind, dtype):
    """Rows that the path does not visit, drafts below them among them, hold what they
    like: the path, the counts and the tokens stay, though entries of theirs are read."""
    for seed in range(3):
        c = Case([24, 3, 0, 90, 1], 1100, 5, kind, dtype, seed=seed, sharp=2.0)
        c.check()
        ref, o = c.run(), 0
        visited = np.zeros(sum(c.new), bool)
        for n in c.new:
            path = ref[0][o:o + n].cpu().numpy()
            visited[o + path[path >= 0]] = True
            o += n
        off = torch.from_numpy(~visited).cuda()
        assert off.any() and not off.all()
        for fill in (float("nan"), float("inf"), -3e38, 3e38):
            for rows in (c.p, c.q):
                if rows is not None:
                    rows[off] = fill
            for a, b in zip(c.run(), ref):
                assert torch.equal(a, b)
