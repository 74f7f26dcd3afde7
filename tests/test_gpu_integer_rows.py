"""The integer rows where a workgroup has several rows one after the other, in every width of team, and the norms' runs of rows in the
width that the other tests leave out: a maximum or a sum left over from another row would show."""
import numpy as np
import pytest
import torch

from oracle import integer as ref
from paper_2607_12121_amd import flashdiff as fdl
from tests import gpu_harness as gh
from tests.test_gpu_integer import FILL, ints
from tests.test_gpu_integer_run import test_norm_runs as norm_runs
from tests.test_gpu_scaled import bf16, count

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    fdl.lib()


# teams of 16 lanes (16 rows a workgroup), 32, 64 and 64 of twice the columns, three and four waves, four of two and of four times the
# columns, 16 of four and of eight times; more rows than 4096 workgroups take at once, and a few of a width that had none
@pytest.mark.parametrize("rows,cols,m", [(70001, 64, None), (40001, 208, 40000), (17001, 400, None), (17001, 1008, 16999), (9001, 1536, 8999), (8999, 2048, None),
                                         (8300, 1552, 8299), (4400, 3088, None), (4500, 4112, 4499), (4300, 8208, 4200), (4111, 32784, 4110), (5, 1552, None), (7, 208, 6)])
def test_rows_one_after_the_other(rows, cols, m):
    """Neighbouring rows differ in magnitude by factors of up to e^12 and more; the bits are the definition's, every step of it being one rounding."""
    gh.say(f"int8 rows {rows}x{cols} m={m}")
    rng = np.random.default_rng([rows, cols])
    base = bf16(rng.standard_normal((61, cols)) * np.exp(4 * rng.standard_normal((61, 1))))
    base[7], base[30, cols - 1] = 0, float("nan")
    pick = torch.arange(rows, device="cuda") * 37 % 61
    x = base.cuda()[pick]
    q, s = ints(rows, cols)
    fdl.fd_int_rows(x, q, s, m=None if m is None else count(m))
    wq, ws = (torch.from_numpy(t).cuda() for t in ref.int_rows(base.float().numpy()))
    n = rows if m is None else m
    assert torch.equal(q[:n], wq[pick[:n]])
    assert torch.equal(s[:n].view(torch.int32), ws[pick[:n]].view(torch.int32))
    assert bool((q[n:] == FILL).all()) and bool((s[n:] == -7).all())


@pytest.mark.parametrize("to", ["bf16", "codes", "ints"])
@pytest.mark.parametrize("rows,D,B,m", [(3100, 2048, 5, 3099), (2300, 1552, 40, 2300)])
def test_norm_runs_of_four_waves(rows, D, B, m, to):
    norm_runs(rows, D, B, m, to)
