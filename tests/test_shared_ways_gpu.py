"""Every way that the kernels of attention behind shared prefixes share the work (shared_cases.py), against the definition in 64 bits."""
import pytest
import torch

from attention_reference import check
from gpu_util import announce
from paper_2203_05016_amd import binding
from shared_cases import CASES
from test_shared_attention_gpu import DEV, DTYPE, Served, _tensor

pytestmark = pytest.mark.gpu


def served(case):
    """The case's cache; its prefixes' table has room for what the host says is the longest."""
    s = Served(list(case.prefix), case.families, list(case.own), case.heads, case.D, case.page, DTYPE[case.fmt])
    width = -(-case.most // case.page)
    if s.prefix_table.shape[1] < width:
        wide = torch.full((len(case.prefix), width), -7, dtype=torch.int32, device=DEV)
        wide[:, :s.prefix_table.shape[1]] = s.prefix_table
        s.prefix_table = wide
    return s


@pytest.mark.parametrize("case", CASES, ids=lambda c: c.name)
def test_definition(case):
    announce("shared, ways", case.name)
    s = served(case)
    q = _tensor(case.q_heads * case.D, sum(case.counts), DTYPE[case.fmt], 9)
    want, tol = s.want(q, case.counts)
    bounds = dict(max_length=max(case.own), max_prefix=case.most, max_sharing=case.sharing)
    q = q.to(DEV)
    got = s.call(q, case.counts, **bounds)
    kernel = case.plan.get("own" if case.plan["behind"] else "prefix")
    if kernel is not None:
        name = "decode_kernel<%d,%d columns" % (case.D, 16 * kernel["col_tiles"]) if kernel["decode"] else "tile_kernel<%d,cache,%d wavefronts" % (case.D, kernel["waves"])
        assert binding.last_kernel().startswith("shflbw_attention_" + name)
    check(got, want, tol, case.name)
    for _ in range(3):
        assert torch.equal(got, s.call(q, case.counts, **bounds))
