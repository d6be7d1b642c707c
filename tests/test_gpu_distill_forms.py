"""The distillation loss on either side of every length at which a row is held
otherwise: steps of a block's waves that are whole for all threads, a partial last
one, rows that no block holds; few tokens and many."""

import pytest

torch = pytest.importorskip("torch")

from paper_2301_09830_amd import optcc  # noqa: E402
from test_gpu_distill import check, inputs  # noqa: E402

pytestmark = pytest.mark.gpu

# bf16 elements; fp32 rows change at half of them
FEW = [2047, 2048, 2049, 6143, 6144, 8193, 24575, 24576, 32768, 40961, 57343, 57344, 65537, 73728,
       139263, 139264]
MANY = [6143, 6144, 10239, 10240, 18431, 18432, 34815, 34816, 36863, 36864, 69631, 69632, 73727]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", FEW)
def test_few_tokens(v, dtype):
    v = v if dtype == "bf16" else v // 2
    S, index, teacher, labels, scale = inputs(5, v, 9, dtype, seed=v)
    check(S, index, teacher, 2.0, 0.5, labels, scale)      # two exponentials a logit
    check(S, index, teacher, 1.0, 0.5, labels, scale)      # one


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", MANY)
def test_many_tokens(v, dtype):
    v = v if dtype == "bf16" else v // 2
    S, index, teacher, labels, scale = inputs(512, v, 9, dtype, seed=v)
    check(S, index, teacher, 2.0, 0.5, labels, scale)


@pytest.mark.parametrize("k", [63, 64, 65, 255, 1023, 1024])
@pytest.mark.parametrize("tokens", [3, 520])
def test_lengths_of_the_list(tokens, k):
    """Every wave stores the entries whose columns it holds; the label is the last."""
    for dtype, v in (("bf16", 20000), ("f32", 9001)):
        S, index, teacher, labels, scale = inputs(tokens, v, k, dtype, seed=k)
        index[:, k // 2] = index[:, 0]
        labels[1] = index[1, k - 1]
        check(S, index, teacher, 2.0, 0.5, labels, scale)


@pytest.mark.parametrize("tokens", [4, 600])
def test_entries_in_every_column_of_a_row(tokens):
    """The vocabulary itself as the teacher's list, and every label's column in it."""
    for dtype in ("bf16", "f32"):
        S, _, _, labels, scale = inputs(tokens, 1000, 1, dtype, seed=2)
        index = torch.randperm(1000, device="cuda").to(torch.int32).expand(tokens, -1).contiguous()
        check(S, index, S.gather(1, index.long()), 3.0, 0.5, labels, scale)


def test_results_do_not_depend_on_the_other_tokens():
    """A token's loss and gradient are those of its row alone in the form that the call
    takes: rows of one call permuted give permuted results."""
    S, index, teacher, labels, scale = inputs(530, 5000, 20, "bf16", seed=3)
    turn = torch.randperm(530, device="cuda")

    def run(p):
        dS = torch.empty_like(S)
        loss = optcc.occ_distill_fwd(S[p], index[p], teacher[p], temperature=2.0, alpha=0.3,
                                     labels=labels[p], scale=scale[p], dS=dS)
        return loss, dS

    same = torch.arange(530, device="cuda")
    for a, b in zip(run(same), run(turn)):
        assert torch.equal(a[turn], b)
