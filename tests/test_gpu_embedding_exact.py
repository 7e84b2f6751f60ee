"""The embedding's gradient in whole numbers: dy within 3 and scale 1, so that every partial sum of any order is exact in
fp32 (3 n below 2^24) and the result has to equal the sum in integers.  The tokens come in runs that, sorted, end beside the
borders of the chunks and groups in which they are added up, and go on through more groups than are looked for at once."""
import pytest
import torch

from gpu_util import announce, has_gpu
from test_gpu_embedding import DT, TOK

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not has_gpu(), reason="needs a GPU")]


def check(counts, V, d, tok, dtype, seed, first=0):
    """counts[i] tokens of value first + i, and a twentieth of them padding (not for bytes), in any order."""
    import paper_2401_13660_amd as mb
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    t = torch.repeat_interleave(torch.arange(first, first + len(counts), device="cuda:0"),
                                torch.tensor(counts, device="cuda:0"))
    if tok != "u8":
        t = torch.cat([t, torch.full((len(t) // 20,), -1, device="cuda:0")])
    t = t[torch.randperm(len(t), generator=g, device="cuda:0")]
    dy = torch.randint(-3, 4, (len(t), d), generator=g, device="cuda:0")
    got = mb.embedding_bwd(t.to(TOK[tok]), dy.to(DT[dtype]), V)
    ref = torch.zeros(V + 1, d, dtype=torch.int64, device="cuda:0").index_add_(0, torch.where(t < 0, V, t), dy)[:V]
    wrong = (got.double() != ref.double()).any(1).nonzero().flatten().tolist()
    assert not wrong, f"rows {wrong[:8]} of {V}"


# groups are of 64 tokens here (128 and 256 below); 64 of them are looked through at a time
@pytest.mark.parametrize("tok,V,first", [("u8", 256, 0), ("i32", 300, 40), ("i64", 70000, 65000)])
@pytest.mark.parametrize("groups", [1, 2, 63, 64, 65, 66, 127, 128, 129, 130, 200])
def test_runs_through_many_groups(tok, V, first, groups):
    announce(f"embedding_bwd exact: runs of {groups} groups, V={V} {tok}")
    for by in (-1, 0, 1):
        n = 64 * groups + by
        check([n], V, 12, tok, "bf16", n, first)
        check([3, n, 60, n, 1, n + 7, 5000], V, 12, tok, "f32", n, first)


@pytest.mark.parametrize("n,d,group", [(40000, 260, 128), (20000, 2048, 256), (40000, 2048, 256), (70000, 512, 256)])
def test_larger_groups(n, d, group):
    announce(f"embedding_bwd exact: n={n} d={d}")
    for run in (group - 1, group, group + 1, 64 * group - 1, 64 * group, 64 * group + 1, 70 * group):
        check([group // 2, run, max(1, n - run)], 256, d, "i32", "bf16", run)


@pytest.mark.parametrize("tok", ["u8", "i32", "i64"])
@pytest.mark.parametrize("n", [1, 64, 500, 2048, 2049, 4096, 4097, 32768, 32769, 262145, 1000003])
def test_texts(tok, n):
    """A few common values, many rare ones: every way of sorting and adding up."""
    announce(f"embedding_bwd exact: {n} tokens of a text, {tok}")
    for V in (256, 1000, 70000) if tok != "u8" else (256,):
        share = torch.arange(1, V + 1).double().reciprocal()
        counts = (share / share.sum() * n).round().long().tolist()
        counts[0] += n - sum(counts)
        check(counts, V, 9, tok, "bf16", n)
