"""delta_verify_drafts with drawn siblings: several rejections at a row of several pieces against exact arithmetic, and
the widest tree of a large vocabulary against float64, in a time that grows with the siblings and no faster."""
import pytest
import torch

from draft_cases import offsets_of
from test_gpu_verify import Call, T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab,siblings", [(9001, 3), (9001, 6), (16385, 4), (20000, 5)])
def test_several_rejections_in_rows_of_several_pieces(vocab, siblings):
    """All siblings but the last are rejected, and that one too or not."""
    n = siblings + 1
    for last in (0.999, 0.001):
        c = Call([n, 2, n + 2], vocab, "star", True, seed=vocab + siblings, sharp=2.0, gap=siblings % 2)
        c.uniform[1:] = 0.999
        c.uniform[siblings] = last
        c.uniform[0], c.uniform[n], c.uniform[n + 2] = 0.3, 0.77, 0.9
        c.check()


def walk(target, draft, tokens, uniform):
    """A star in float64: (accepted place or None, next token's residual row, the least distance to a border)."""
    p, q = target[0].double(), draft[0].double()
    r, R, near = p.clone(), 1.0, 1.0
    for j in range(1, len(tokens)):
        x = tokens[j]
        a, b = float(uniform[j]) * float(q[x]) * R, float(r[x])
        near = min(near, abs(a - b) / max(a, b, 1e-300))
        if a < b:
            return j, target[j].double(), near
        r = (r - R * q).clamp(min=0)
        R = float(r.sum())
    return None, (r if R > 0 else p), near


@pytest.mark.parametrize("seed", [1, 2])
def test_the_widest_tree_of_a_large_vocabulary(seed):
    n, vocab = 512, 151936
    g = torch.Generator().manual_seed(seed)
    target, draft = torch.zeros((n, vocab)), torch.zeros((n, vocab))
    target[0], draft[0] = (torch.softmax(2.5 * torch.randn((vocab,), generator=g), -1) for _ in range(2))
    target[1:, 0] = 1.0
    tokens = torch.multinomial(draft[0], n, replacement=True, generator=g).int()
    uniform = torch.full((n,), 0.9999) if seed == 1 else torch.rand((n,), generator=g)
    uniform[0] = 0.61
    step, r, near = walk(target, draft, tokens.tolist(), uniform)
    assert near > 1e-9
    parents = torch.tensor([-1] + [0] * (n - 1), dtype=torch.int32)
    out = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((1, n), (1,), (1,))]
    args = (target.cuda(), draft.cuda(), tokens.cuda(), parents.cuda(), uniform.cuda(), offsets_of([n]).cuda(), *out,
            T().alloc_verify_workspace(1, vocab))
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    T().delta_verify_drafts(*args)
    torch.cuda.synchronize()
    a.record()
    T().delta_verify_drafts(*args)
    b.record()
    torch.cuda.synchronize()
    path, count, token = (x.cpu() for x in out)
    want = [0] if step is None else [0, step]
    assert path[0, :int(count)].tolist() == want and bool((path[0, len(want):] == -1).all())
    sums = r.cumsum(0) / r.sum()
    v = int(token)
    assert float(sums[v]) > 0.61 - 1e-9 and (v == 0 or float(sums[v - 1]) <= 0.61 + 1e-9) and float(r[v]) > 0
    # every sibling takes about as long as the next: some 20 us each, with all that is not the GPU's
    assert a.elapsed_time(b) < 60
