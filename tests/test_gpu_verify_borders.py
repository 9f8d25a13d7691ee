"""psa_verify_drafts right beside its borders, where sums in 32 bits must not decide: numbers of the comparison are set to 1e-6 on either side of it, which 64 bits tell apart (1e-12) and 32 do not."""
import pytest
import torch

import drafts_reference as ref
import serving_reference as sref
from paper_2012_01114_b200 import binding as psa

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rising(V, step, every, parts):
    """Numbers that rise by `step` after every `every` of them, from zero again at the beginning of each of `parts` parts."""
    i = torch.arange(V, device="cuda")
    return ((i % (V // parts) // every).double() * step).float()


@pytest.mark.parametrize("drafts", [False, True])
@pytest.mark.parametrize("step", [1518 * 2.0 ** -23, 2749 * 2.0 ** -23, 1.0e-4])
@pytest.mark.parametrize("V,every,parts,seqs", [(1 << 26, 2048, 8, 1), (11000 * 1024, 1024, 1, 300)])
def test_rows_that_rise_slowly(V, every, parts, seqs, step, drafts):
    """A new greatest number again and again, with the weight of the others hardly changed by it: what is summed up is multiplied by a factor just below one thousands of times (the steps are such that
    its 32-bit exponential is off by 1.1 to 1.3 times 2^-24, always the same way).  The child takes half of its row's weight.  Shared by eight CTAs, and by one (sequences without rows behind it)."""
    row = _rising(V, step, every, parts)
    row[V - 1] = torch.logsumexp(row[:V - 1].double(), 0).float()
    p = float(torch.softmax(row.double(), 0)[V - 1])
    other = None
    if drafts:                                   # u q(x) against p(x): the target's row is flat but for the child, of a tenth; q(x) a half
        other, row = row, torch.zeros_like(row)
        row[V - 1] = float(torch.log(torch.tensor((V - 1) / 9.0, dtype=torch.float64)))
        p = float(torch.softmax(row.double(), 0)[V - 1]) / p
    logits = torch.stack([row, row])
    q = None if other is None else torch.stack([other, other])
    for near in (-1e-6, 1e-6):
        u = torch.tensor([0.5, p * (1 + near)], device="cuda", dtype=torch.float64).float()
        want = float(u[1]) < p
        assert abs(float(u[1]) / p - 1) > 5e-7 and want == (near < 0)
        path, accepted, following = psa.psa_verify_drafts(logits, _ints([0, V - 1]), _ints([-1, 0]), sref.starts([2] + [0] * (seqs - 1)), u, drafts=q)
        assert psa.psa_last_issued()[0] == psa.OK
        assert int(accepted[0]) == int(want) and path.tolist() == [0, 1 if want else -1] and 0 <= int(following[0]) < V


def test_rows_that_rise_slowly_for_many_sequences():
    """One CTA a sequence: 260,000 numbers, the border a different one in each."""
    V, B = 260000, 300
    g = torch.Generator().manual_seed(1)
    steps = (torch.rand(B, generator=g) * 4e-3 + 1e-4).tolist()
    rows, u, want = torch.empty(2 * B, V, device="cuda"), [], []
    for b in range(B):
        row = _rising(V, steps[b], 1024, 1)
        row[V - 1] = torch.logsumexp(row[:V - 1].double(), 0).float()
        p = float(torch.softmax(row.double(), 0)[V - 1])
        rows[2 * b] = rows[2 * b + 1] = row
        near = 1e-6 if b % 2 else -1e-6
        u += [0.5, p * (1 + near)]
        want.append(int(near < 0))
    u = torch.tensor(u, dtype=torch.float64).float().cuda()
    path, accepted, following = psa.psa_verify_drafts(rows, _ints([0, V - 1] * B), _ints([-1, 0] * B), sref.starts([2] * B), u)
    assert psa.psa_last_issued()[0] == psa.OK and accepted.tolist() == want


@pytest.mark.parametrize("left", [1e-8, 1e-10, 1e-12, 1e-14])
def test_certain_drafts_behind_a_nearly_certain_token(left):
    """Children that take all but `left` of a row are refused (u = 1 - 2^-24), the next one is 1e-5 on either side of its border with what is left, which one minus a sum in 64 bits gives to 1e-16 / left.
    Behind what is left of 1e-14 no child is tried, and the token is drawn from the row as it is."""
    B, V = 128, 40
    g = torch.Generator().manual_seed(7)
    rows, u, tokens, want = [], [], [], []
    for b in range(B):
        row = torch.full((V,), -60.0)
        a, c, d = torch.rand(3, generator=g).tolist()
        heads = [0.0, -15.5 - a] if left < 5e-8 else [0.0]
        row[:len(heads)] = torch.tensor(heads)
        n = len(heads)
        row[n], row[n + 1], row[n + 2] = torch.log(torch.tensor(left, dtype=torch.float64)).float() - c, torch.log(torch.tensor(left, dtype=torch.float64)).float() - 1 - d, -55.0
        order = torch.randperm(V, generator=g)
        e = torch.exp(row.double())
        border = float(e[n] / e[n:].sum())
        near = 1e-5 if b % 2 else -1e-5
        logits = torch.empty(V)
        logits[order] = row
        rows += [logits] * (n + 2)
        tokens += [0] + [int(order[i]) for i in range(n + 1)]
        first = float(torch.rand(1, generator=g))
        u += [first] + [1 - 2.0 ** -24] * n + [border * (1 + near)]
    n += 1
    uniform = torch.tensor(u, dtype=torch.float64).float()
    parents = [-1] + [0] * n
    path, accepted, following = psa.psa_verify_drafts(torch.stack(rows).cuda(), _ints(tokens), _ints(parents * B), sref.starts([n + 1] * B), uniform.cuda())
    assert psa.psa_last_issued()[0] == psa.OK
    sure = 0
    for b in range(B):
        at = slice(b * (n + 1), (b + 1) * (n + 1))
        p, k, x, margin = ref.verify(torch.stack(rows[at]), None, tokens[at], parents, uniform[at], 1.0, True)
        if margin > 1e-7 / V:
            assert (path[at].tolist(), int(accepted[b]), int(following[b])) == (p + [-1] * (n + 1 - len(p)), k, x), (b, margin)
            sure += 1
    assert sure > 0.9 * B
