"""Drafted tokens judged, against the rules of include/lc_serve.h one node after the other in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def lc():
    from paper_2009_13003_amd import lc
    return lc


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def judge(target, tokens, uniform, draft=None, parent=None, count=None):
    """Paths and tokens by the rules, and how near the running sum came to what was wanted of it, of the whole sum."""
    clean = lambda t: np.where(np.isfinite(t) & (t > 0), t, 0.0)
    p_all = clean(target.double().cpu().numpy())
    q_all = clean(draft.double().cpu().numpy()) if draft is not None else None
    tokens, u = tokens.tolist(), uniform.double().tolist()
    batch, nodes, vocab = p_all.shape
    paths, lengths, nexts, near = [], [], [], 1.0
    for b in range(batch):
        n = nodes if count is None else min(max(int(count[b]), 1), nodes)
        path, walking = [0], True
        while walking:
            cur, walking = path[-1], False
            left, rest, gone = p_all[b, cur].copy(), 1.0, False
            for i in range(cur + 1, n):
                above = i - 1 if parent is None else int(parent[b][i])
                if above != cur:
                    continue
                t = tokens[b][i]
                if draft is not None:
                    p, q = (p_all[b, cur, t], q_all[b, i - 1, t]) if 0 <= t < vocab else (0.0, 0.0)
                    take = u[b][i] * q < p
                    left = np.maximum(p_all[b, cur] - q_all[b, i - 1], 0.0)
                else:
                    p = left[t] if 0 <= t < vocab else 0.0
                    take = u[b][i] * rest < p
                    rest -= p
                    if 0 <= t < vocab:
                        left[t] = 0.0
                if take:
                    path.append(i)
                    walking = True
                    break
        if not left.sum() > 0:
            left = p_all[b, cur]
        run = np.cumsum(left)
        paths.append(path + [-1] * (nodes - len(path)))
        lengths.append(len(path))
        if not run[-1] > 0:
            nexts.append(-1)
            continue
        nexts.append(int(np.argmax(run > u[b][0] * run[-1])))
        near = min(near, np.abs(run - u[b][0] * run[-1]).min() / run[-1])
    return paths, lengths, nexts, near


def compare(lc, *a, **kw):
    """Equal, since sums in 64 bits of up to 2^17 numbers are right to 2^-36 of the whole and no running sum of these inputs comes that near to what is wanted."""
    paths, lengths, nexts, near = judge(*a, **kw)
    got = lc.lc_draft_verify(*a, **kw)
    assert near > 2.0 ** -36 and a[0].shape[2] <= 1 << 17
    assert got["path"].tolist() == paths and got["count"].tolist() == lengths and got["next"].tolist() == nexts
    return lengths, nexts


def made(seed, batch, nodes, vocab, dtype, tree, near=0.4):
    g = torch.Generator(DEV).manual_seed(seed)
    logits = 2 * torch.randn(batch, nodes, vocab, device=DEV, generator=g)
    target = torch.softmax(logits, -1).to(dtype)
    uniform = torch.rand(batch, nodes, device=DEV, generator=g).clamp(min=2.0 ** -20)
    tokens = torch.zeros(batch, nodes, dtype=torch.int32, device=DEV)
    if tree:
        parent = ints([[-1] + [max(0, i - 1 - int(x * i)) for i, x in zip(range(1, nodes), torch.rand(nodes - 1, generator=g, device=DEV).tolist())] for _ in range(batch)])
        likely = target.float().topk(min(vocab, 3), -1).indices
        above = parent.long().clamp(min=0)
        tokens = torch.gather(likely, 1, above[..., None].expand(-1, -1, likely.shape[-1]))
        tokens = torch.gather(tokens, 2, torch.randint(likely.shape[-1], (batch, nodes, 1), device=DEV, generator=g))[..., 0].to(torch.int32)
        return target, tokens, uniform, None, parent
    draft = torch.softmax(logits[:, :nodes - 1] + near * torch.randn(batch, nodes - 1, vocab, device=DEV, generator=g), -1).to(dtype)
    if nodes > 1:
        tokens[:, 1:] = torch.multinomial(draft.float().view(-1, vocab), 1, generator=g).view(batch, nodes - 1).to(torch.int32)
    return target, tokens, uniform, draft, None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,nodes,vocab", [(1, 1, 1), (1, 2, 1), (1, 5, 32000), (7, 9, 1000), (3, 64, 257), (20, 4, 2048), (5, 3, 2049), (40, 9, 50257), (1, 2, 131072), (800, 3, 50)])
@pytest.mark.parametrize("tree", [False, True])
def test_sizes(lc, batch, nodes, vocab, dtype, tree):
    target, tokens, uniform, draft, parent = made(batch + nodes, batch, nodes, vocab, dtype, tree)
    lengths, _ = compare(lc, target, tokens, uniform, draft, parent)
    if batch >= 20 and not tree:                             # (guesses among 2048 tokens are seldom right)
        assert len(set(lengths)) > 1                         # (some are taken and some are not)


@pytest.mark.parametrize("tree", [False, True])
def test_fewer_nodes(lc, tree):
    target, tokens, uniform, draft, parent = made(3, 30, 6, 300, torch.float32, tree, near=0.05)
    compare(lc, target, tokens, uniform, draft, parent, ints([0, 1, 2, 3, 4, 5, 6, 7, -2, 100] * 3))


def test_guesses_in_a_row(lc):
    """Neither what they were drawn from nor parents: each below the one before."""
    target, tokens, uniform, _, _ = made(4, 50, 5, 12, torch.float32, False)
    lengths, _ = compare(lc, target, tokens, uniform)
    assert len(set(lengths)) > 2


def test_the_same_guess_twice(lc):
    """Refused once it has no probability left; and the vocabulary's last token among the refused."""
    p = torch.tensor([0.5, 0.25, 0.125, 0.125], device=DEV).repeat(1, 4, 1)
    tokens, parent = ints([[0, 3, 3, 3]]), ints([[-1, 0, 0, 0]])
    u = torch.tensor([[0.99, 0.5, 2.0 ** -20, 2.0 ** -20]], device=DEV)
    got = lc.lc_draft_verify(p, tokens, u, parent=parent)
    assert got["path"].tolist() == [[0, -1, -1, -1]] and got["next"].tolist() == [2]
    compare(lc, p, tokens, u, None, parent)


def test_refused_one_after_the_other(lc):
    """1 less what was refused: 0.5 of 1, 0.25 of 0.5, then all of what is left."""
    p = torch.tensor([0.5, 0.25, 0.25, 0.0], device=DEV).repeat(1, 4, 1)
    tokens, parent = ints([[0, 0, 1, 2]]), ints([[-1, 0, 0, 0]])
    for u1, u2, u3, want in ((0.49, 0.9, 0.9, 1), (0.5, 0.49, 0.9, 2), (0.5, 0.5, 0.99, 3)):
        got = lc.lc_draft_verify(p, tokens, torch.tensor([[0.1, u1, u2, u3]], device=DEV), parent=parent)
        assert got["path"].tolist() == [[0, want, -1, -1]] and got["count"].tolist() == [2]


def test_parents_that_are_none(lc):
    """A node above itself, or below itself, or of the lowest number: never reached."""
    p = torch.full((1, 4, 5), 0.2, device=DEV)
    u = torch.zeros(1, 4, device=DEV)
    got = lc.lc_draft_verify(p, ints([[0, 1, 2, 3]]), u, parent=ints([[0, 1, 3, -2147483648]]))
    assert got["path"].tolist() == [[0, -1, -1, -1]] and got["next"].tolist() == [0]


@pytest.mark.parametrize("draft", [True, False])
def test_tokens_outside_the_vocabulary(lc, draft):
    p = torch.full((3, 2, 8), 0.125, device=DEV)
    u = torch.zeros(3, 2, device=DEV)
    got = lc.lc_draft_verify(p, ints([[0, 8], [0, -1], [0, 7]]), u, p[:, :1] if draft else None)
    assert got["count"].tolist() == [1, 1, 2]


def test_numbers_that_are_no_probabilities(lc):
    """Negative ones, infinities and NaN count as zero; rows of zeros give -1; where p never exceeds q the token is drawn from p."""
    inf, nan = float("inf"), float("nan")
    p = torch.tensor([[0.25, -1.0, nan, inf, 0.5, -inf, 0.25, 0.0]], device=DEV).repeat(4, 2, 1)
    p[2] = 0
    p[3] = nan
    u = torch.tensor([[0.3, 0.0], [0.9, 0.0], [0.5, 0.0], [0.5, 0.0]], device=DEV)
    got = lc.lc_draft_verify(p, ints([[0, 3], [0, 2], [0, 0], [0, 0]]), u)
    assert got["count"].tolist() == [1] * 4 and got["next"].tolist() == [4, 6, -1, -1]
    p = torch.full((1, 2, 4), 0.25, device=DEV)
    p[..., 3] = 0
    got = lc.lc_draft_verify(p, ints([[0, 3]]), torch.tensor([[0.5, 0.5]], device=DEV), torch.full((1, 1, 4), 0.25, device=DEV))
    assert got["count"].tolist() == [1] and got["next"].tolist() == [1]


@pytest.mark.parametrize("u0", [0.0, 0.5, 1.0 - 2.0 ** -24, 1.0, 2.0, float("nan")])
def test_the_ends_of_the_random_numbers(lc, u0):
    """0: the first token that has any probability; from 1 on, which is not in their range, the last one."""
    p = torch.zeros(1, 1, 5000, device=DEV)
    p[0, 0, 7], p[0, 0, 4000], p[0, 0, 4990] = 0.25, 0.5, 0.25
    got = lc.lc_draft_verify(p, ints([[0]]), torch.tensor([[u0]], device=DEV))["next"].tolist()
    assert got == [7 if u0 == 0 else 4000 if u0 == 0.5 else 4990]


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_with_pitches(lc, dtype):
    """Rows off 16 bytes and apart."""
    target, tokens, uniform, draft, _ = made(9, 6, 4, 2051, dtype, False)
    wide, wide_q = torch.full((7, 5, 2060), 1.0, dtype=dtype, device=DEV), torch.full((6, 4, 2099), 1.0, dtype=dtype, device=DEV)
    wide[:6, :4, 3:2054], wide_q[:, 1:, 1:2052] = target, draft
    compare(lc, wide[:6, :4, 3:2054], tokens, uniform, wide_q[:, 1:, 1:2052])


def test_the_distribution(lc):
    """Tokens behind a drafted one have the model's probabilities, whatever they were drawn from: of 40000 draws each of 6 tokens within 5 standard deviations."""
    n, vocab = 40000, 6
    g = torch.Generator(DEV).manual_seed(1)
    p, q = (torch.softmax(torch.randn(vocab, device=DEV, generator=g), 0) for _ in range(2))
    seen = torch.zeros(vocab)
    for at in range(0, n, 10000):
        tokens = torch.zeros(10000, 2, dtype=torch.int32, device=DEV)
        tokens[:, 1] = torch.multinomial(q, 10000, replacement=True, generator=g).to(torch.int32)
        got = lc.lc_draft_verify(p.expand(10000, 2, vocab), tokens, torch.rand(10000, 2, device=DEV, generator=g), q.expand(10000, 1, vocab).contiguous())
        first = torch.where(got["count"] == 2, tokens[:, 1], got["next"])
        seen += torch.bincount(first.long(), minlength=vocab).cpu()
    want = p.cpu().double()
    assert ((seen.double() / n - want).abs() <= 5 * (want * (1 - want) / n).sqrt()).all()


def test_no_sequences(lc):
    got = lc.lc_draft_verify(torch.empty(0, 3, 10, device=DEV), torch.empty(0, 3, dtype=torch.int32, device=DEV), torch.empty(0, 3, device=DEV))
    assert got["path"].shape == (0, 3) and got["next"].shape == (0,)


def test_on_another_stream_and_in_a_graph(lc):
    target, tokens, uniform, draft, _ = made(5, 12, 5, 9000, torch.float32, False)
    _, _, want, _ = judge(target, tokens, uniform, draft)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = lc.lc_draft_verify(target, tokens, uniform, draft, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert got["next"].tolist() == want
    ws = lc.new_draft_workspace(12)
    ws.fill_(0x5a)
    out = (torch.empty(12, 5, dtype=torch.int32, device=DEV), torch.empty(12, dtype=torch.int32, device=DEV), torch.empty(12, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lc.lc_draft_verify(target, tokens, uniform, draft, out=out, ws=ws)
    g = torch.Generator(DEV).manual_seed(2)
    for _ in range(4):
        uniform.copy_(torch.rand(12, 5, device=DEV, generator=g).clamp(min=2.0 ** -20))
        paths, lengths, nexts, near = judge(target, tokens, uniform, draft)
        graph.replay()
        assert out[0].tolist() == paths and out[1].tolist() == lengths and out[2].tolist() == nexts
        assert lc.lc_draft_verify(target, tokens, uniform, draft, ws=ws)["next"].tolist() == nexts


def test_refused(lc):
    target, tokens, uniform, draft, _ = made(5, 2, 3, 20, torch.float32, False)
    parent = ints([[-1, 0, 1]] * 2)
    with pytest.raises(lc.LcError):
        lc.lc_draft_verify(target, tokens, uniform, draft, parent)
    with pytest.raises(AssertionError):
        lc.lc_draft_verify(target, tokens.long(), uniform)
    with pytest.raises(AssertionError):
        lc.lc_draft_verify(target.requires_grad_(), tokens, uniform)
    with pytest.raises(lc.LcError):
        lc.lc_draft_verify(target.detach(), tokens, uniform, ws=torch.empty(64, dtype=torch.uint8, device=DEV))
