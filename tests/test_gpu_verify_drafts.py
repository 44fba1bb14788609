"""squat_verify_drafts against its definition, token by token in numpy (64 bits): whole numbers, equal."""
import numpy as np
import pytest
import torch

from paper_2503_24358_amd import squat

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _ref(tokens, target, draft, u, u_next, n_draft=None):
    b, k = tokens.shape
    v = target.shape[2]
    accepted, out = np.zeros(b, np.int32), np.full((b, k + 1), -1, np.int64)
    for s in range(b):
        n = k if n_draft is None else min(max(int(n_draft[s]), 0), k)
        j = 0
        while j < n:
            x = int(tokens[s, j])
            inside = 0 <= x < v
            q = (draft[s, j, x] if draft is not None else 1.0) if inside else 1.0
            if not (float(u[s, j]) * float(q) < (float(target[s, j, x]) if inside else 0.0)):
                break
            j += 1
        p = target[s, j].astype(np.float64)
        r = p
        if j < n:
            if draft is not None:
                r = np.maximum(p - draft[s, j], 0)
            elif 0 <= tokens[s, j] < v:
                r = p.copy()
                r[tokens[s, j]] = 0
        if not r.sum() > 0:
            r = p
        over = np.flatnonzero(np.cumsum(r) > float(u_next[s]) * r.sum())
        positive = np.flatnonzero(r > 0)
        out[s, :j] = tokens[s, :j]
        out[s, j] = over[0] if len(over) else (positive[-1] if len(positive) else 0)
        accepted[s] = j
    return accepted, out


def _inputs(seed, b, k, v, dtype, sharp=2.5, noise=0.7):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn(b, k + 1, v, generator=g) * sharp
    target = torch.softmax(logits, -1).to(DT[dtype])
    draft = torch.softmax(logits[:, :k] + noise * torch.randn(b, k, v, generator=g), -1).to(DT[dtype])
    tokens = torch.stack([torch.multinomial(draft[s].float().clamp(min=1e-9), 1, generator=g)[:, 0] for s in range(b)]) if k else torch.zeros(b, 0, dtype=torch.int64)
    return tokens, target, draft, torch.rand(b, k, generator=g), torch.rand(b, generator=g)


def _check(tokens, target, draft, u, u_next, n_draft=None):
    dev = lambda t: None if t is None else t.cuda()       # noqa: E731
    acc, out = squat.verify_drafts(dev(tokens), dev(target), dev(draft), dev(u), dev(u_next), n_draft=dev(n_draft))
    wide = lambda t: None if t is None else t.double().numpy()    # noqa: E731
    want = _ref(tokens.numpy(), wide(target), wide(draft), u.numpy(), u_next.numpy(), None if n_draft is None else n_draft.numpy())
    assert np.array_equal(acc.cpu().numpy(), want[0])
    assert np.array_equal(out.cpu().numpy(), want[1])
    return want


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [1, 2, 7, 255, 1000, 4095, 4096, 4097, 32001])
def test_vocabularies(dtype, vocab):
    _check(*_inputs(vocab, 9, 4, vocab, dtype))


@pytest.mark.parametrize("drafts", [0, 1, 2, 5, 8, 63, 64])
def test_draft_counts(drafts):
    t = _inputs(drafts, 5, drafts, 501, "f32", noise=0.05)
    _check(*t)
    _check(t[0], t[1], None, t[3] * 0.05, t[4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_drafts_chosen_outright(dtype):
    tokens, target, _, u, u_next = _inputs(3, 40, 3, 700, dtype, sharp=6.0)
    tokens = target[:, :3].float().argmax(-1)
    acc, _ = _check(tokens, target, None, u, u_next)
    assert 0 < (acc == 3).sum() < 40


def test_a_sequence_of_its_own_number_of_drafts():
    t = _inputs(4, 12, 6, 333, "f32", noise=0.1)
    _check(*t, n_draft=torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, -1, 100, 6, 0], dtype=torch.int32))


def test_more_pieces_than_threads():
    _check(*_inputs(5, 2, 1, 1100003, "f32"))


def test_borders():
    """Numbers of 0, the largest below 1, probabilities of 0 and 1, rows without anything, a residual that is zero everywhere."""
    v, below = 5000, float(np.nextafter(np.float32(1), np.float32(0)))
    one = torch.zeros(6, 3, v)
    one[:, :, 4999] = 1.0
    one[0, 0] = 0                                         # a row without a positive entry: refused, token 0
    one[1, 0] = 0
    one[1, 0, 4097] = 0.25
    one[2] = 1.0 / 4096                                   # equal weights that sum up exactly: marks fall on borders
    one[3, 1] = 0
    one[3, 1, [5, 4099]] = 0.5
    tokens = torch.tensor([[4999, 0], [3, 0], [17, 4097], [4999, 5], [4999, 4999], [-1, 9]])
    for u, w in ((0.0, 0.0), (0.5, 0.5), (below, below), (0.25, 0.75)):
        a, b = torch.full((6, 2), u), torch.full((6,), w)
        _check(tokens, one, one[:, :2].clone(), a, b)     # draft = target: a refusal leaves a residual of zero
        _check(tokens, one, None, a, b)
        _check(tokens, one, torch.full((6, 2, v), 2.0), a, b)


def test_tokens_outside_the_vocabulary_are_refused():
    tokens, target, draft, u, u_next = _inputs(6, 4, 2, 100, "f32", noise=0.01)
    tokens[0, 0], tokens[1, 1], tokens[2, 0] = 100, -1, 1 << 40
    for d in (draft, None):
        acc, _ = _check(tokens, target, d, u * 0.01, u_next)
        assert acc[0] == 0 and acc[1] <= 1 and acc[2] == 0


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_strides_and_given_outputs(dtype):
    tokens, target, draft, u, u_next = _inputs(7, 5, 3, 1001, dtype)
    want = _ref(tokens.numpy(), target.double().numpy(), draft.double().numpy(), u.numpy(), u_next.numpy())
    t = torch.zeros(4, 5, 1005, dtype=target.dtype, device="cuda")
    t[:, :, 3:1004] = target.transpose(0, 1).cuda()
    d = torch.zeros(5, 9, 1003, dtype=target.dtype, device="cuda")
    d[:, ::3, 1:1002] = draft.cuda()
    acc = torch.empty(5, dtype=torch.int32, device="cuda")
    out = torch.empty(5, 4, dtype=torch.int64, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    got = squat.verify_drafts(tokens.cuda(), t[:, :, 3:1004].transpose(0, 1), d[:, ::3, 1:1002], u.cuda(), u_next.cuda(), accepted=acc, out=out, ws=ws)
    assert got[0].data_ptr() == acc.data_ptr() and got[1].data_ptr() == out.data_ptr()
    assert np.array_equal(acc.cpu().numpy(), want[0]) and np.array_equal(out.cpu().numpy(), want[1])


def test_the_first_token_is_the_target_s():
    """Over many drafts from q the first token of the answer is distributed as p: every token's count within five deviations."""
    n, v = 20000, 8
    p = torch.tensor([0.3, 0.02, 0.18, 0.0, 0.1, 0.25, 0.05, 0.1])
    q = torch.tensor([0.1, 0.3, 0.1, 0.2, 0.1, 0.1, 0.05, 0.05])
    g = torch.Generator().manual_seed(8)
    tokens = torch.multinomial(q, n, replacement=True, generator=g).view(n, 1)
    _, out = squat.verify_drafts(tokens.cuda(), p.expand(n, 2, v).contiguous().cuda(), q.expand(n, 1, v).contiguous().cuda(),
                                 torch.rand(n, 1, generator=g).cuda(), torch.rand(n, generator=g).cuda())
    count = torch.bincount(out[:, 0].cpu(), minlength=v).double()
    assert ((count - n * p.double()).abs() <= 5 * (n * p.double() * (1 - p.double())).sqrt()).all()


def test_a_graph():
    tokens, target, draft, u, u_next = (t.cuda() for t in _inputs(9, 6, 4, 9001, "f32"))
    acc = torch.empty(6, dtype=torch.int32, device="cuda")
    out = torch.empty(6, 5, dtype=torch.int64, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    squat.verify_drafts(tokens, target, draft, u, u_next, accepted=acc, out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            squat.verify_drafts(tokens, target, draft, u, u_next, accepted=acc, out=out, ws=ws)
    torch.cuda.synchronize()
    for i in range(4):
        u.copy_(torch.rand(u.shape))
        u_next.copy_(torch.rand(u_next.shape))
        graph.replay()
        torch.cuda.synchronize()
        a, o = squat.verify_drafts(tokens, target, draft, u, u_next)
        assert torch.equal(a, acc) and torch.equal(o, out)
