"""squat_paged_attention with many rows of bf16 queries (from 512 a sequence on, where there are tiles enough), which meet dequantized keys and values: against the definition in 64 bits.  Keys are rounded
to fp16 there, so a logit's bound has 2^-11 of its products beside what test_gpu_paged_attention counts."""
import numpy as np
import pytest
import torch

from paper_2503_24358_amd import squat
from tests import paged_ref as P
from tests.test_gpu_paged_attention import _case, _close, _i32

pytestmark = pytest.mark.gpu


def _run(seed, lens, new, heads, qpk, bits, group, page, scale=128 ** -0.5):
    store, table, starts, q = _case(seed, lens, new, heads, qpk, bits, group, page, "bf16")
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    out = squat.paged_attention(q.cuda(), *P.to_device(store), bits, group, _i32(table), _i32(lens), _i32(starts), scale, lse=lse,
                                max_new=max(new), max_kv=max(lens))
    _close(out, lse, P.attention(q.double().numpy(), store, bits, table, lens, starts, scale, rounded_keys=True), "bf16")


@pytest.mark.parametrize("bits", [2, 4, 8])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_chunk(bits, group):
    _run(bits + group, [700], [512], 16, 4, bits, group, 32)


@pytest.mark.parametrize("bits", [2, 4, 8])
def test_steps_that_end_anywhere(bits):
    _run(30 + bits, [200], [129], 16, 16, bits, 32, 16)
    _run(40 + bits, [256], [128], 16, 16, bits, 128, 64, scale=-0.2)
    _run(45 + bits, [385], [133], 16, 16, bits, 64, 16)


def test_ragged_chunks():
    """Whole prompts, a chunk behind a long beginning, a decoded token and a sequence without tokens in one call; lengths that end inside a step."""
    _run(50, [521, 1337, 90, 0, 31], [521, 77, 1, 0, 31], 10, 4, 4, 32, 64)
    _run(51, [515, 1, 65], [515, 1, 40], 12, 4, 2, 64, 16)


@pytest.mark.parametrize("bits, group", [(2, 128), (4, 32), (8, 64)])
def test_many_short_chunks(bits, group):
    """528 rows a sequence, and as many tiles as that takes; lengths from the chunk's own on."""
    _run(57, [33, 34, 47, 64, 65, 95, 128, 129, 160, 200, 256, 257], [33] * 12, 14, 16, bits, group, 16)
    _run(58, [90, 33, 400, 5, 0, 70, 33, 60, 80, 41, 129, 222, 301], [33, 33, 33, 5, 0, 33, 33, 33, 33, 33, 33, 33, 33], 14, 16, bits, group, 32)


def test_rows_that_see_nothing():
    """More new tokens than tokens."""
    store, table, starts, q = _case(52, [100], [150], 13, 16, 4, 32, 16, "bf16")
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    out = squat.paged_attention(q.cuda(), *P.to_device(store), 4, 32, _i32(table), _i32([100]), _i32(starts), 0.1, lse=lse)
    _close(out, lse, P.attention(q.double().numpy(), store, 4, table, [100], starts, 0.1, rounded_keys=True), "bf16")
    assert (out[:50] == 0).all() and torch.isneginf(lse[:50]).all()


@pytest.mark.parametrize("new, heads, qpk", [(150, 13, 16), (2, 3, 2), (9, 3, 4)])
def test_lists_of_no_pages(new, heads, qpk):
    """The lists may be nowhere where no sequence has room for a token (this form, one row a step, and several)."""
    store, _, starts, q = _case(56, [0], [new], heads, qpk, 4, 32, 16, "bf16")
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    for length in (0, 700):
        squat.paged_attention(q.cuda(), *P.to_device(store), 4, 32, torch.empty((1, 0), dtype=torch.int32, device="cuda"), _i32([length]), _i32(starts),
                              0.1, out=out, lse=lse)
        assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("where", [0, 5, 12])
def test_pages_that_do_not_exist(where):
    store, table, starts, q = _case(53, [400], [128], 16, 16, 4, 32, 32, "bf16")
    table[0, where] = -1
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    out = squat.paged_attention(q.cuda(), *P.to_device(store), 4, 32, _i32(table), _i32([400]), _i32(starts), 0.1, lse=lse)
    _close(out, lse, P.attention(q.double().numpy(), store, 4, table, [400], starts, 0.1, rounded_keys=True), "bf16")


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("which", ["key", "value"])
@pytest.mark.parametrize("length", [180, 600])
def test_what_is_masked_does_not_show(what, which, length):
    new = 140
    store, table, starts, q = _case(54, [length], [new], 16, 16, 4, 32, 16, "bf16")
    dev = P.to_device(store)
    args = (4, 32, _i32(table), _i32([length]), _i32(starts), 0.1)
    clean = squat.paged_attention(q.cuda(), *dev, *args)
    at = 61
    token = length - new + at
    meta = dev[1] if which == "key" else dev[3]
    meta[table[0, token // 16], 1, token % 16, 2, :] = what
    dev[1][table[0, length // 16], :, length % 16:] = what           # behind the end
    dev[3][table[0, length // 16], :, length % 16:] = what
    got = squat.paged_attention(q.cuda(), *dev, *args).cpu()
    seen = torch.zeros(new, 256, dtype=torch.bool)
    seen[at:, 16:32] = True
    assert torch.equal(got[~seen], clean.cpu()[~seen])
    hit = got[seen]
    assert not (hit if which == "key" else hit[:, 64:96]).isfinite().any()
    if which == "value":
        assert torch.equal(torch.cat([hit[:, :64], hit[:, 96:]], 1), torch.cat([clean.cpu()[seen][:, :64], clean.cpu()[seen][:, 96:]], 1))


def test_strides_and_a_graph():
    store, table, starts, q = _case(55, [300], [128], 16, 16, 4, 64, 32, "bf16")
    dev = P.to_device(store)
    want = P.attention(q.double().numpy(), store, 4, table, [300], starts, 0.1, rounded_keys=True)
    wide = torch.zeros(128, 260, 136, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:258, :128] = q.cuda()
    big = torch.full((128, 3, 256, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    tb, ln, st = _i32(table), _i32([300]), _i32(starts)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    run = lambda: squat.paged_attention(wide[:, 2:258, :128], *dev, 4, 64, tb, ln, st, 0.1, out=big[:, 1], ws=ws)        # noqa: E731
    run()
    _close(big[:, 1], None, want, "bf16")
    assert (big[:, 0] == 7).all() and (big[:, 2] == 7).all()
    first = big[:, 1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.synchronize()
    for _ in range(3):
        big[:, 1] = 0
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(big[:, 1], first)
