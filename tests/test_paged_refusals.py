"""What the calls on paged stores and drafted tokens refuse, without a GPU: through the C ABI on made-up addresses (every call below has to
fail, or to find nothing to do, before anything is launched), and through the binding."""
import ctypes

import pytest
import torch

from paper_2503_24358_amd import squat

A, ODD = 0x100000, 0x100004
NULL, SHAPE, DTYPE, ALIGN, WS, VALUE = -1, -2, -3, -4, -5, -7


def _store(**kw):
    f = dict(key_codes=A, key_meta=A, value_codes=A, value_meta=A, n_pages=8, n_kv_heads=2, page_tokens=16, d=128, bits=4, group=32)
    f.update(kw)
    return squat.PagedStoreArrays(*[f[n] for n, _ in squat.PagedStoreArrays._fields_])


def _write(store=None, **kw):
    f = dict(k=A, v=A, dt=2, n=4, st=256, sh=128, slots=A, update=None, g=32, ws=None, wsb=0)
    f.update(kw)
    s = _store() if store is None else store
    return squat.lib().squat_paged_write(ctypes.byref(s), f["k"], f["v"], f["dt"], f["n"], f["st"], f["sh"], f["slots"], f["update"], f["g"],
                                         f["ws"], f["wsb"], None)


def _read(store=None, **kw):
    f = dict(slots=A, n=4, k=A, v=A, dt=2, st=256, sh=128)
    f.update(kw)
    s = _store() if store is None else store
    return squat.lib().squat_paged_read(ctypes.byref(s), f["slots"], f["n"], f["k"], f["v"], f["dt"], f["st"], f["sh"], None)


def _attend(store=None, **kw):
    f = dict(q=A, dt=2, n=4, qpk=4, qst=1024, qsh=128, start=A, kv=A, pages=A, ps=4, width=4, seqs=2, new=0, max_kv=0, scale=0.1, out=A,
             ost=1024, osh=128, lse=None, ws=A, wsb=1 << 40)
    f.update(kw)
    s = _store() if store is None else store
    return squat.lib().squat_paged_attention(ctypes.byref(s), f["q"], f["dt"], f["n"], f["qpk"], f["qst"], f["qsh"], f["start"], f["kv"], f["pages"],
                                             f["ps"], f["width"], f["seqs"], f["new"], f["max_kv"], f["scale"], f["out"], f["ost"], f["osh"],
                                             f["lse"], f["ws"], f["wsb"], None)


def _verify(**kw):
    f = dict(tokens=A, seqs=2, drafts=3, vocab=100, target=A, tss=400, tsp=100, draft=A, dss=300, dsp=100, dt=0, u=A, un=A, nd=None, acc=A,
             out=A, ws=A, wsb=1 << 40)
    f.update(kw)
    return squat.lib().squat_verify_drafts(f["tokens"], f["seqs"], f["drafts"], f["vocab"], f["target"], f["tss"], f["tsp"], f["draft"], f["dss"],
                                           f["dsp"], f["dt"], f["u"], f["un"], f["nd"], f["acc"], f["out"], f["ws"], f["wsb"], None)


BAD_STORES = [(dict(d=64), SHAPE), (dict(bits=3), SHAPE), (dict(bits=16), SHAPE), (dict(group=48), SHAPE), (dict(page_tokens=8), SHAPE),
              (dict(page_tokens=48), SHAPE), (dict(page_tokens=2048), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 31), SHAPE),
              (dict(n_kv_heads=0), SHAPE), (dict(n_kv_heads=70000), SHAPE), (dict(key_codes=None), NULL), (dict(value_meta=None), NULL),
              (dict(value_codes=ODD), ALIGN), (dict(key_meta=ODD), ALIGN)]


@pytest.mark.parametrize("change,status", BAD_STORES)
def test_stores(change, status):
    s = _store(**change)
    assert _write(s) == status and _read(s) == status and _attend(s) == status
    assert squat.lib().squat_paged_attention_workspace(ctypes.byref(s), 2, 4, 4, 4, 0, 0) == 0
    assert squat.lib().squat_paged_write_workspace(ctypes.byref(s), 4, 1) == 0


@pytest.mark.parametrize("change,status", [
    (dict(dt=9), DTYPE), (dict(n=-1), SHAPE), (dict(st=120), SHAPE), (dict(sh=64), SHAPE), (dict(st=260), ALIGN), (dict(sh=132), ALIGN),
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL), (dict(k=ODD), ALIGN), (dict(v=ODD), ALIGN), (dict(slots=ODD), ALIGN),
    (dict(update=A), WS), (dict(update=A, ws=A, wsb=10), WS), (dict(update=A, ws=A + 16, wsb=1 << 20), ALIGN), (dict(update=A, g=16, ws=A, wsb=1 << 20), SHAPE),
    (dict(update=ODD, ws=A, wsb=1 << 20), ALIGN), (dict(n=0, k=None), 0)])
def test_write(change, status):
    assert _write(**change) == status


def test_write_of_eight_bits_takes_no_update_matrix():
    assert _write(_store(bits=8), update=A, ws=A, wsb=1 << 20) == SHAPE


@pytest.mark.parametrize("change,status", [
    (dict(dt=-1), DTYPE), (dict(n=-1), SHAPE), (dict(st=100), SHAPE), (dict(sh=0), SHAPE), (dict(st=257), ALIGN), (dict(slots=None), NULL),
    (dict(k=ODD), ALIGN), (dict(v=ODD), ALIGN), (dict(slots=ODD), ALIGN), (dict(k=None, v=None), 0), (dict(n=0), 0)])
def test_read(change, status):
    assert _read(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(dt=0), DTYPE), (dict(dt=7), DTYPE), (dict(qpk=0), SHAPE), (dict(qpk=17), SHAPE), (dict(n=-1), SHAPE), (dict(seqs=-1), SHAPE),
    (dict(width=-1), SHAPE), (dict(width=1 << 30), SHAPE), (dict(ps=3), SHAPE), (dict(qst=64), SHAPE), (dict(osh=64), SHAPE), (dict(qsh=130), ALIGN),
    (dict(ost=1028), ALIGN), (dict(scale=float("nan")), VALUE), (dict(q=None), NULL), (dict(out=None), NULL), (dict(start=None), NULL),
    (dict(kv=None), NULL), (dict(pages=None), NULL), (dict(q=ODD), ALIGN), (dict(out=ODD), ALIGN), (dict(pages=A + 2), ALIGN), (dict(lse=A + 1), ALIGN),
    # (long page lists: sequences are met in parts, and their sums need the workspace)
    (dict(width=256, ps=256, ws=None), WS), (dict(width=256, ps=256, wsb=100), WS), (dict(width=256, ps=256, ws=A + 8), ALIGN),
    (dict(n=0, q=None), 0), (dict(seqs=0), 0), (dict(n=1 << 30), SHAPE)])
def test_attention(change, status):
    assert _attend(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(seqs=-1), SHAPE), (dict(seqs=70000), SHAPE), (dict(drafts=-1), SHAPE), (dict(drafts=65), SHAPE), (dict(vocab=0), SHAPE),
    (dict(vocab=(1 << 31) - 1), SHAPE), (dict(tss=-1), SHAPE), (dict(dsp=-1), SHAPE), (dict(dt=3), DTYPE), (dict(tokens=None), NULL),
    (dict(target=None), NULL), (dict(u=None), NULL), (dict(un=None), NULL), (dict(acc=None), NULL), (dict(out=None), NULL), (dict(tokens=ODD), ALIGN),
    (dict(target=A + 2), ALIGN), (dict(draft=A + 1), ALIGN), (dict(out=ODD), ALIGN), (dict(u=A + 2), ALIGN), (dict(ws=None), WS), (dict(wsb=8), WS),
    (dict(ws=A + 16), ALIGN), (dict(seqs=0, target=None), 0)])
def test_verify(change, status):
    assert _verify(**change) == status


def test_the_binding_refuses_what_lies_on_the_host():
    s = squat.PagedStore(2, 2, 16, 4, 32, device="cpu")
    k, slots = torch.zeros(3, 2, 128), torch.arange(3)
    i32 = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        s.write(k, k, slots)
    with pytest.raises(ValueError):
        s.read(slots)
    with pytest.raises(ValueError):
        s.attention(k.half(), torch.zeros(1, 2, dtype=torch.int32), i32[:1], i32, 1.0)
    with pytest.raises(ValueError):
        squat.verify_drafts(torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 4, 9), None, torch.zeros(2, 3), torch.zeros(2))
    with pytest.raises(AttributeError):
        squat.paged_write("no tensor", k, slots, *s.arrays)
    with pytest.raises(TypeError):
        squat.native().paged_read(slots)
