"""Host side of the rollout step: refusals of the C entries (nothing is launched, so made-up device pointers do), and
pins of the oracle's operators."""
import ctypes as C

import numpy as np
import pytest

from oracle import rollout as orc
from paper_2609_25442_b200 import binding as wb

A = 1 << 20     # an aligned address that is never dereferenced


def desc(**kw):
    d = dict(dtype=wb.WB_BF16, n_kv_heads=2, head_dim=64, page_size=16, n_pages=8, page_stride=2 * 16 * 64, head_stride=16 * 64,
             k=A, v=2 * A, k_scale=None, v_scale=None)
    d.update(kw)
    return wb.wb_kv_desc(*[d[n] for n, _ in wb.wb_kv_desc._fields_])


def open_status(d):
    h = C.c_void_p()
    st = wb.load().wb_kv_open(C.byref(d) if d is not None else None, C.byref(h))
    if h:
        wb.load().wb_kv_free(h)
    return wb.STATUS_NAMES[st]


BAD_CACHES = [
    (dict(dtype=wb.WB_F32), "WB_ERR_DTYPE"), (dict(dtype=7), "WB_ERR_DTYPE"),
    (dict(head_dim=32), "WB_ERR_INVALID_ARG"), (dict(head_dim=96), "WB_ERR_INVALID_ARG"), (dict(head_dim=0), "WB_ERR_INVALID_ARG"),
    (dict(n_kv_heads=0), "WB_ERR_INVALID_ARG"), (dict(n_pages=0), "WB_ERR_INVALID_ARG"),
    (dict(page_size=0), "WB_ERR_INVALID_ARG"), (dict(page_size=24), "WB_ERR_INVALID_ARG"), (dict(page_size=1 << 17), "WB_ERR_INVALID_ARG"),
    (dict(n_pages=1 << 31), "WB_ERR_INVALID_ARG"), (dict(n_pages=(1 << 26) + 1, n_kv_heads=2), "WB_ERR_INVALID_ARG"),
    (dict(k=None), "WB_ERR_INVALID_ARG"), (dict(v=None), "WB_ERR_INVALID_ARG"), (dict(k=A + 8), "WB_ERR_INVALID_ARG"),
    (dict(page_stride=100), "WB_ERR_INVALID_ARG"), (dict(head_stride=16 * 64 - 16), "WB_ERR_INVALID_ARG"),
    (dict(page_stride=2 * 16 * 64 - 16), "WB_ERR_INVALID_ARG"), (dict(page_stride=1 << 39), "WB_ERR_INVALID_ARG"),
    (dict(k_scale=A), "WB_ERR_INVALID_ARG"), (dict(dtype=wb.WB_E4M3), "WB_ERR_INVALID_ARG"),
    (dict(dtype=wb.WB_E4M3, k_scale=A), "WB_ERR_INVALID_ARG"), (dict(dtype=wb.WB_E4M3, k_scale=A + 2, v_scale=A), "WB_ERR_INVALID_ARG"),
]


@pytest.mark.parametrize("kw,name", BAD_CACHES)
def test_open_refuses(kw, name):
    assert open_status(desc(**kw)) == name


def test_open_refuses_null():
    assert open_status(None) == "WB_ERR_INVALID_ARG"


def test_layouts_still_refuse_e4m3():
    t = np.zeros(1, np.dtype([("rank", "<u4"), ("dtype", "<u4"), ("numel", "<u8")]))
    t[0] = (0, wb.WB_E4M3, 8)
    with pytest.raises(wb.WbError) as e:
        wb.Layout(t, np.zeros(0, wb.SLICE_DTYPE))
    assert e.value.name == "WB_ERR_DTYPE"


@pytest.fixture(scope="module")
def kv():
    """A handle over memory that does not exist.  Opening needs the driver's tensor-map encoder, so without a driver
    there is no handle, and the refusals of the calls that take one are checked on the GPU's machine only."""
    h = C.c_void_p()
    if wb.load().wb_kv_open(C.byref(desc()), C.byref(h)) != wb.WB_OK:
        pytest.skip("no driver here")
    yield h
    wb.load().wb_kv_free(h)


def batch(**kw):
    d = dict(n_seqs=2, n_tokens=3, max_new=2, max_len=20, table_stride=2, reserved=0, page_table=A, new_start=A, kv_len=A)
    d.update(kw)
    return wb.wb_kv_batch(*[d[n] for n, _ in wb.wb_kv_batch._fields_])


def heads(**kw):
    d = dict(data=A, dtype=wb.WB_BF16, reserved=0, token_stride=512, head_stride=64)
    d.update(kw)
    return wb.wb_heads(*[d[n] for n, _ in wb.wb_heads._fields_])


BAD_BATCHES = [dict(reserved=1), dict(n_seqs=4097), dict(max_new=4), dict(max_len=1 << 31), dict(new_start=None), dict(kv_len=None),
               dict(page_table=None), dict(table_stride=1 << 28)]
BAD_HEADS = [(dict(reserved=1), "WB_ERR_INVALID_ARG"), (dict(data=None), "WB_ERR_INVALID_ARG"), (dict(data=A + 2), "WB_ERR_INVALID_ARG"),
             (dict(token_stride=510), "WB_ERR_INVALID_ARG"), (dict(head_stride=65), "WB_ERR_INVALID_ARG"), (dict(dtype=wb.WB_E4M3), "WB_ERR_DTYPE")]


@pytest.mark.parametrize("kw", BAD_BATCHES)
def test_calls_refuse_batches(kv, kw):
    lib, b, h = wb.load(), batch(**kw), heads()
    for st in (lib.wb_kv_write(kv, C.byref(b), C.byref(h), C.byref(h), None), lib.wb_kv_read(kv, C.byref(b), C.byref(h), C.byref(h), None),
               lib.wb_kv_attend(kv, C.byref(b), C.byref(h), 4, C.byref(h), None, 1.0, 0, A, 1 << 30, None)):
        assert wb.STATUS_NAMES[st] == "WB_ERR_INVALID_ARG"


@pytest.mark.parametrize("kw,name", BAD_HEADS)
def test_calls_refuse_tensors(kv, kw, name):
    lib, b, good, bad = wb.load(), batch(), heads(), heads(**kw)
    for f in (lib.wb_kv_write, lib.wb_kv_read):
        assert wb.STATUS_NAMES[f(kv, C.byref(b), C.byref(good), C.byref(bad), None)] == name
        assert wb.STATUS_NAMES[f(kv, C.byref(b), C.byref(bad), C.byref(good), None)] == name
    for q, o in ((good, bad), (bad, good)):
        assert wb.STATUS_NAMES[lib.wb_kv_attend(kv, C.byref(b), C.byref(q), 4, C.byref(o), None, 1.0, 0, A, 1 << 30, None)] == name


def test_rows_of_two_types_are_refused(kv):
    b, h, f = batch(), heads(), heads(dtype=wb.WB_F32)
    assert wb.STATUS_NAMES[wb.load().wb_kv_write(kv, C.byref(b), C.byref(h), C.byref(f), None)] == "WB_ERR_DTYPE"
    assert wb.STATUS_NAMES[wb.load().wb_kv_attend(kv, C.byref(b), C.byref(f), 4, C.byref(h), None, 1.0, 0, A, 1 << 30, None)] == "WB_ERR_DTYPE"


@pytest.mark.parametrize("kw", [dict(n_heads=0), dict(n_heads=3), dict(n_heads=130), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                dict(scale=float("inf")), dict(window=1 << 31), dict(ws=None), dict(ws=A + 16), dict(ws_bytes=8)])
def test_attend_refuses(kv, kw):
    d = dict(n_heads=4, scale=1.0, window=0, ws=A, ws_bytes=1 << 30)
    d.update(kw)
    b, h = batch(), heads()
    st = wb.load().wb_kv_attend(kv, C.byref(b), C.byref(h), d["n_heads"], C.byref(h), None, d["scale"], d["window"], d["ws"], d["ws_bytes"], None)
    assert wb.STATUS_NAMES[st] == "WB_ERR_INVALID_ARG"


def verify_args(**kw):
    d = dict(n_seqs=1, vocab=10, max_drafts=2, dtype=wb.WB_F32, n_drafts=2, reserved=0, target=A, draft=A, target_stride=10, draft_stride=10,
             race_stride=10, draft_tokens=A, draft_start=A, uniform=A, race=A, accepted=A, tokens=A)
    d.update(kw)
    return wb.wb_verify_args(*[d[n] for n, _ in wb.wb_verify_args._fields_])


@pytest.mark.parametrize("kw,name", [
    (dict(dtype=wb.WB_E4M3), "WB_ERR_DTYPE"), (dict(vocab=0), "WB_ERR_INVALID_ARG"), (dict(target_stride=9), "WB_ERR_INVALID_ARG"),
    (dict(draft_stride=9), "WB_ERR_INVALID_ARG"), (dict(race_stride=9), "WB_ERR_INVALID_ARG"), (dict(target=None), "WB_ERR_INVALID_ARG"),
    (dict(draft_start=None), "WB_ERR_INVALID_ARG"), (dict(race=None), "WB_ERR_INVALID_ARG"), (dict(accepted=None), "WB_ERR_INVALID_ARG"),
    (dict(tokens=None), "WB_ERR_INVALID_ARG"), (dict(draft_tokens=None), "WB_ERR_INVALID_ARG"), (dict(uniform=None), "WB_ERR_INVALID_ARG"),
    (dict(target=A + 2), "WB_ERR_INVALID_ARG"), (dict(uniform=A + 1), "WB_ERR_INVALID_ARG"), (dict(reserved=3), "WB_ERR_INVALID_ARG"),
    (dict(max_drafts=1 << 21), "WB_ERR_INVALID_ARG"), (dict(n_drafts=1 << 31), "WB_ERR_INVALID_ARG")])
def test_verify_refuses(kw, name):
    with pytest.raises(wb.WbError) as e:
        wb.wb_verify_drafts(verify_args(**kw))
    assert e.value.name == name


@pytest.mark.parametrize("ws", [None, A + 8])
def test_attend_check_refuses(ws):
    assert wb.STATUS_NAMES[wb.load().wb_kv_attend_check(ws, None)] == "WB_ERR_INVALID_ARG"


def test_workspace_of_nothing():
    assert wb.load().wb_kv_attend_workspace_bytes(None, 4, 1) == 0


def test_verify_refuses_null():
    assert wb.STATUS_NAMES[wb.load().wb_verify_drafts(None, None)] == "WB_ERR_INVALID_ARG"


# ---- the oracle's own pins ------------------------------------------------------------------------
def test_oracle_attention_of_one_key_is_its_value():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(1, 2, 8)), rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8))
    out, lse, _ = orc.attend(q, k, v, 1, 0.5)
    assert np.allclose(out, np.broadcast_to(v[0], (1, 2, 8)), rtol=1e-15) and np.allclose(lse, 0.5 * (q @ k[0, 0]), rtol=1e-14)


def test_oracle_attention_masks():
    """A window equals a cut of the keys, later keys do not matter, and rows before the sequence are empty."""
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(3, 2, 8)), rng.normal(size=(1, 9, 8)), rng.normal(size=(1, 9, 8))
    out, lse, _ = orc.attend(q, k, v, 3, 0.3, window=4)
    one, l1, _ = orc.attend(q[1:2], k[:, 4:8], v[:, 4:8], 1, 0.3)
    assert np.allclose(out[1], one[0]) and np.allclose(lse[1], l1[0])
    short, ls, _ = orc.attend(q, k[:, :2], v[:, :2], 3, 0.3)
    assert (short[0] == 0).all() and (ls[0] == -np.inf).all() and np.isfinite(ls[1:]).all()


def test_oracle_verify_keeps_the_target_distribution():
    """Over many draws the first emitted token follows the target, whatever the drafter proposes."""
    rng = np.random.default_rng(2)
    p = np.array([[0.5, 0.3, 0.15, 0.05], [0.25] * 4], np.float32)
    q = np.array([[0.1, 0.2, 0.3, 0.4]], np.float32)
    counts = np.zeros(4)
    n = 20000
    for _ in range(n):
        x = rng.choice(4, p=q[0].astype(np.float64) / q[0].astype(np.float64).sum())
        _, out = orc.verify(p, q, [x], rng.random(1).astype(np.float32), rng.exponential(size=4).astype(np.float32), 1)
        counts[out[0]] += 1
    # five standard deviations of a multinomial count
    assert (np.abs(counts / n - p[0]) < 5 * np.sqrt(p[0] * (1 - p[0]) / n)).all()


def test_oracle_rows_quantise_as_tensors_do():
    x = np.array([0.0, 1.0, -448.0, 3.3, 1e-3], np.float32)
    codes, s = orc.quantize_row(x)
    assert s == np.float32(1.0) and orc.dequantize_row(codes, s)[2] == -448.0
    codes, s = orc.quantize_row(np.zeros(4, np.float32))
    assert s == 1.0 and not codes.any()
    codes, s = orc.quantize_row(np.array([1e-40, 0, 0, -1e-40], np.float32))
    assert s > 0 and codes[1] == 0 and codes[0] != 0
