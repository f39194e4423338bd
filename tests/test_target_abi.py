"""Argument checks and plans of the target's operators through the C ABI (CPU only:
every call ends before any HIP call, no address is dereferenced)."""

import ctypes

import pytest

from paper_2607_04244_amd import qlin

A = 1 << 36                                     # stand-in addresses, 2^32 apart
STEP = 1 << 32
INVALID, UNSUPPORTED, ALIGN = qlin.QLIN_ERR_INVALID, qlin.QLIN_ERR_UNSUPPORTED, qlin.QLIN_ERR_ALIGN


def batch(**kw):
    f = dict(n_seq=3, rows=40, max_new=16, max_len=500, new_start=A, length=A + 64, cache_start=None)
    f.update(kw)
    return qlin.Batch(*(f[n] for n, _ in qlin.Batch._fields_))


def cache(**kw):
    f = dict(k=A + STEP, v=A + 2 * STEP, heads=8, slots=3 * 8 * 512, token_stride=128, head_stride=512 * 128, seq_slots=8 * 512)
    f.update(kw)
    return qlin.KVCache(*(f[n] for n, _ in qlin.KVCache._fields_))


def append(b=None, c=None, **kw):
    f = dict(Hq=32, D=128, q=A + 3 * STEP, qs=4096, k=A + 4 * STEP, ks=1024, v=A + 5 * STEP, vs=1024, qn=A + 128, kn=A + 512,
             eps=1e-6, freq=A + 1024, rot=128, il=0, out=A + 6 * STEP, os=4096)
    f.update(kw)
    return qlin.qlin_norm_rope_append(b if b is not None else batch(), c if c is not None else cache(), f["Hq"], f["D"],
                                      f["q"], f["qs"], f["k"], f["ks"], f["v"], f["vs"], f["qn"], f["kn"], f["eps"],
                                      f["freq"], f["rot"], f["il"], f["out"], f["os"], None)


def attend(b=None, c=None, **kw):
    f = dict(Hq=32, D=128, scale=0.0, splits=0, q=A + 3 * STEP, qs=4096, out=A + 6 * STEP, os=4096, ws=A + 7 * STEP, wb=1 << 31)
    f.update(kw)
    return qlin.qlin_causal_attention(b if b is not None else batch(), c if c is not None else cache(), f["Hq"], f["D"],
                                      f["scale"], f["splits"], f["q"], f["qs"], f["out"], f["os"], f["ws"], f["wb"], None)


BAD_BATCH = [(dict(n_seq=0), INVALID), (dict(n_seq=65537), UNSUPPORTED), (dict(rows=-1), INVALID),
             (dict(rows=(1 << 22) + 1), UNSUPPORTED), (dict(max_new=41), INVALID), (dict(max_new=-1), INVALID),
             (dict(max_len=-1), INVALID), (dict(max_len=(1 << 28) + 1), UNSUPPORTED)]
BAD_ARRAYS = [(dict(new_start=None), INVALID), (dict(length=None), INVALID), (dict(new_start=A + 2), ALIGN),
              (dict(length=A + 1), ALIGN), (dict(cache_start=A + 4), ALIGN)]
BAD_CACHE = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + STEP + 8), ALIGN), (dict(heads=0), INVALID),
             (dict(heads=-8), INVALID), (dict(heads=5), INVALID), (dict(slots=0), INVALID), (dict(slots=(1 << 40) + 1), UNSUPPORTED),
             (dict(token_stride=120), INVALID), (dict(token_stride=132), ALIGN), (dict(head_stride=64), INVALID),
             (dict(head_stride=129), ALIGN), (dict(seq_slots=-1), INVALID), (dict(seq_slots=1 << 41), UNSUPPORTED),
             (dict(slots=1 << 39, token_stride=1 << 39), UNSUPPORTED), (dict(head_stride=1 << 41), UNSUPPORTED)]


@pytest.mark.parametrize("call", [append, attend])
def test_batches_and_caches_are_checked(call):
    for kw, code in BAD_BATCH + BAD_ARRAYS:
        assert call(b=batch(**kw)) == code, kw
    for kw, code in BAD_CACHE:
        assert call(c=cache(**kw)) == code, kw
    f = qlin.lib().qlin_causal_attention if call is attend else qlin.lib().qlin_norm_rope_append
    n = len(f.argtypes)
    zeros = [None if t is ctypes.c_void_p or issubclass(t, ctypes._Pointer) else t(0) for t in f.argtypes]
    assert n > 2 and f(*zeros) == INVALID                                        # NULL batch
    zeros[0] = batch()
    assert f(*zeros) == INVALID and "cache" in qlin.last_error()                 # NULL cache


@pytest.mark.parametrize("call", [append, attend])
def test_no_rows_is_a_no_op_after_the_checks(call):
    assert call(b=batch(rows=0, max_new=0)) == qlin.QLIN_OK
    assert call(b=batch(rows=0, max_new=0, new_start=None, length=None)) == qlin.QLIN_OK
    assert call(b=batch(rows=0, max_new=0), D=64) == UNSUPPORTED


COMMON = [(dict(D=64), UNSUPPORTED), (dict(D=0), UNSUPPORTED), (dict(Hq=0), INVALID), (dict(Hq=30), INVALID),
          (dict(Hq=8 * 65), UNSUPPORTED), (dict(Hq=4104), UNSUPPORTED), (dict(q=None), INVALID), (dict(q=A + 3 * STEP + 2), ALIGN),
          (dict(qs=4088), INVALID), (dict(qs=4100), ALIGN), (dict(qs=1 << 33), INVALID), (dict(out=None), INVALID),
          (dict(out=A + 6 * STEP + 4), ALIGN), (dict(os=4095), INVALID), (dict(os=4097), ALIGN),
          (dict(out=A + 3 * STEP + 64), INVALID),                        # overlaps q
          (dict(out=A + STEP + 4096), INVALID), (dict(out=A + 2 * STEP - 64), INVALID)]   # overlaps k, v of the cache


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 4 * STEP + 8), ALIGN), (dict(ks=1016), INVALID),
    (dict(vs=1025), ALIGN), (dict(qn=A + 4), ALIGN), (dict(kn=A + 2), ALIGN), (dict(freq=A + 4), ALIGN), (dict(freq=None), INVALID),
    (dict(rot=8), INVALID), (dict(rot=144), INVALID), (dict(rot=-16), INVALID), (dict(eps=-1e-6), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(out=A + 4 * STEP), INVALID),
    (dict(out=A + 5 * STEP + 32), INVALID), (dict(k=A + STEP), INVALID), (dict(v=A + 2 * STEP + 2048), INVALID),
    (dict(q=A + 2 * STEP), INVALID), (dict(out=A + 3 * STEP, os=4104), INVALID),
    # rows of 6144: q, k, v side by side; q_out on them must be q itself or columns of no input
    (dict(qs=6144, ks=6144, vs=6144, os=6144, k=A + 3 * STEP + 8192, v=A + 3 * STEP + 10240, out=A + 3 * STEP + 2048), INVALID),
    (dict(qs=6144, ks=6144, vs=6144, os=6144, k=A + 3 * STEP + 8000, v=A + 3 * STEP + 10240, out=A + 3 * STEP), INVALID),
    (dict(qs=8192, ks=8192, vs=8192, os=8192, k=A + 3 * STEP + 8192, v=A + 3 * STEP + 10240, out=A + 3 * STEP + 10240), INVALID),
])
def test_append_refuses(kw, code):
    assert append(**kw) == code and qlin.qlin_last_status() == code


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(splits=-1), INVALID), (dict(splits=257), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(wb=-1), INVALID), (dict(ws=A + 7 * STEP + 8), ALIGN),
])
def test_attention_refuses(kw, code):
    assert attend(**kw) == code and qlin.qlin_last_status() == code


def test_attention_plan_is_checked():
    for kw, code in BAD_BATCH:
        with pytest.raises(qlin.QlinError) as e:
            qlin.qlin_causal_plan(batch(**kw), 32, 8, 128, 1)
        assert e.value.code == code
    for args, code in [((30, 8, 128, 1), INVALID), ((32, 8, 96, 1), UNSUPPORTED), ((32, 8, 128, -1), INVALID),
                       ((32, 8, 128, 300), INVALID), ((65, 1, 128, 1), UNSUPPORTED)]:
        with pytest.raises(qlin.QlinError) as e:
            qlin.qlin_causal_plan(batch(), *args)
        assert e.value.code == code
    splits, _, text = qlin.qlin_causal_plan(batch(new_start=None, length=None), 32, 8, 128, 1)
    assert splits == 1 and text.startswith("kernel=")
    assert qlin.lib().qlin_causal_plan(batch(), 32, 8, 128, 1, None, None, None, 0) == qlin.QLIN_OK


def verify(**kw):
    f = dict(n_seq=4, n=5, V=1000, t=A, ts=1000, d=A + STEP, ds=1000, x=A + 2 * STEP, c=A + 3 * STEP, temp=A + 4 * STEP,
             u=A + 5 * STEP, a=A + 6 * STEP, tok=A + 7 * STEP, ws=A + 8 * STEP, wb=1 << 31)
    f.update(kw)
    return qlin.qlin_verify_draft(f["n_seq"], f["n"], f["V"], f["t"], f["ts"], f["d"], f["ds"], f["x"], f["c"], f["temp"],
                                  f["u"], f["a"], f["tok"], f["ws"], f["wb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_seq=-1), INVALID), (dict(n_seq=65536), UNSUPPORTED), (dict(n=-1), INVALID), (dict(n=65), UNSUPPORTED),
    (dict(V=0), INVALID), (dict(V=(1 << 24) + 1), UNSUPPORTED), (dict(t=None), INVALID), (dict(u=None), INVALID),
    (dict(a=None), INVALID), (dict(tok=None), INVALID), (dict(x=None), INVALID), (dict(ts=999), INVALID),
    (dict(ds=999), INVALID), (dict(ts=1 << 33), INVALID), (dict(t=A + 2), ALIGN), (dict(d=A + STEP + 8), ALIGN),
    (dict(x=A + 2 * STEP + 2), ALIGN), (dict(temp=A + 4 * STEP + 1), ALIGN), (dict(tok=A + 7 * STEP + 2), ALIGN),
    (dict(ws=A + 8 * STEP + 4), ALIGN), (dict(wb=-1), INVALID), (dict(a=A + 64), INVALID), (dict(tok=A + 2 * STEP + 4), INVALID),
    (dict(tok=A + 6 * STEP + 8), INVALID), (dict(a=A + 3 * STEP), INVALID), (dict(a=A + 4 * STEP), INVALID),
    (dict(tok=A + 5 * STEP), INVALID), (dict(tok=A + STEP + 64), INVALID),
])
def test_verify_refuses(kw, code):
    assert verify(**kw) == code and qlin.qlin_last_status() == code


def test_verify_without_sequences_is_a_no_op():
    assert verify(n_seq=0, t=None, u=None, a=None, tok=None) == qlin.QLIN_OK


def test_verify_workspace_is_checked():
    need = qlin.qlin_verify_plan(4, 5, 1000)
    if need:
        assert verify(wb=need - 16) == INVALID and verify(ws=None, wb=0) == INVALID
        assert "workspace" in qlin.last_error()
        assert verify(tok=A + 8 * STEP) == INVALID                       # tokens overlaps the workspace
    for args in ((-1, 5, 10), (1, -1, 10), (1, 5, 0)):
        with pytest.raises(qlin.QlinError) as e:
            qlin.qlin_verify_plan(*args)
        assert e.value.code == INVALID


def test_attention_workspace_is_checked():
    """Forced key ranges need no device: the plan is arithmetic."""
    splits, need, text = qlin.qlin_causal_plan(batch(), 32, 8, 128, 3)
    assert (splits, need) == (3, 3 * 8 * 64 * 3 * 130 * 4) and "k_causal_mid<2>" in text and "combine=1" in text
    assert attend(splits=3, wb=need - 16) == INVALID and attend(splits=3, ws=None, wb=0) == INVALID
    assert "workspace" in qlin.last_error()
    assert attend(splits=3, out=A + 7 * STEP + 64) == INVALID
    assert "k_causal_few " in qlin.qlin_causal_plan(batch(max_new=1), 128, 8, 128, 1)[2]
    assert "k_causal_mid<1>" in qlin.qlin_causal_plan(batch(max_new=16), 16, 8, 128, 1)[2]
    assert "k_causal_prompt" in qlin.qlin_causal_plan(batch(max_new=17), 32, 8, 128, 1)[2]
    assert qlin.qlin_causal_plan(batch(max_new=0), 32, 8, 128, 1)[0] == 1
    with pytest.raises(qlin.QlinError) as e:
        qlin.qlin_causal_plan(batch(rows=1 << 22, max_new=1 << 22), 4096, 64, 128, 2)
    assert e.value.code == UNSUPPORTED


def test_a_workspace_on_an_input_is_refused():
    assert attend(splits=3, ws=A + 3 * STEP, wb=1 << 31) == INVALID and "workspace" in qlin.last_error()     # q
    assert attend(splits=3, ws=A + STEP + 256, wb=1 << 31) == INVALID and "workspace" in qlin.last_error()   # k of the cache
    assert attend(splits=3, ws=A + 2 * STEP, wb=1 << 31) == INVALID and "workspace" in qlin.last_error()     # v
    for i in (0, 1, 2, 3, 4, 5, 6, 7):                                   # target, draft, drafted, ..., accepted, tokens
        assert verify(ws=A + i * STEP) == INVALID and "workspace" in qlin.last_error()


def test_prompts_in_two_halves_are_planned():
    """Forced ranges of long walks over few items; short ones, and many items, in one half."""
    plan = lambda n, L, S: qlin.qlin_causal_plan(batch(rows=n, max_new=n, max_len=L), 32, 8, 128, S)[2]
    assert "k_causal_prompt<2> splits=1" in plan(500, 8000, 1) and "k_causal_prompt<2> splits=2" in plan(500, 8000, 2)
    assert "k_causal_prompt<1>" in plan(500, 500, 1) and "k_causal_prompt<1>" in plan(500, 2000, 4)
    assert "k_causal_prompt<1>" in plan(8192, 8192, 1)


def test_remembered_plans_are_the_plans():
    """More calls than a thread remembers, in two orders and in two threads."""
    import threading
    asks = [(n, rows, L, Hq, S) for n in (1, 3, 40) for rows in (40, 700, 4000) for L in (500, 9000) for Hq in (8, 32) for S in (1, 2, 9)]
    ask = lambda n, rows, L, Hq, S: qlin.qlin_causal_plan(batch(n_seq=n, rows=rows, max_new=rows // n, max_len=L), Hq, 8, 128, S)
    assert len(asks) > 64
    first = [ask(*a) for a in asks]
    assert len(set(first)) > 40
    assert [ask(*a) for a in asks] == first and [ask(*a) for a in asks[::-1]] == first[::-1]
    other = []
    t = threading.Thread(target=lambda: other.extend(ask(*a) for a in asks for _ in (0, 1)))
    t.start()
    t.join()
    assert other[::2] == first and other[1::2] == first
    assert [p[0] for p in first] == [a[4] for a in asks]
