"""Argument checks and plans of the operators in fewer bits through the C ABI (CPU only: every
call ends before any HIP call, no address is dereferenced)."""

import ctypes

import pytest

from paper_2607_04244_amd import qlin

A = 1 << 36                                     # stand-in addresses, 2^32 apart
STEP = 1 << 32
OK, INVALID, UNSUPPORTED, ALIGN = qlin.QLIN_OK, qlin.QLIN_ERR_INVALID, qlin.QLIN_ERR_UNSUPPORTED, qlin.QLIN_ERR_ALIGN
NAN, INF = float("nan"), float("inf")


def norm(**kw):
    f = dict(rows=10, width=256, y=A, ys=256, res=A + STEP, rs=256, post=A + 2 * STEP, gate=A + 3 * STEP, gs=256, sig=1, scale=1.0,
             pre=A + 4 * STEP, eps=1e-6, new=A + 5 * STEP, ns=256, out=A + 6 * STEP, os=256)
    f.update(kw)
    return qlin.qlin_block_norm(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(rows=1 << 22), UNSUPPORTED), (dict(width=0), INVALID), (dict(width=252), INVALID),
    (dict(width=65544, ys=65544), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID), (dict(eps=INF), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(res=None), INVALID), (dict(new=None), INVALID), (dict(y=None), INVALID),
    (dict(y=None, post=None, gate=None), INVALID), (dict(y=None, post=None, gate=None, new=None, pre=None, out=None), INVALID),
    (dict(pre=None), INVALID), (dict(out=None), INVALID), (dict(ys=248), INVALID), (dict(rs=260), ALIGN), (dict(gs=252), INVALID),
    (dict(gs=8), INVALID), (dict(ns=1 << 33), INVALID), (dict(y=A + 8), ALIGN), (dict(res=A + STEP + 2), ALIGN), (dict(gate=A + 8), ALIGN),
    (dict(gate=A + 8, gs=0), ALIGN), (dict(post=A + 4), ALIGN), (dict(pre=A + 4), ALIGN), (dict(out=A + 6 * STEP + 8), ALIGN),
    # overlaps: outputs on other rows of the inputs, on each other, the gate, the weights
    (dict(out=A + 512), INVALID), (dict(out=A, os=264), INVALID), (dict(new=A + STEP + 16), INVALID), (dict(out=A + 5 * STEP), INVALID),
    (dict(out=A + 5 * STEP + 512), INVALID), (dict(out=A + 3 * STEP), INVALID), (dict(new=A + 3 * STEP + 512), INVALID),
    (dict(out=A + 2 * STEP - 256), INVALID), (dict(new=A + 4 * STEP), INVALID), (dict(gate=A + 6 * STEP + 512, gs=0), INVALID),
])
def test_norm_refuses(kw, code):
    assert norm(**kw) == code and qlin.qlin_last_status() == code


def test_norm_no_rows():
    assert norm(rows=0) == OK and norm(rows=0, y=None, res=None, out=None) == OK
    assert norm(rows=0, width=7) == INVALID


def tokens(**kw):
    f = dict(rows=10, width=256, x=A, xs=512, gated=0, c=A + STEP, cs=256, s=A + 2 * STEP)
    f.update(kw)
    return qlin.qlin_quantize_tokens(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), INVALID), (dict(rows=1 << 22), UNSUPPORTED), (dict(width=0), INVALID), (dict(width=8), INVALID), (dict(width=264), INVALID),
    (dict(width=65552, xs=65552), UNSUPPORTED), (dict(x=None), INVALID), (dict(c=None), INVALID), (dict(s=None), INVALID), (dict(xs=248), INVALID),
    (dict(xs=504, gated=1), INVALID), (dict(xs=516), ALIGN), (dict(cs=240), INVALID), (dict(cs=264), ALIGN), (dict(cs=1 << 33), INVALID),
    (dict(x=A + 8), ALIGN), (dict(c=A + STEP + 8), ALIGN), (dict(s=A + 2), ALIGN), (dict(c=A + 16), INVALID), (dict(s=A + 512), INVALID),
    (dict(s=A + STEP + 2560 - 4), INVALID),
])
def test_tokens_refuse(kw, code):
    assert tokens(**kw) == code and qlin.qlin_last_status() == code


def test_tokens_no_rows():
    assert tokens(rows=0) == OK and tokens(rows=0, x=None, c=None, s=None) == OK


def linear(**kw):
    f = dict(M=100, N=500, K=1024, S=0, x=A, xs=1024, sx=A + STEP, w=A + 2 * STEP, ws=1024, sw=A + 3 * STEP, y=A + 4 * STEP, ys=504,
             wsp=A + 5 * STEP, wb=1 << 31)
    f.update(kw)
    return qlin.qlin_eight_bit_linear(*f.values(), None)


BAD_SIZES = [(dict(M=-1), INVALID), (dict(M=(1 << 22) + 1), UNSUPPORTED), (dict(N=0), INVALID), (dict(N=(1 << 22) + 1), UNSUPPORTED),
             (dict(K=0), INVALID), (dict(K=8), INVALID), (dict(K=1000), INVALID), (dict(K=131072), UNSUPPORTED), (dict(S=-1), INVALID),
             (dict(S=65), INVALID), (dict(M=1 << 22, N=1 << 22, S=1), UNSUPPORTED), (dict(M=1 << 18, N=1 << 18, S=2), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", BAD_SIZES + [
    (dict(S=1, x=None), INVALID), (dict(S=1, w=None), INVALID), (dict(S=1, sx=None), INVALID), (dict(S=1, sw=None), INVALID),
    (dict(S=1, y=None), INVALID), (dict(S=1, xs=1008), INVALID), (dict(S=1, ws=1032), ALIGN), (dict(S=1, ws=1 << 33), INVALID),
    (dict(S=1, x=A + 8), ALIGN), (dict(S=1, w=A + 4), ALIGN), (dict(S=1, sx=A + 2), ALIGN), (dict(S=1, sw=A + 1), ALIGN),
    (dict(S=1, y=A + 8), ALIGN), (dict(S=1, ys=500), ALIGN), (dict(S=1, ys=496), INVALID), (dict(S=1, wb=-1), INVALID),
    (dict(S=1, wsp=A + 8), ALIGN), (dict(S=2, wsp=None), INVALID), (dict(S=2, wb=2 * 100 * 500 * 4 - 1), INVALID), (dict(S=2, M=10, wb=2 * 10 * 500 * 4 - 1), INVALID),
    (dict(S=1, y=A + 1024), INVALID), (dict(S=1, y=A + 2 * STEP + 16), INVALID), (dict(S=1, y=A + STEP), INVALID), (dict(S=1, y=A + 3 * STEP), INVALID),
    (dict(S=2, wsp=A), INVALID), (dict(S=2, wsp=A + 4 * STEP + 1024), INVALID), (dict(S=2, wsp=A + 3 * STEP), INVALID),
])
def test_linear_refuses(kw, code):
    assert linear(**kw) == code and qlin.qlin_last_status() == code


def test_linear_no_rows_and_plans():
    assert linear(M=0, S=1, x=None, w=None, sx=None, sw=None, y=None) == OK
    for kw, code in BAD_SIZES:
        f = dict(M=100, N=500, K=1024, S=1)
        f.update(kw)
        with pytest.raises(qlin.QlinError) as e:
            qlin.qlin_eight_bit_plan(*f.values())
        assert e.value.code == code
    assert qlin.qlin_eight_bit_plan(100, 500, 1024, 1)[:2] == (1, 0)
    splits, need, text = qlin.qlin_eight_bit_plan(100, 500, 1024, 4)
    assert splits == 4 and need >= 4 * 100 * 500 * 4 and "splits=4" in text       # whole tiles
    # no more ranges than steps, and none without a step
    for M in (1, 20, 100):
        for K in (16, 272, 1040):
            for S in (1, 2, 3, 5, 64):
                splits, need, _ = qlin.qlin_eight_bit_plan(M, 64, K, S)
                assert 1 <= splits <= S and (need >= splits * M * 64 * 4 if splits > 1 else need == 0)
    assert qlin.lib().qlin_eight_bit_plan(1, 16, 16, 1, None, None, None, 0) == OK


def batch(**kw):
    f = dict(n_seq=3, rows=40, max_new=16, max_len=500, new_start=A, length=A + 64, cache_start=None)
    f.update(kw)
    return qlin.Batch(*(f[n] for n, _ in qlin.Batch._fields_))


def cache(**kw):
    f = dict(capacity=512, k=A + STEP, v=A + 2 * STEP, k_grid=A + 8 * STEP, v_grid=A + 9 * STEP, heads=8, slots=3 * 8 * 512, token_stride=1,
             head_stride=512, seq_slots=8 * 512)
    f.update(kw)
    return qlin.KV4Cache(*(f[n] for n, _ in qlin.KV4Cache._fields_))


def plain_cache(**kw):
    f = dict(k=A + 10 * STEP, v=A + 11 * STEP, heads=8, slots=3 * 8 * 512, token_stride=128, head_stride=512 * 128, seq_slots=8 * 512)
    f.update(kw)
    return qlin.KVCache(*(f[n] for n, _ in qlin.KVCache._fields_))


def append(b=None, c=None, **kw):
    f = dict(Hq=32, D=128, q=A + 3 * STEP, qs=4096, k=A + 4 * STEP, ks=1024, v=A + 5 * STEP, vs=1024, qn=A + 128, kn=A + 512,
             eps=1e-6, freq=A + 1024, rot=128, il=0, out=A + 6 * STEP, os=4096)
    f.update(kw)
    return qlin.qlin_norm_rope_append_four_bit(b if b is not None else batch(), c if c is not None else cache(), *f.values(), None)


def attend(b=None, c=None, **kw):
    f = dict(Hq=32, D=128, scale=0.0, splits=1, q=A + 3 * STEP, qs=4096, out=A + 6 * STEP, os=4096, ws=A + 7 * STEP, wb=1 << 31)
    f.update(kw)
    return qlin.qlin_causal_attention_four_bit(b if b is not None else batch(), c if c is not None else cache(), *f.values(), None)


def unpack(b=None, c=None, to=None, D=128, new_only=0):
    return qlin.qlin_unpack_four_bit(b if b is not None else batch(), c if c is not None else cache(), to if to is not None else plain_cache(), D, new_only, None)


BAD_BATCH = [(dict(n_seq=0), INVALID), (dict(n_seq=65537), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(rows=(1 << 22) + 1), UNSUPPORTED),
             (dict(max_new=41), INVALID), (dict(max_new=-1), INVALID), (dict(max_len=-1), INVALID), (dict(max_len=(1 << 28) + 1), UNSUPPORTED),
             (dict(new_start=None), INVALID), (dict(length=None), INVALID), (dict(new_start=A + 2), ALIGN), (dict(length=A + 1), ALIGN),
             (dict(cache_start=A + 4), ALIGN)]
BAD_CACHE = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k_grid=None), INVALID), (dict(v_grid=None), INVALID), (dict(k=A + STEP + 8), ALIGN),
             (dict(v=A + 2 * STEP + 4), ALIGN), (dict(k_grid=A + 8 * STEP + 2), ALIGN), (dict(v_grid=A + 9 * STEP + 1), ALIGN), (dict(heads=0), INVALID),
             (dict(heads=-8), INVALID), (dict(heads=5), INVALID), (dict(slots=0), INVALID), (dict(slots=(1 << 40) + 1), UNSUPPORTED),
             (dict(capacity=-1), INVALID), (dict(capacity=1 << 41), UNSUPPORTED), (dict(token_stride=0), INVALID), (dict(head_stride=0), INVALID),
             (dict(token_stride=(1 << 20) + 1), UNSUPPORTED), (dict(head_stride=1 << 37), UNSUPPORTED), (dict(seq_slots=-1), INVALID),
             (dict(seq_slots=1 << 41), UNSUPPORTED), (dict(slots=1 << 40, token_stride=1 << 20), UNSUPPORTED)]


@pytest.mark.parametrize("call", [append, attend, unpack])
def test_batches_and_caches_are_checked(call):
    for kw, code in BAD_BATCH:
        assert call(b=batch(**kw)) == code, kw
    for kw, code in BAD_CACHE:
        assert call(c=cache(**kw)) == code, kw
    f = dict(append=qlin.lib().qlin_norm_rope_append_four_bit, attend=qlin.lib().qlin_causal_attention_four_bit, unpack=qlin.lib().qlin_unpack_four_bit)[call.__name__]
    zeros = [None if t is ctypes.c_void_p or issubclass(t, ctypes._Pointer) else t(0) for t in f.argtypes]
    assert f(*zeros) == INVALID
    zeros[0] = batch()
    assert f(*zeros) == INVALID and "cache" in qlin.last_error()


@pytest.mark.parametrize("call", [append, attend])
def test_no_rows_is_a_no_op_after_the_checks(call):
    assert call(b=batch(rows=0, max_new=0)) == OK
    assert call(b=batch(rows=0, max_new=0, new_start=None, length=None)) == OK
    assert call(b=batch(rows=0, max_new=0), D=64) == UNSUPPORTED


COMMON = [(dict(D=64), UNSUPPORTED), (dict(Hq=0), INVALID), (dict(Hq=30), INVALID), (dict(Hq=8 * 65), UNSUPPORTED), (dict(q=None), INVALID),
          (dict(q=A + 3 * STEP + 2), ALIGN), (dict(qs=4088), INVALID), (dict(qs=4100), ALIGN), (dict(out=None), INVALID),
          (dict(out=A + 6 * STEP + 4), ALIGN), (dict(os=4095), INVALID), (dict(out=A + 3 * STEP + 64), INVALID),
          # on each of the cache's arrays: 3 x 8 x 512 rows of 64 and 4 bytes
          (dict(out=A + STEP + 4096), INVALID), (dict(out=A + 2 * STEP - 64), INVALID), (dict(out=A + 8 * STEP + 12288 * 4 - 16), INVALID),
          (dict(out=A + 9 * STEP), INVALID), (dict(out=A + 2 * STEP + 12288 * 64 - 16), INVALID), (dict(out=A - 64), INVALID)]


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(ks=1016), INVALID), (dict(vs=1025), ALIGN), (dict(qn=A + 4), ALIGN),
    (dict(freq=A + 4), ALIGN), (dict(freq=None), INVALID), (dict(rot=8), INVALID), (dict(rot=144), INVALID), (dict(eps=-1e-6), INVALID),
    (dict(eps=NAN), INVALID), (dict(out=A + 4 * STEP), INVALID), (dict(k=A + 8 * STEP), INVALID), (dict(v=A + 9 * STEP + 2048), INVALID),
    (dict(q=A + STEP), INVALID), (dict(kn=A + 8 * STEP), INVALID), (dict(freq=A + 2 * STEP), INVALID),
])
def test_append_refuses(kw, code):
    assert append(**kw) == code and qlin.qlin_last_status() == code


def test_append_refuses_a_cache_on_itself():
    for kw in [dict(v=A + STEP + 64), dict(k_grid=A + STEP), dict(v_grid=A + 8 * STEP + 16), dict(k_grid=A + 2 * STEP + 4)]:
        assert append(c=cache(**kw)) == INVALID, kw
    assert append(b=batch(length=A + STEP)) == INVALID and append(b=batch(new_start=A + 9 * STEP + 64)) == INVALID


@pytest.mark.parametrize("kw,code", COMMON + [
    (dict(splits=-1), INVALID), (dict(splits=257), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
    (dict(wb=-1), INVALID), (dict(ws=A + 7 * STEP + 8), ALIGN), (dict(splits=2, ws=None), INVALID), (dict(splits=2, wb=1000), INVALID),
    (dict(splits=2, ws=A + 3 * STEP), INVALID), (dict(splits=2, ws=A + 8 * STEP), INVALID), (dict(splits=2, ws=A + 6 * STEP), INVALID),
    (dict(splits=2, ws=A), INVALID),
])
def test_attention_refuses(kw, code):
    assert attend(**kw) == code and qlin.qlin_last_status() == code


def test_attention_plans():
    for kw, code in BAD_BATCH[:8]:
        with pytest.raises(qlin.QlinError) as e:
            qlin.qlin_causal_four_bit_plan(batch(**kw), 32, 8, 128, 1)
        assert e.value.code == code
    for args, code in [((30, 8, 128, 1), INVALID), ((32, 8, 96, 1), UNSUPPORTED), ((32, 8, 128, -1), INVALID), ((32, 8, 128, 300), INVALID),
                       ((65, 1, 128, 1), UNSUPPORTED)]:
        with pytest.raises(qlin.QlinError) as e:
            qlin.qlin_causal_four_bit_plan(batch(), *args)
        assert e.value.code == code
    splits, need, text = qlin.qlin_causal_four_bit_plan(batch(new_start=None, length=None), 32, 8, 128, 1)
    assert (splits, need) == (1, 0) and text.startswith("kernel=k_kv4")
    # a long chunk: the cache in 16 bits in the workspace
    b = batch(rows=3000, max_new=1000, max_len=5000)
    splits, need, text = qlin.qlin_causal_four_bit_plan(b, 32, 8, 128, 1)
    assert text.startswith("unpack=") and need >= 3 * 8 * 5000 * 512
    assert attend(b=b, wb=need - 1) == INVALID
    # too large for that, past 16 GiB: the codes themselves; too many tiles for one grid
    for n, kind in ((32, "unpack="), (33, "kernel=k_kv4_rows")):
        text = qlin.qlin_causal_four_bit_plan(batch(n_seq=n, rows=2000 * n, max_new=2000, max_len=1 << 17), 32, 8, 128, 1)[2]
        assert text.startswith(kind)
    text = qlin.qlin_causal_four_bit_plan(batch(n_seq=65536, rows=1 << 22, max_new=1 << 22, max_len=1 << 20), 32, 8, 128, 1)[2]
    assert text.startswith("kernel=k_kv4_rows")
    with pytest.raises(qlin.QlinError) as e:
        qlin.qlin_causal_four_bit_plan(batch(n_seq=65536, rows=1 << 22, max_new=1 << 22, max_len=1 << 20), 4096, 64, 128, 1)
    assert e.value.code == UNSUPPORTED


def test_unpack_refuses():
    assert unpack(D=64) == UNSUPPORTED
    assert unpack(c=cache(heads=4), to=plain_cache(heads=8)) == INVALID
    for kw, code in [(dict(k=None), INVALID), (dict(v=A + 11 * STEP + 8), ALIGN), (dict(token_stride=120), INVALID), (dict(slots=0), INVALID)]:
        assert unpack(to=plain_cache(**kw)) == code, kw
    # the caches on each other, the bf16 one on itself and on the batch
    for kw in [dict(k=A + STEP), dict(v=A + 2 * STEP + 1024), dict(k=A + 8 * STEP), dict(v=A + 9 * STEP), dict(v=A + 10 * STEP + 1024), dict(k=A)]:
        assert unpack(to=plain_cache(**kw)) == INVALID, kw
    assert unpack(b=batch(max_new=0), new_only=1) == OK
