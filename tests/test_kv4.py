"""GPU tests of the 4-bit key/value cache: its append, its unpacking and the causal attention
over it (include/qlin_lowbit.h), against the float64 oracles, through the Python entry points.

Tolerances, derived (a rounding is off by at most half a step: bf16 2^-8 of the value, f16
2^-12, fp32 2^-24):
* append: queries as for the bf16 cache.  Keys run in 64 bits and are rounded as the oracle's,
  values are given, and divisions are correctly rounded: words and grids equal, bit for bit.
* unpacking: one fused product, rounded to fp32 and bf16: equal.
* attention, with B = sum_j p_j (15 s_j + |o_j|), the size of what is summed: the scores'
  error is e = scale (c 2^-24 (15 s + |o|) sum|q|), c = 140 for 128 products, their scaling
  and the exponent's rounding, and 2^-20 for the exponential; a weight over their sum moves by
  a factor of at most exp(2 (e + 2^-20)) either way, the result by that less 1 times B.  Each weight times step is rounded to f16,
  2^-12 of 15 p s; below f16's normal range by 2^-25 of the unit 2^E <= s_max / 16, or for odd
  keys, whose operands are over 16, by 2^-21 of it: n 15 s_max 2^-25 for n keys.  fp32 sums over n keys: 2 n 2^-24 B.  The output's rounding 2^-8.
* in the forms that unpack, keys and values are f16: 2^-12 of each, so e has scale 2^-12
  sum|q||k| more, and the result 2^-11 sum_j p_j |v_j| for values and weights.  A row's values
  below f16's normal range are off by 2^-25 where its largest is at least 2^2: 2^-24 of B.
"""

import numpy as np
import pytest
import torch

from oracle import lowbit_ref as low
from oracle import target_ref as ref
from paper_2607_04244_amd import qlin

pytestmark = pytest.mark.gpu
HEAD = 128


def rand(seed, shape, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (sigma * torch.randn(shape, generator=g)).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts(new):
    return [0, *np.cumsum(new).tolist()]


def words_of(codes):
    return torch.from_numpy(low.pack_codes(codes).view(np.int32))


def bits(t):
    return t.cpu().view(torch.int16) if t.dtype == torch.bfloat16 else t.cpu()


class Cache:
    """A 4-bit cache of random rows in one of several layouts: `host` its four tensors (words and
    grids of keys, then of values), `dev` the same on the device."""

    def __init__(self, layout, length, Hkv, seed, capacity=None, spread=1.0):
        n, cap = len(length), capacity or max(max(length), 1) + 3
        self.layout, self.length, self.start = layout, length, None
        if layout == "packed":                 # [tokens, heads], sequences in mixed order, gaps between, a head more in memory
            at, self.at = 2, [0] * n
            for b in sorted(range(n), key=lambda b: (b * 5 + 2) % 7):
                self.at[b] = at
                at += length[b] + b % 3
            shape = (at + 1, Hkv + 1)
            self.start = torch.tensor(self.at, dtype=torch.int64, device="cuda")
        else:
            shape = (n, Hkv, cap) if layout == "heads" else (n, cap, Hkv)
        g = np.random.default_rng(seed)
        parts = []
        for _ in range(2):
            parts.append(torch.from_numpy(g.integers(-2 ** 31, 2 ** 31, (*shape, 16)).astype(np.int32)))
            step = 0.3 * np.exp(spread * g.standard_normal(shape))
            offset = -7.5 * step + 0.3 * g.standard_normal(shape)
            parts.append(torch.from_numpy(np.stack([step, offset], -1)).to(torch.bfloat16))
        self.host, self.dev = parts, [p.cuda() for p in parts]
        view = {"heads": lambda t: t, "tokens": lambda t: t.transpose(1, 2), "packed": lambda t: t[:, :Hkv]}[layout]
        self.host, self.dev = [view(t) for t in self.host], [view(t) for t in self.dev]

    def rows(self, part, b, source=None):
        """[L, heads, ...] of a sequence."""
        t, L = (source or self.host)[part], self.length[b]
        return t[self.at[b]:self.at[b] + L] if self.layout == "packed" else t[b, :, :L].transpose(0, 1)

    def values(self, which, b):
        """(values, steps, offsets) [L, heads, 128] and [L, heads], float64."""
        w, g = self.rows(2 * which, b).contiguous(), f64(self.rows(2 * which + 1, b))
        return low.row_values(w.numpy().view(np.uint32), g[..., 0], g[..., 1]), g[..., 0], g[..., 1]

    def kwargs(self):
        return dict(length=i32(self.length), cache_start=self.start)


LAYOUTS = ("heads", "tokens", "packed")


# ---------------------------------------------------------------- append


def check_append(new, length, layout="heads", Hq=4, Hkv=2, norm=True, rot=128, interleaved=False, pad=0, eps=1e-6, fused=False,
                 in_place=False, theta=1e4, seed=0, max_new=None):
    M = sum(new) + pad
    c = Cache(layout, length, Hkv, seed + 10)
    if fused:
        qkv = rand(seed, (M, (Hq + 2 * Hkv) * HEAD + 16), 1.5)
        cut = [0, Hq * HEAD, (Hq + Hkv) * HEAD, (Hq + 2 * Hkv) * HEAD]
        host = [qkv[:, cut[i]:cut[i + 1]] for i in range(3)]
        dev = qkv.cuda()
        devs = [dev[:, cut[i]:cut[i + 1]] for i in range(3)]
    else:
        host = [rand(seed + i, (M, h * HEAD), 1.5) for i, h in enumerate((Hq, Hkv, Hkv))]
        devs = [t.cuda() for t in host]
    wq, wk = (1 + rand(seed + 5 + i, (HEAD,), 0.2) if norm else None for i in (0, 1))
    freq = theta ** (-torch.arange(rot // 2, dtype=torch.float64) / max(rot // 2, 1))
    out = devs[0].view(M, Hq, HEAD) if in_place else torch.full((M, Hq, HEAD), 7.0, dtype=torch.bfloat16, device="cuda")
    got = qlin.norm_rope_append_kv4(*devs, c.dev, i32(starts(new)), max_new=max_new, q_norm=None if wq is None else wq.cuda(),
                                    k_norm=None if wk is None else wk.cuda(), eps=eps, inv_freq=freq.cuda() if rot else None,
                                    interleaved=interleaved, out=out, **c.kwargs())
    torch.cuda.synchronize()
    assert got is out
    freq = freq.numpy() if rot else np.zeros(0)
    want = [t.clone() for t in c.host]
    want_q = f64(host[0]).reshape(M, Hq, HEAD) if in_place else np.full((M, Hq, HEAD), 7.0)
    tol_q = np.zeros(want_q.shape)
    eps = float(np.float32(eps))
    for m, (b, p) in enumerate(ref.positions(new, length)):
        if max_new is not None and m - starts(new)[b] >= max_new:
            continue
        n = ref.norm(f64(host[0][m]).reshape(Hq, HEAD), None if wq is None else f64(wq), eps)
        want_q[m] = ref.rotate(n, p, freq, interleaved)
        tol_q[m] = 2.0 ** -8 * np.abs(want_q[m]) + 2.0 ** -19 * np.abs(n).max(axis=1, keepdims=True) + 1e-38
        if p < 0:
            continue
        at = (c.at[b] + p,) if layout == "packed" else (b, slice(None), p)
        k = ref.rotate(ref.norm(f64(host[1][m]).reshape(Hkv, HEAD), None if wk is None else f64(wk), eps), p, freq, interleaved)
        for part, x in ((0, low.to_bf16(k)), (2, f64(host[2][m]).reshape(Hkv, HEAD))):
            codes, step, offset = low.lay_on_grid(x)
            want[part][at] = words_of(codes)
            want[part + 1][at] = torch.from_numpy(np.stack([step, offset], -1)).to(torch.bfloat16)
    assert np.all(np.abs(f64(out) - want_q) <= tol_q)
    for have, w in zip(c.dev, want):
        assert torch.equal(bits(have.contiguous()), bits(w.contiguous()))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("new,length", [([1], [1]), ([1], [300]), ([16, 3, 0, 1], [16, 77, 9, 1]), ([5], [3]), ([0, 0, 2], [4, 0, 2]),
                                        ([40, 1, 30], [40, 333, 31])])
def test_append_batches(layout, new, length):
    check_append(new, length, layout)


@pytest.mark.parametrize("kw", [dict(norm=False), dict(rot=0), dict(rot=64), dict(rot=16), dict(rot=96), dict(interleaved=True),
                                dict(rot=48, interleaved=True), dict(fused=True), dict(fused=True, in_place=True, Hq=6, Hkv=1),
                                dict(in_place=True), dict(pad=9), dict(Hq=1, Hkv=1), dict(Hq=32, Hkv=8), dict(Hq=70, Hkv=7),
                                dict(Hq=5, Hkv=5, pad=3), dict(eps=0.0), dict(eps=2.0), dict(norm=False, rot=0)])
def test_append_forms(kw):
    check_append([7, 1, 12], [20, 1, 55], seed=3, **kw)


@pytest.mark.parametrize("rows,kw", [(639, dict(fused=True)), (640, dict(fused=True, in_place=True)), (643, dict(pad=6, interleaved=True, rot=48)),
                                     (645, dict(rot=0, max_new=300))])
def test_append_around_the_change_of_form(rows, kw):
    check_append([rows - 333, 1, 0, 2, 330], [rows, 1, 0, 1, 331], "packed", Hq=3, Hkv=1, seed=rows, **kw)


def test_append_more_new_tokens_than_declared_are_left_out():
    check_append([9, 2], [20, 30], max_new=4, seed=5)


def test_append_rows_at_the_ends():
    """Rows of one value, of zeros, of the grid itself, with ties, of far values, of subnormal
    steps, with infinities and NaN, and whose range is past fp32."""
    v = torch.zeros((14, HEAD))
    v[0] = 5.0
    v[2] = torch.arange(HEAD) % 16
    v[3, 0], v[3, 1:40] = 15.0, torch.arange(39) % 15 + 0.5
    v[4] = 1000.0 + torch.arange(HEAD) % 3 * 4
    v[5] = torch.arange(HEAD) * 2.0 ** -133
    v[6] = torch.arange(HEAD) * 2.0 ** -126
    v[7, 9], v[8, 10], v[9, 11] = float("inf"), float("nan"), float("-inf")
    v[10, 0], v[10, 1] = 3e38, -3e38
    v[11, 0], v[11, 1] = 3e38, -1.0
    v[12] = -torch.arange(HEAD) - 0.0
    v[13, 0] = -0.0
    v = v.to(torch.bfloat16)
    c = Cache("heads", [14], 1, 0)
    k = rand(1, (14, HEAD))
    qlin.norm_rope_append_kv4(k.cuda(), v.cuda(), v.cuda(), c.dev, i32([0, 14]), **c.kwargs())
    torch.cuda.synchronize()
    codes, step, offset = low.lay_on_grid(f64(v))
    for part in (0, 2):
        grid = f64(c.dev[part + 1][0, 0, :14])
        assert torch.equal(c.dev[part][0, 0, :14].cpu(), words_of(codes))
        assert np.array_equal(grid[:, 0], step, equal_nan=True) and np.array_equal(grid[:, 1], offset, equal_nan=True)


def test_append_outside_the_room_writes_nothing():
    """Lengths past the capacity, slots before and behind the cache: q_out only."""
    c = Cache("heads", [8, 8, 8], 2, 1, capacity=8)
    x = [rand(i, (3, h * HEAD)).cuda() for i, h in enumerate((2, 2, 2))]
    qlin.norm_rope_append_kv4(*x, c.dev, i32([0, 1, 2, 3]), i32([9, 8, 1 << 30]))
    torch.cuda.synchronize()
    for part, (have, was) in enumerate(zip(c.dev, c.host)):
        have = have.cpu()
        assert torch.equal(bits(have[0]), bits(was[0])) and torch.equal(bits(have[2]), bits(was[2]))
        assert torch.equal(bits(have[1, :, :7]), bits(was[1, :, :7])) and (part % 2 or not torch.equal(have[1, :, 7], was[1, :, 7]))
    before = [t.clone() for t in c.dev]
    for start in ([-1, 48, 47], [1 << 40, -(1 << 40), 1 << 62]):
        qlin.norm_rope_append_kv4(*x, c.dev, i32([0, 1, 2, 3]), i32([2, 2, 2]), cache_start=torch.tensor(start, dtype=torch.int64, device="cuda"))
        torch.cuda.synchronize()
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(before, c.dev))


# ---------------------------------------------------------------- unpacking


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("new_only", [False, True])
@pytest.mark.parametrize("new,length", [([1], [1]), ([3, 0, 70, 5], [200, 9, 70, 3]), ([1, 1], [65, 64])])
def test_unpack(layout, new_only, new, length):
    Hkv = 3
    c = Cache(layout, length, Hkv, sum(length))
    shape = (*c.host[0].shape[:-1], HEAD)
    to = [torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    if layout == "tokens":                     # the same order of slots
        to = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in to]
    got = qlin.unpack_kv4(c.dev, *to, i32(starts(new)), new_only=new_only, **c.kwargs())
    torch.cuda.synchronize()
    assert got[0] is to[0] and got[1] is to[1]
    for which in (0, 1):
        want = torch.full(shape, 7.0, dtype=torch.float64)
        for b, (n, L) in enumerate(zip(new, length)):
            first = max(L - n, 0) if new_only else 0
            v = torch.from_numpy(low.to_bf16(c.values(which, b)[0]))
            if layout == "packed":
                want[c.at[b] + first:c.at[b] + L] = v[first:]
            else:
                want[b, :, first:L] = v[first:].transpose(0, 1)
        assert torch.equal(to[which].cpu().double(), want)


def test_unpack_bounds():
    """A longer sequence than max_len, one past its room and one outside write nothing."""
    c = Cache("heads", [8, 8, 8, 8], 2, 1, capacity=8)
    to = [torch.zeros((4, 2, 8, HEAD), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    qlin.unpack_kv4(c.dev, *to, i32([0, 1, 2, 3, 4]), i32([9, 6, 5, -3]), max_len=5)
    torch.cuda.synchronize()
    for t in to:
        assert not t[[0, 1, 3]].any() and t[2, :, :5].any() and not t[2, :, 5:].any()


# ---------------------------------------------------------------- attention


def plan_text(new, length, Hq, Hkv, splits=0, max_new=None, max_len=None):
    b = qlin.Batch(len(new), max(sum(new), 1), max(new) if max_new is None else max_new, max(length) if max_len is None else max_len, None, None, None)
    return qlin.qlin_causal_four_bit_plan(b, Hq, Hkv, HEAD, splits)[2]


def bound(qb, c, b, Hq, Hkv, scale, unpacked):
    """(float64 result, tolerance) of a sequence's new tokens."""
    (k, ks, ko), (v, vs, vo) = c.values(0, b), c.values(1, b)
    want, A = ref.causal_attention(qb, k, v, scale)
    n, G, L = len(qb), Hq // Hkv, len(k)
    tol = np.zeros(want.shape)
    for i in range(n):
        seen = L - n + i + 1
        if seen <= 0:
            continue
        for h in range(Hq):
            g = h // G
            s = k[:seen, g] @ qb[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            size = 15 * vs[:seen, g] + np.abs(vo[:seen, g])
            B = float(p @ size)
            q1 = np.abs(qb[i, h])
            e = 140 * 2.0 ** -24 * scale * float((15 * ks[:seen, g] + np.abs(ko[:seen, g])).max() * q1.sum())
            extra = np.zeros(HEAD)
            if unpacked:
                e += scale * 2.0 ** -12 * float((np.abs(k[:seen, g]) @ q1).max())
                extra = 2.0 ** -11 * A[i, h] + 2.0 ** -24 * B
            x = e + 2.0 ** -20
            tol[i, h] = np.expm1(2 * x) * B + 2.0 ** -12 * 15 * float(p @ vs[:seen, g]) + seen * 15 * vs[:seen, g].max() * 2.0 ** -25 \
                + 2 * seen * 2.0 ** -24 * B + 2.0 ** -8 * np.abs(want[i, h]) + extra + 1e-38
    return want, tol


def check_attention(new, length, layout="heads", Hq=4, Hkv=2, splits=0, seed=0, sigma=1.0, scale=0.0, pad=0, fused=False, max_new=None,
                    max_len=None, cache=None, q=None, spread=1.0):
    M = sum(new) + pad
    c = cache or Cache(layout, length, Hkv, seed + 10, spread=spread)
    if q is None:
        q = rand(seed, (M, Hq + (3 if fused else 0), HEAD), sigma)[:, :Hq]
    dev = q.cuda() if not fused else torch.cat([q, torch.zeros(M, 3, HEAD, dtype=torch.bfloat16)], 1).cuda()[:, :Hq]
    out = torch.full((M, Hq, HEAD), 7.0, dtype=torch.bfloat16, device="cuda")
    bound_new = max(new) if max_new is None else max_new
    got = qlin.causal_attention_kv4(dev, c.dev, i32(starts(new)), max_new=bound_new, max_len=max_len, scale=scale, splits=splits, out=out, **c.kwargs())
    torch.cuda.synchronize()
    assert got is out
    unpacked = plan_text(new, length, Hq, Hkv, splits, bound_new, max_len).startswith("unpack")
    have, m = f64(out), 0
    for b, n in enumerate(new):
        done = n if max_new is None else min(n, max_new)
        if done and length[b] == 0:
            assert np.all(have[m:m + done] == 0)
        elif done:
            want, tol = bound(f64(q[m:m + n]), c, b, Hq, Hkv, scale or HEAD ** -0.5, unpacked)
            err = np.abs(have[m:m + done] - want[:done])
            assert np.all(err <= tol[:done]), f"sequence {b}: {np.max(err / tol[:done])}"
        assert np.all(have[m + done:m + n] == 7.0)
        m += n
    assert np.all(have[m:] == 7.0)
    return out


# Many queries over what might be many keys take the form that unpacks the cache.
UNPACKED = dict(Hq=64, Hkv=1, max_len=100000)


def test_which_form_a_call_takes():
    assert "k_kv4_few" in plan_text([1], [300], 4, 1) and "k_kv4_rows" in plan_text([16], [300], 4, 1) and "k_kv4_rows" in plan_text([300], [333], 4, 2)
    for new in (70, 35, 200):
        assert plan_text([new], [300], 64, 1, max_len=100000).startswith("unpack")
    assert plan_text([80, 5], [300, 40], 128, 2, max_len=400000).startswith("unpack")


BATCHES = [([1], [1]), ([1, 1, 1], [65, 1, 200]), ([16], [16]), ([16, 0, 7], [300, 8, 131]), ([70], [70]), ([200, 3, 1, 64], [200, 3, 150, 190]),
           ([5, 9], [3, 0]), ([1, 1], [64, 128]), ([33, 40], [333, 64]), ([1], [63])]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("new,length", BATCHES)
def test_attention_batches(layout, new, length):
    check_attention(new, length, layout, seed=sum(new))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("new,length", [([70], [70]), ([40, 1, 33], [190, 65, 140]), ([50, 9], [3, 0]), ([100], [333])])
@pytest.mark.parametrize("splits", [0, 3])
def test_attention_unpacked(layout, new, length, splits):
    check_attention(new, length, layout, seed=sum(new), splits=splits, pad=2, **UNPACKED)


def test_attention_unpacked_heads():
    check_attention([80, 5], [300, 40], Hq=128, Hkv=2, max_len=400000, seed=3)
    check_attention([80, 5], [300, 40], Hq=128, Hkv=2, max_len=400000, seed=3, spread=3.0, max_new=78)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (6, 2), (10, 2), (7, 1), (16, 2), (64, 1), (24, 8), (3, 3), (40, 8)])
@pytest.mark.parametrize("new,length", [([1, 1], [129, 40]), ([16], [100]), ([90], [131])])
def test_attention_head_groups(Hq, Hkv, new, length):
    check_attention(new, length, Hq=Hq, Hkv=Hkv, seed=Hq)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64, 256])
@pytest.mark.parametrize("new,length", [([1, 1, 1], [1000, 3, 64]), ([16, 5], [500, 5]), ([150], [600])])
def test_attention_forced_splits(splits, new, length):
    check_attention(new, length, Hq=8, Hkv=2, splits=splits, seed=splits)


@pytest.mark.parametrize("kw", [dict(pad=5), dict(fused=True), dict(scale=0.3), dict(sigma=6.0), dict(max_len=100000), dict(max_new=2), dict(spread=3.0),
                                dict(spread=0.0)])
@pytest.mark.parametrize("new,length", [([1, 1], [300, 77]), ([9, 16], [200, 16]), ([300], [333])])
def test_attention_forms(kw, new, length):
    check_attention(new, length, seed=9, **kw)


def test_attention_many_sequences():
    n = 150
    check_attention([b % 3 for b in range(n)], [b % 3 + b % 70 for b in range(n)], "packed", Hq=2, Hkv=1, seed=6)


def test_attention_every_length_up_to_two_steps():
    """One new token behind every number of keys up to past two steps, in one call."""
    n = 140
    check_attention([1] * n, list(range(n)), Hq=4, Hkv=1, seed=8)


@pytest.mark.parametrize("new,kw", [(1, dict(Hq=4, Hkv=1)), (16, dict(Hq=4, Hkv=1)), (300, dict(Hq=4, Hkv=1)), (60, UNPACKED)])
def test_attention_weights_over_steps_of_all_sizes(new, kw):
    """Steps from 2^-40 to 2^20 in growing and falling order; a row of zeros among the values."""
    L = 400
    for order in (1, -1):
        c = Cache("heads", [L], 1, 5)
        size = 2.0 ** torch.linspace(-40, 20, L).flip(0) if order < 0 else 2.0 ** torch.linspace(-40, 20, L)
        grid = torch.stack([size, -7 * size], -1).to(torch.bfloat16)
        grid[17] = 0
        c.host[3][0, 0, :L] = grid
        c.dev[3][0, 0, :L] = grid.cuda()
        check_attention([new], [L], cache=c, seed=order + 5, **kw)


def test_attention_unpacked_keys_of_all_sizes():
    """Keys whose rows are far apart, against queries that bring their scores into range."""
    c = Cache("heads", [200], 1, 6)
    grid = torch.stack([2.0 ** torch.linspace(-30, 0, 200), -7 * 2.0 ** torch.linspace(-30, 0, 200)], -1).to(torch.bfloat16)
    c.host[1][0, 0, :200] = grid
    c.dev[1][0, 0, :200] = grid.cuda()
    check_attention([60], [200], cache=c, seed=5, **UNPACKED)


@pytest.mark.parametrize("power", [-60, -20, 20, 40])
@pytest.mark.parametrize("new,kw", [(1, dict(Hq=4, Hkv=2)), (12, dict(Hq=4, Hkv=2)), (300, dict(Hq=4, Hkv=2)), (40, UNPACKED)])
def test_attention_queries_of_all_sizes(new, power, kw):
    q = (rand(3, (new, kw["Hq"], HEAD)).double() * 2.0 ** power).to(torch.bfloat16)
    check_attention([new], [320], q=q, scale=2.0 ** -power * 0.1, seed=power + 100, **kw)


@pytest.mark.parametrize("new,length,Hq,Hkv,max_len", [([1, 1], [70, 300], 8, 2, None), ([16, 4], [40, 200], 8, 2, None), ([60], [60], 8, 2, None),
                                                       ([300, 20], [300, 120], 8, 2, None), ([70, 20], [70, 120], 64, 1, 100000)])
def test_attention_what_is_hidden_has_no_influence(new, length, Hq, Hkv, max_len):
    """Codes, steps and offsets behind a token's position, infinities and NaN among them: the rows
    of earlier tokens keep every bit."""
    q = rand(1, (sum(new), Hq, HEAD))
    c = Cache("heads", length, Hkv, 4)
    outs = []
    for junk in (None, float("nan"), float("inf"), 3e38):
        dev = [t.clone() for t in c.dev]
        if junk is not None:
            for b, (n, L) in enumerate(zip(new, length)):
                cut = L - n + n // 2 + 1              # hidden from the first half of the new tokens
                for part in range(4):
                    dev[part][b, :, cut:] = -1 if part % 2 == 0 else junk
        outs.append(qlin.causal_attention_kv4(q.cuda(), dev, i32(starts(new)), i32(length), max_new=max(new), max_len=max_len))
    torch.cuda.synchronize()
    m = 0
    for n in new:
        for other in outs[1:]:
            assert torch.equal(bits(outs[0][m:m + n // 2 + 1]), bits(other[m:m + n // 2 + 1]))
        m += n


@pytest.mark.parametrize("new,G,max_len", [(1, 3, None), (12, 3, None), (300, 3, None), (100, 64, 400000)])
def test_attention_rows_without_numbers(new, G, max_len):
    """A visible NaN row of the cache, and a query of NaN, give NaN; other heads do not see them."""
    L = new + 50
    c = Cache("heads", [L], 2, 1)
    c.dev[1][0, 0, 3] = float("nan")
    q = rand(0, (new, 2 * G, HEAD))
    q[0, G + 1, 7] = float("nan")
    out = qlin.causal_attention_kv4(q.cuda(), c.dev, i32([0, new]), i32([L]), max_new=new, max_len=max_len)
    torch.cuda.synchronize()
    assert torch.isnan(out[:, :G]).all() and torch.isnan(out[0, G + 1]).all()
    assert torch.isfinite(out[:, [G, G + 2]]).all() and torch.isfinite(out[1:, G + 1]).all()


@pytest.mark.parametrize("new,Hq,max_len", [(1, 4, None), (16, 4, None), (300, 4, None), (50, 128, 400000)])
def test_attention_sequences_that_count_as_empty(new, Hq, max_len):
    """Outside the cache, past the room, longer than max_len: zeros."""
    c = Cache("heads", [400] * 4, 2, 2, capacity=400)
    q = rand(0, (4 * new, Hq, HEAD)).cuda()
    at = starts([new] * 4)
    out = qlin.causal_attention_kv4(q, c.dev, i32(at), i32([401, 400, 1 << 30, -5]), max_new=new, max_len=max_len)
    assert not out[:new].any() and out[new:2 * new].any() and not out[2 * new:].any()
    out = qlin.causal_attention_kv4(q, c.dev, i32(at), i32([399, 350, 351, 0]), max_new=new, max_len=350)
    assert not out[:new].any() and out[new:2 * new].any() and not out[2 * new:].any()
    start = torch.tensor([-1, 0, 3200, 2801], dtype=torch.int64, device="cuda")
    out = qlin.causal_attention_kv4(q, c.dev, i32(at), i32([400] * 4), max_new=new, max_len=max_len, cache_start=start)
    assert not out[:new].any() and out[new:2 * new].any() and not out[2 * new:].any()


def test_attention_and_append_past_32_bits_of_offset():
    """A cache whose words begin past 4 GiB of the array."""
    rows = (1 << 26) + 700
    dev = [t for t in qlin.new_kv4_cache(rows, 1)]
    c = Cache("heads", [600], 1, 3)
    at = rows - 650
    for part in range(4):
        dev[part][at:at + 600, 0] = c.dev[part][0, 0, :600]
    start = torch.tensor([at], dtype=torch.int64, device="cuda")
    for new, Hq, max_len in ((1, 2, 600), (16, 2, 600), (300, 2, 600), (100, 64, 100000)):
        q = rand(new, (new, Hq, HEAD)).cuda()
        far = qlin.causal_attention_kv4(q, dev, i32([0, new]), i32([600]), max_new=new, max_len=max_len, cache_start=start)
        near = qlin.causal_attention_kv4(q, c.dev, i32([0, new]), i32([600]), max_new=new, max_len=max_len)
        assert torch.equal(far, near)
    x = [rand(i, (4, HEAD)).cuda() for i in range(3)]
    qlin.norm_rope_append_kv4(*x, dev, i32([0, 4]), i32([640]), cache_start=start)
    codes, step, offset = low.lay_on_grid(f64(x[2]))
    assert torch.equal(dev[2][at + 636:at + 640, 0].cpu(), words_of(codes))
    to = [torch.zeros((rows, 1, HEAD), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    qlin.unpack_kv4(dev, *to, i32([0, 4]), i32([640]), max_len=640, cache_start=start, new_only=True)
    want = low.to_bf16(low.row_values(low.pack_codes(codes), step, offset))
    assert np.array_equal(f64(to[1][at + 636:at + 640, 0]), want) and not to[1][:at + 636].any()


def test_append_and_attention_together():
    """Prompt, blocks cut back and single tokens through one cache: what the attention reads is what
    the append stored, and lengths that change between replays of one graph."""
    Hq, Hkv, cap = 8, 2, 700
    freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    cache = qlin.new_kv4_cache(2, Hkv, cap)
    mirror = [torch.zeros((2, Hkv, cap, HEAD), dtype=torch.bfloat16, device="cuda") for _ in "kv"]

    def step(x, at, length, n):
        q = qlin.norm_rope_append_kv4(x[:, :Hq * HEAD], x[:, Hq * HEAD:(Hq + Hkv) * HEAD], x[:, (Hq + Hkv) * HEAD:], cache, at, length,
                                      max_new=n, inv_freq=freq)
        return q, qlin.causal_attention_kv4(q, cache, at, length, max_new=n)

    wide = (Hq + 2 * Hkv) * HEAD
    for new, length in [([300, 211], [300, 211]), ([16, 16], [316, 227]), ([16, 16], [309, 230]), ([1, 1], [310, 231])]:
        x = rand(sum(length), (sum(new), wide)).cuda()
        q, out = step(x, i32(starts(new)), i32(length), max(new))
        # the bf16 attention over the unpacked cache
        qlin.unpack_kv4(cache, *mirror, i32(starts(new)), i32(length))
        same = qlin.causal_attention(q, *mirror, i32(starts(new)), i32(length), max_new=max(new))
        # keys and values rounded to bf16, and weights: 2^-8 each, of scores up to about 10 and values up to about 4
        assert (out.float() - same.float()).abs().max() < 0.1 and (out.float() - same.float()).norm() < 0.01 * same.float().norm()
    x, at, length = rand(1, (2, wide)).cuda(), i32([0, 1, 2]), i32([311, 232])
    step(x, at, length, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, out = step(x, at, length, 1)
    for i in range(5):
        x.copy_(rand(50 + i, (2, wide)))
        length.copy_(i32([312 + i, 233 + 2 * i]))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step(x, at, length, 1)[1])


@pytest.mark.parametrize("new,Hq,Hkv,max_len", [(1, 8, 2, 603), (40, 8, 2, 603), (100, 64, 1, 100000)])
def test_graphs_that_share_a_workspace_and_streams(new, Hq, Hkv, max_len):
    L = 600
    c = Cache("heads", [L], Hkv, 1)
    b = qlin.Batch(1, new, new, max_len, None, None, None)
    ws = torch.empty(qlin.qlin_causal_four_bit_plan(b, Hq, Hkv, HEAD)[1], dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    qs, at, length = [rand(i, (new, Hq, HEAD)).cuda() for i in range(2)], i32([0, new]), i32([L])
    run = lambda q, w: qlin.causal_attention_kv4(q, c.dev, at, length, max_new=new, max_len=max_len, workspace=w)
    want = [run(q, None).clone() for q in qs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(q, ws))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
        ws.fill_(255)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    results = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            results.append(run(qs[i % 2], None))
    torch.cuda.synchronize()
    assert all(torch.equal(r, want[i % 2]) for i, r in enumerate(results))


def test_binding_checks():
    c = qlin.new_kv4_cache(2, 2, 32)
    q = torch.zeros((1, 4, HEAD), dtype=torch.bfloat16, device="cuda")
    at, length = i32([0, 1]), i32([3])
    for bad in [(c[0][:, :1], *c[1:]), (c[0].cpu(), *c[1:]), (c[0], c[1].float(), *c[2:]), (c[0][..., :8], c[1], c[2][..., :8], c[3]),
                (c[0].transpose(0, 1), *c[1:]), (c[0][:, :, ::2], c[1][:, :, :16], c[2][:, :, ::2], c[3][:, :, :16])]:
        with pytest.raises(ValueError):
            qlin.causal_attention_kv4(q, bad, at, length)
    with pytest.raises(ValueError):
        qlin.causal_attention_kv4(q, c, at, length.long())
    with pytest.raises(ValueError):
        qlin.causal_attention_kv4(q, qlin.new_kv4_cache(32, 2), i32([0, 1, 1]), i32([3, 2]))
    to = [torch.zeros((2, 2, 31, HEAD), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    with pytest.raises(ValueError):
        qlin.unpack_kv4(c, *to, at, length)
