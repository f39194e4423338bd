"""GPU tests of the target's operators (include/qlin_target.h) against the float64
oracle, through the Python entry points.

Tolerances, derived (bf16 rounds by at most half a step, 2^-8 of the value):
* append: 2^-8 |y| for the one rounding; 2^-20 (|x| + |partner|) for the norm (128
  squares summed in fp32, at most 2^-17 of the sum over 2 in its root, far more than the
  rounding errors can reach when they do not all agree, so 2^-20 is used) and for cosine
  and sine (a turn's rest rounded to fp32, 2^-25 of a turn, and 2 ulp).
* attention: each weight is rounded to bf16 once, w (1 + d) with |d| <= 2^-8, and the
  sum adds the rounded weights, so |out - ref| <= d / (1 - d) (A + |ref|) with A = sum_j
  p_j |v_j|.  d also holds exp2 (2^-20) and the fp32 scores (128 products: 128 2^-24
  scale sum |q||k|, and the rounding of score times scale, in exponent units).  fp32 sums
  over n keys add 2 n 2^-24 A, the output's rounding 2^-8 |ref|.
* verification gives whole numbers: equal.
"""

import numpy as np
import pytest
import torch

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


class Cache:
    """A cache in one of several layouts, and its tokens as [L, heads, 128] float64."""

    def __init__(self, layout, length, Hkv, seed, capacity=None, fill=None):
        n, cap = len(length), capacity or max(max(length), 1) + 3
        self.layout, self.length, self.start = layout, length, None
        make = (lambda s, shape: rand(s, shape)) if fill is None else (lambda s, shape: torch.full(shape, fill).to(torch.bfloat16))
        if layout == "heads":                 # [sequences, heads, capacity, 128]
            self.host = [make(seed + i, (n, Hkv, cap, HEAD)) for i in (0, 1)]
            self.dev = [t.cuda() for t in self.host]
        elif layout == "tokens":              # [sequences, capacity, heads, 128] seen with heads first
            self.host = [make(seed + i, (n, cap, Hkv, HEAD)).transpose(1, 2) for i in (0, 1)]
            self.dev = [t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in self.host]
        else:                                 # packed [tokens, heads, 128], sequences in mixed order, gaps between
            at, self.at = 2, [0] * n
            for b in sorted(range(n), key=lambda b: (b * 5 + 2) % 7):
                self.at[b] = at
                at += length[b] + b % 3
            wide = [make(seed + i, (at + 1, Hkv, HEAD + 8)) for i in (0, 1)]
            self.host = [t[:, :, :HEAD] for t in wide]
            self.dev = [t.cuda()[:, :, :HEAD] for t in wide]
            self.start = torch.tensor(self.at, dtype=torch.int64, device="cuda")

    def tokens(self, which, b, source=None):
        t = (source or self.host)[which]
        L = self.length[b]
        return t[self.at[b]:self.at[b] + L] if self.layout == "packed" else t[b, :, :L].transpose(0, 1)

    def kwargs(self):
        return dict(length=i32(self.length), cache_start=self.start)


LAYOUTS = ("heads", "tokens", "packed")


# ---------------------------------------------------------------- append


def check_append(new, length, layout="heads", Hq=4, Hkv=2, norm=True, rot=128, interleaved=False, pad=0, eps=1e-6, fused=False,
                 in_place=False, theta=1e4, seed=0, max_new=None, offset=0):
    M = sum(new) + pad
    c = Cache(layout, length, Hkv, seed + 10)
    if fused:                              # q, k, v are slices of one projection's rows
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
    got = qlin.norm_rope_append(*devs, *c.dev, i32(starts(new)), max_new=max_new, q_norm=None if wq is None else wq.cuda(),
                                k_norm=None if wk is None else wk.cuda(), eps=eps, inv_freq=freq.cuda() if rot else None,
                                interleaved=interleaved, out=out, **c.kwargs())
    torch.cuda.synchronize()
    assert got is out
    rows = ref.positions(new, length)
    freq = freq.numpy() if rot else np.zeros(0)
    want_k, want_v = f64(c.host[0]).copy(), c.host[1].clone()
    tol_k = np.zeros(want_k.shape)
    want_q = f64(host[0]).reshape(M, Hq, HEAD) if in_place else np.full((M, Hq, HEAD), 7.0)
    tol_q = np.zeros(want_q.shape)

    def expected(x, w):
        n = ref.norm(x, None if w is None else f64(w), eps)
        y = ref.rotate(n, p, freq, interleaved)
        big = np.abs(n).max(axis=1, keepdims=True)
        return y, 2.0 ** -8 * np.abs(y) + 2.0 ** -19 * big + 1e-38

    for m, (b, p) in enumerate(rows):
        if max_new is not None and m - starts(new)[b] >= max_new:
            continue
        want_q[m], tol_q[m] = expected(f64(host[0][m]).reshape(Hq, HEAD), wq)
        if p < 0:
            continue
        at = (c.at[b] + p,) if layout == "packed" else (b, slice(None), p)
        want_k[at], tol_k[at] = expected(f64(host[1][m]).reshape(Hkv, HEAD), wk)
        want_v[at] = host[2][m].view(Hkv, HEAD)
    assert np.all(np.abs(f64(out) - want_q) <= tol_q)
    assert np.all(np.abs(f64(c.dev[0]) - want_k) <= tol_k)
    assert torch.equal(c.dev[1].cpu().view(torch.int16), want_v.view(torch.int16))


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


def test_append_many_rows():
    """The form for many tokens (several a workgroup), a last workgroup partly filled."""
    check_append([700, 1, 0, 522], [700, 900, 5, 600], "packed", Hq=3, Hkv=1, pad=4, seed=9)


@pytest.mark.parametrize("rows,kw", [(639, dict(fused=True)), (640, dict(fused=True, in_place=True)), (641, dict(pad=6, interleaved=True, rot=48)),
                                     (643, dict(rot=0, max_new=300))])
def test_append_around_the_change_of_form(rows, kw):
    """Either side of the rows from which a workgroup takes several tokens; sequences that meet
    inside a workgroup, one of them ahead of its first position."""
    check_append([rows - 333, 1, 0, 2, 330], [rows, 1, 0, 1, 331], "packed", Hq=3, Hkv=1, seed=rows, **kw)


def test_append_far_positions_keep_their_angles():
    """Position 2^24 + 5: the first frequency turns 2.7 million times."""
    n = (1 << 24) + 6
    k = torch.zeros((1, 1, n, HEAD), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    x = rand(1, (2, HEAD))
    freq = 1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)
    qlin.norm_rope_append(x.cuda(), x.cuda(), x.cuda(), k, v, i32([0, 2]), i32([n]), inv_freq=freq.cuda())
    torch.cuda.synchronize()
    for i in (0, 1):
        want = ref.rotate(f64(x[i:i + 1]), n - 2 + i, freq.numpy(), False)[0]
        tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.abs(f64(x[i])).max()
        assert np.all(np.abs(f64(k[0, 0, n - 2 + i]) - want) <= tol)
    assert torch.all(k[0, 0, :n - 2] == 0)


def test_append_more_new_tokens_than_declared_are_left_out():
    check_append([9, 2], [20, 30], max_new=4, seed=5)


def test_append_many_sequences():
    n = 150
    check_append([b % 3 for b in range(n)], [b % 3 + b % 5 for b in range(n)], "packed", Hq=2, Hkv=1, seed=6)


def test_append_infinite_and_zero_rows():
    """A zero row stays zero under a norm (eps > 0); infinities and NaN stay in their head."""
    q = torch.zeros((2, 2 * HEAD), dtype=torch.bfloat16)
    q[1] = rand(0, (2 * HEAD,))
    q[1, 3] = float("inf")
    k, v = rand(1, (2, HEAD)), rand(2, (2, HEAD))
    v[0, 5], v[1, 6] = float("inf"), float("nan")
    c = Cache("heads", [2], 1, 4)
    w = torch.ones(HEAD, dtype=torch.bfloat16, device="cuda")
    out = qlin.norm_rope_append(q.cuda(), k.cuda(), v.cuda(), *c.dev, i32([0, 2]), q_norm=w, k_norm=w,
                                inv_freq=torch.ones(64, dtype=torch.float64, device="cuda"), **c.kwargs())
    torch.cuda.synchronize()
    assert torch.all(out[0] == 0) and not torch.isfinite(out[1, 0]).all() and torch.isfinite(out[1, 1]).all()
    assert torch.equal(c.dev[1][0, 0, :2].cpu().view(torch.int16), v.view(torch.int16))


# ---------------------------------------------------------------- attention


def check_attention(new, length, layout="heads", Hq=4, Hkv=2, splits=0, seed=0, sigma=2.0, scale=0.0, pad=0, fused=False,
                    max_new=None, max_len=None, cache=None, q=None, out=None):
    M = sum(new) + pad
    c = cache or Cache(layout, length, Hkv, seed + 10)
    if q is None:
        q = rand(seed, (M, Hq + (3 if fused else 0), HEAD), sigma)[:, :Hq]
    dev = q.cuda() if not fused else torch.cat([q, torch.zeros(M, 3, HEAD, dtype=torch.bfloat16)], 1).cuda()[:, :Hq]
    out = torch.full((M, Hq, HEAD), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    got = qlin.causal_attention(dev, *c.dev, i32(starts(new)), max_new=max(new) if max_new is None else max_new,
                                max_len=max_len, scale=scale, splits=splits, out=out, **c.kwargs())
    torch.cuda.synchronize()
    assert got is out
    have, m = f64(out), 0
    sc = scale or HEAD ** -0.5
    for b, n in enumerate(new):
        done = n if max_new is None else min(n, max_new)
        if done:
            keys, values, qb = f64(c.tokens(0, b)), f64(c.tokens(1, b)), f64(q[m:m + n])
            want, A = ref.causal_attention(qb, keys, values, sc)
            size = max([float((np.abs(qb[:, h]) @ np.abs(keys[:, h // (Hq // Hkv)]).T).max()) for h in range(Hq)] or [0.0]) if len(keys) else 0.0
            d = 2.0 ** -8 + 2.0 ** -20 + (HEAD + 2) * 2.0 ** -24 * size * sc
            tol = d / (1 - d) * (A + np.abs(want)) + 2 * length[b] * 2.0 ** -24 * A + 2.0 ** -8 * np.abs(want) + 1e-38
            err = np.abs(have[m:m + done] - want[:done])
            assert np.all(err <= tol[:done]), f"sequence {b}: {np.max(err - tol[:done])}"
        assert np.all(have[m + done:m + n] == 7.0)
        m += n
    assert np.all(have[m:] == 7.0)
    return out


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("new,length", [([1], [1]), ([1, 1, 1], [65, 1, 200]), ([16], [16]), ([16, 0, 7], [300, 8, 131]),
                                        ([70], [70]), ([200, 3, 1, 64], [200, 3, 150, 190]), ([5, 9], [3, 0])])
def test_attention_batches(layout, new, length):
    check_attention(new, length, layout, seed=sum(new))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (6, 2), (10, 2), (7, 1), (16, 2), (64, 1), (24, 8), (3, 3), (40, 8)])
@pytest.mark.parametrize("new,length", [([1, 1], [129, 40]), ([16], [100]), ([90], [131])])
def test_attention_head_groups(Hq, Hkv, new, length):
    check_attention(new, length, Hq=Hq, Hkv=Hkv, seed=Hq)


@pytest.mark.parametrize("splits", [1, 2, 5])
@pytest.mark.parametrize("new,length", [([33], [33]), ([40, 200, 1, 64], [40, 995, 1, 64]), ([130, 17], [1100, 16]), ([20, 0, 34], [352, 0, 65]),
                                        ([300], [300]), ([25], [2000])])
def test_attention_prompts_in_two_halves(splits, new, length):
    """A large bound of the lengths takes the form whose workgroups walk two halves of a range:
    one step of keys and none, odd numbers of steps, a last step that is no whole one."""
    b = qlin.Batch(len(new), sum(new), max(new), 1 << 20, None, None, None)
    assert "k_causal_prompt<2>" in qlin.qlin_causal_plan(b, 8, 2, HEAD, splits)[2]
    check_attention(new, length, Hq=8, Hkv=2, splits=splits, max_len=1 << 20, pad=3, seed=7)


@pytest.mark.parametrize("splits", [1, 2, 3, 7, 64, 256])
@pytest.mark.parametrize("new,length", [([1, 1, 1], [1000, 3, 64]), ([16, 5], [500, 5]), ([150], [600])])
def test_attention_forced_splits(splits, new, length):
    check_attention(new, length, Hq=8, Hkv=2, splits=splits, seed=splits)


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 127, 128, 129, 257])
def test_attention_prompt_lengths(n):
    check_attention([n, 1, n // 2], [n, n, n], "packed", seed=n)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513])
def test_attention_single_token_lengths(n):
    check_attention([1, 1], [n, max(n - 1, 1)], Hq=8, Hkv=2, seed=n)


@pytest.mark.parametrize("kw", [dict(pad=11), dict(fused=True), dict(scale=0.3), dict(scale=1e-6), dict(max_len=1), dict(sigma=12.0),
                                dict(max_new=3), dict(max_new=0), dict(max_len=1 << 28)])
@pytest.mark.parametrize("new,length", [([4, 1, 9], [60, 70, 9]), ([100, 40], [100, 300])])
def test_attention_forms(kw, new, length):
    check_attention(new, length, Hq=8, Hkv=2, seed=2, **kw)


@pytest.mark.parametrize("new,length,Hq,Hkv", [([1], [5000], 32, 8), ([16], [3000], 32, 8), ([1] * 70, list(range(1, 141, 2)), 8, 2),
                                               ([16] * 20, [16 + 9 * b for b in range(20)], 16, 4)])
def test_attention_larger_batches(new, length, Hq, Hkv):
    check_attention(new, length, Hq=Hq, Hkv=Hkv, seed=4)


def planned(new, length, Hq, Hkv, splits=0):
    b = qlin.Batch(len(new), sum(new), max(new), max(length), None, None, None)
    return qlin.qlin_causal_plan(b, Hq, Hkv, HEAD, splits)


@pytest.mark.parametrize("new,length", [([1, 1], [70, 200]), ([16], [90]), ([33], [161]), ([150], [150]), ([64, 70], [256, 70])])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_attention_sees_the_past_exactly(new, length, splits):
    """q = 0 gives every visible key the weight 1, and one-hot values count them: key j
    has a 1 in dimension j % 128, so dimension d is (visible keys of that residue) / (visible
    keys), and a key too many or too few shows."""
    Hq, Hkv = 8, 2
    c = Cache("heads", length, Hkv, 1)
    c.host[1].zero_()
    for j in range(c.host[1].shape[2]):
        c.host[1][:, :, j, j % HEAD] = 1.0
    c.dev[1].copy_(c.host[1])
    q = torch.zeros((sum(new), Hq, HEAD), dtype=torch.bfloat16)
    out = f64(check_attention(new, length, Hq=Hq, Hkv=Hkv, splits=splits, cache=c, q=q))
    for m, (b, p) in enumerate(ref.positions(new, length)):
        count = np.array([len(range(d, p + 1, HEAD)) for d in range(HEAD)])
        assert np.all(np.abs(out[m] - count / (p + 1)) <= 2.0 ** -8 * count / (p + 1)), (m, p)
        assert np.all(out[m][:, count == 0] == 0)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan"), 3e38, -3e38])
@pytest.mark.parametrize("new,length,splits", [([16], [100], 0), ([16], [100], 3), ([130], [130], 0), ([130], [330], 2), ([3, 1], [40, 40], 0)])
def test_attention_keys_and_values_behind_a_token_have_no_influence(new, length, splits, bad):
    """The bits of every output stay the same when what is behind its token is replaced:
    later tokens of the sequence (from the last few on) and the unused capacity."""
    Hq, Hkv = 8, 2
    c = Cache("heads", length, Hkv, 5)
    q = rand(6, (sum(new), Hq, HEAD), 2.0)
    first = check_attention(new, length, Hq=Hq, Hkv=Hkv, splits=splits, cache=c, q=q).clone()
    for b, L in enumerate(length):
        for t in c.dev:
            t[b, :, L - 2:] = bad
            t[b, 0, L - 2:, 5] = -bad
    second = torch.zeros_like(first)
    qlin.causal_attention(q.cuda(), *c.dev, i32(starts(new)), max_new=max(new), splits=splits, out=second, **c.kwargs())
    torch.cuda.synchronize()
    m = 0
    for b, n in enumerate(new):
        keep = slice(m, m + max(n - 2, 0))
        assert torch.equal(first[keep].view(torch.int16), second[keep].view(torch.int16)), (b, n)
        m += n


@pytest.mark.parametrize("new,length,splits,max_len", [([130], [130], 1, 1 << 20), ([130, 20], [611, 33], 2, 1 << 20), ([64], [32 * 5 + 64], 1, 1 << 20),
                                                       ([60], [700], 1, None), ([61], [900], 2, None), ([3], [900], 1, None), ([4, 4], [600, 33], 2, None),
                                                       ([7], [1000], 1, None), ([16, 9], [1100, 70], 1, None)])
def test_attention_of_long_walks_without_influence_from_behind(new, length, splits, max_len):
    """As above over many steps of every kernel, the first ones in the form of two halves, where
    the keys and values behind a token lie in its tile; and one-hot values that count the keys of
    each row."""
    Hq, Hkv = 8, 2
    c = Cache("heads", length, Hkv, 5)
    c.host[1].zero_()
    for j in range(c.host[1].shape[2]):
        c.host[1][:, :, j, j % HEAD] = 1.0
    c.dev[1].copy_(c.host[1])
    q = torch.zeros((sum(new), Hq, HEAD), dtype=torch.bfloat16)
    form = dict(splits=splits, max_len=max_len)
    out = f64(check_attention(new, length, Hq=Hq, Hkv=Hkv, cache=c, q=q, **form))
    for m, (b, p) in enumerate(ref.positions(new, length)):
        count = np.array([len(range(d, p + 1, HEAD)) for d in range(HEAD)])
        assert np.all(np.abs(out[m] - count / (p + 1)) <= 2.0 ** -8 * count / (p + 1)), (m, p)
        assert np.all(out[m][:, count == 0] == 0)
    q = rand(6, (sum(new), Hq, HEAD), 2.0)
    first = check_attention(new, length, Hq=Hq, Hkv=Hkv, cache=c, q=q, **form).clone()
    for bad in (float("inf"), float("nan"), -3e38, 40.0):
        for b, L in enumerate(length):
            for t in c.dev:
                t[b, :, L - 2:] = bad
        second = torch.zeros_like(first)
        qlin.causal_attention(q.cuda(), *c.dev, i32(starts(new)), max_new=max(new), out=second, **form, **c.kwargs())
        torch.cuda.synchronize()
        m = 0
        for b, n in enumerate(new):
            assert torch.equal(first[m:m + n - 2].view(torch.int16), second[m:m + n - 2].view(torch.int16)), (b, bad)
            m += n


def test_attention_infinite_values_reach_those_that_see_them():
    """A visible infinite value makes its dimension infinite, the others stay; a visible NaN
    key makes the row NaN; a key of -infinity score has no weight."""
    new, length = [20], [60]
    c = Cache("heads", length, 1, 7)
    q = rand(8, (20, 2, HEAD), 0.1).abs()
    base = f64(check_attention(new, length, Hq=2, Hkv=1, cache=c, q=q))
    c.dev[1][0, 0, 50, 9] = float("inf")           # seen from row 10 on
    c.dev[0][0, 0, 55] = float("nan")              # seen from row 15 on
    out = torch.zeros((20, 2, HEAD), dtype=torch.bfloat16, device="cuda")
    qlin.causal_attention(q.cuda(), *c.dev, i32([0, 20]), max_new=20, out=out, **c.kwargs())
    torch.cuda.synchronize()
    out = f64(out)
    rest = np.arange(HEAD) != 9
    assert np.array_equal(out[:10], base[:10]) and np.all(np.isposinf(out[10:15, :, 9])) and np.all(np.isnan(out[15:]))
    assert np.all(np.abs(out[10:15][..., rest] - base[10:15][..., rest]) <= 2.0 ** -7 * np.abs(base[10:15][..., rest]) + 1e-30)
    c2 = Cache("heads", length, 1, 7)
    c2.dev[0][0, 0, 3] = float("-inf")             # positive queries: score -infinity
    c2.dev[1][0, 0, 3] = 1e4
    qlin.causal_attention(q.cuda(), *c2.dev, i32([0, 20]), max_new=20, out=(o2 := torch.zeros((20, 2, HEAD), dtype=torch.bfloat16, device="cuda")), **c2.kwargs())
    torch.cuda.synchronize()
    assert torch.isfinite(o2).all() and float(o2.abs().max()) < 100


def test_attention_far_heads_and_sequences():
    """Heads and sequences more than 2^32 bytes apart."""
    cap = 9 << 20                                   # 2.4 GB a head
    k, v = (torch.zeros((2, 2, cap, HEAD), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for new, L in ((3, 150), (80, 150)):
        host = [rand(20 + i, (2, 2, L, HEAD)) for i in (0, 1)]
        k[:, :, :L], v[:, :, :L] = host[0].cuda(), host[1].cuda()
        q = rand(3, (2 * new, 4, HEAD), 2.0)
        out = qlin.causal_attention(q.cuda(), k, v, i32([0, new, 2 * new]), i32([L, L]), max_new=new, max_len=L)
        torch.cuda.synchronize()
        for b in (0, 1):
            want, A = ref.causal_attention(f64(q[b * new:(b + 1) * new]), f64(host[0][b].transpose(0, 1)), f64(host[1][b].transpose(0, 1)), HEAD ** -0.5)
            assert np.all(np.abs(f64(out[b * new:(b + 1) * new]) - want) <= 2.0 ** -7 * (A + np.abs(want)) + 2.0 ** -8 * np.abs(want))


def test_attention_sequences_outside_the_cache_are_empty():
    c = Cache("packed", [30, 40, 20], 2, 3)
    q = rand(1, (12, 4, HEAD))
    for start, length in (([-1, 0, 5], [30, 40, 20]), ([0, 1 << 50, 0], [30, 40, 20]), ([0, 0, 0], [30, 1 << 30, -5])):
        out = torch.full((12, 4, HEAD), 7.0, dtype=torch.bfloat16, device="cuda")
        s = torch.tensor(start, dtype=torch.int64, device="cuda")
        qlin.causal_attention(q.cuda(), *c.dev, i32([0, 4, 8, 12]), i32(length), max_new=4, cache_start=s, out=out)
        before = [t.clone() for t in c.dev]
        qlin.norm_rope_append(q.cuda().view(12, 512), q.cuda().view(12, 512)[:, :256], q.cuda().view(12, 512)[:, :256],
                              *c.dev, i32([0, 4, 8, 12]), i32(length), cache_start=s)
        torch.cuda.synchronize()
        slots = c.dev[0].shape[0]
        for b in range(3):
            L = max(length[b], 0)
            inside = start[b] >= 0 and start[b] + L <= slots and L > 0
            assert bool((out[4 * b:4 * b + 4] == 0).all()) != inside
        for t, t0 in zip(c.dev, before):
            for j in range(slots):
                written = any(0 <= start[b] and start[b] + max(length[b], 0) <= slots and length[b] > 0 and
                              start[b] + length[b] - 4 <= j < start[b] + length[b] for b in range(3))
                assert written or torch.equal(t[j].view(torch.int16), t0[j].view(torch.int16))


def test_bounds_that_are_not_ascending_stay_inside():
    """Row bounds out of order or range: no access outside (the results are the caller's)."""
    c = Cache("heads", [30, 40], 2, 3)
    q = rand(1, (12, 4, HEAD)).cuda()
    for bounds in ([5, 3, 12], [-7, 6, 100], [12, 12, 12], [0, 1 << 30, 4]):
        out = torch.full((12, 4, HEAD), 7.0, dtype=torch.bfloat16, device="cuda")
        qlin.causal_attention(q, *c.dev, i32(bounds), i32([30, 40]), out=out)
        qlin.norm_rope_append(q.view(12, 512), q.view(12, 512)[:, :256], q.view(12, 512)[:, :256], *c.dev, i32(bounds), i32([30, 40]))
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()


def test_attention_repeats_its_bits_on_any_stream():
    new, length = [16, 1, 40], [900, 700, 40]
    c = Cache("heads", length, 2, 1)
    q = rand(2, (57, 8, HEAD), 2.0).cuda()
    b = dict(new_start=i32(starts(new)), max_new=40, **c.kwargs())
    a = qlin.causal_attention(q, *c.dev, **b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        d = qlin.causal_attention(q, *c.dev, **b)
    s.synchronize()
    assert torch.equal(a.view(torch.int16), d.view(torch.int16))


# ---------------------------------------------------------------- verification


def check_verify(target, draft, drafted, u, T=None, count=None, stride=None):
    n, rows, V = target.shape
    dev = target.cuda()
    ddev = None if draft is None else draft.cuda()
    if stride:
        wide = torch.zeros((n, rows, stride), dtype=torch.bfloat16, device="cuda")
        wide[:, :, :V] = dev
        wide[:, :, V:] = 1e4
        dev = wide[:, :, :V]
        if draft is not None:
            wide = torch.full((n, rows - 1, stride), 1e4, dtype=torch.bfloat16, device="cuda")
            wide[:, :, :V] = ddev
            ddev = wide[:, :, :V]
    acc, tok = qlin.verify_draft(dev, i32(drafted).view(n, rows - 1), torch.tensor(u, dtype=torch.float32, device="cuda").view(n, rows), draft=ddev,
                                 n_draft=None if count is None else i32(count),
                                 temperature=None if T is None else torch.tensor(T, dtype=torch.float32, device="cuda"))
    torch.cuda.synchronize()
    acc, tok = acc.cpu().tolist(), tok.cpu().tolist()
    t64, d64 = f64(target), None if draft is None else f64(draft)
    for b in range(n):
        c = rows - 1 if count is None else min(max(count[b], 0), rows - 1)
        ub = np.float32(u[b]).astype(np.float64)
        a, nxt = ref.verify(t64[b, :c + 1], None if draft is None else d64[b, :c], drafted[b][:c], [*ub[:c], ub[rows - 1]],
                            1.0 if T is None else float(np.float32(T[b])))
        assert (acc[b], tok[b]) == (a, [*drafted[b][:a], nxt] + [-1] * (rows - 1 - a)), b
    return acc


def verify_case(n, drafts, V, seed, near=0.4, with_draft=True):
    rng = np.random.default_rng(seed)
    target = rand(seed, (n, drafts + 1, V), 2.0)
    draft = (target[:, :drafts].float() + near * torch.randn((n, drafts, V), generator=torch.Generator().manual_seed(seed + 1))).to(torch.bfloat16)
    z = draft.float().numpy() - np.log(-np.log(rng.random((n, drafts, V)))) if with_draft else draft.float().numpy()
    drafted = z.argmax(2).tolist() if drafts else [[] for _ in range(n)]
    u = rng.random((n, drafts + 1)).astype(np.float32).tolist()
    return target, draft if with_draft else None, drafted, u


@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("n,drafts,V", [(1, 1, 2), (5, 3, 1), (4, 0, 700), (3, 15, 1000), (6, 5, 4097), (2, 2, 50257), (1, 64, 333), (9, 4, 2055), (40, 7, 129)])
def test_verify(n, drafts, V, with_draft):
    acc = check_verify(*verify_case(n, drafts, V, n + drafts + V, with_draft=with_draft))
    assert len(acc) == n


@pytest.mark.parametrize("with_draft", [True, False])
def test_verify_large_vocabulary_temperatures_and_counts(with_draft):
    target, draft, drafted, u = verify_case(8, 7, 151936, 3, with_draft=with_draft)
    acc = check_verify(target, draft, drafted, u, T=[0.0, 0.5, 1.0, 1.7, -1.0, 0.01, float("nan"), 30.0], count=[7, 0, 3, 9, 7, 2, -4, 7])
    assert max(acc) > 0


@pytest.mark.parametrize("V,stride", [(1000, 1001), (777, 1024), (50257, 50260), (8, 9)])
def test_verify_rows_at_any_distance(V, stride):
    target, draft, drafted, u = verify_case(3, 4, V, V)
    check_verify(target, draft, drafted, u, T=[1.0, 0.0, 0.8], stride=stride)


def test_verify_masked_tokens_and_empty_rows():
    target, draft, drafted, u = verify_case(6, 3, 500, 1)
    target[0, 0] = float("-inf")                                       # nothing left at the first token
    target[1, 1] = float("nan")
    target[2, :, 100:] = float("-inf")
    target[3, 0, 17] = float("inf")
    target[3, 1, 40:60] = float("inf")
    draft[4, 0] = float("-inf")
    draft[5, :, ::2] = float("nan")
    target[5, 3, :499] = float("-inf")
    for T in ([1.0] * 6, [0.0] * 6):
        check_verify(target, draft, drafted, u, T=T)
        check_verify(target, None, drafted, u, T=T)


def test_verify_drafted_tokens_outside_the_vocabulary():
    target, draft, drafted, u = verify_case(4, 2, 300, 2)
    drafted = [[-1, 5], [300, 5], [2 ** 31 - 1, 0], [-2 ** 31, 0]]
    for d in (draft, None):
        assert check_verify(target, d, drafted, u) == [0, 0, 0, 0]


def test_verify_edges_of_the_uniform_numbers():
    """u = 0 keeps whatever has any probability and draws the first possible token; the
    largest number below 1 draws the last."""
    target, draft, drafted, _ = verify_case(2, 3, 400, 5)
    target[:, :, 7] = float("-inf")
    top = float(np.nextafter(np.float32(1), np.float32(0)))
    assert check_verify(target, draft, drafted, [[0.0] * 4, [0.0] * 4])[0] >= 0
    check_verify(target, draft, drafted, [[top] * 4, [top] * 4])
    check_verify(target, target[:, :3].clone(), drafted, [[top] * 4, [top] * 4])         # the same laws: all kept
    same = check_verify(target, target[:, :3].clone(), [[1, 2, 3], [4, 5, 6]], [[top] * 4, [0.3] * 4])
    assert same == [3, 3]


def test_verify_ties_take_the_lowest_index():
    target = torch.zeros((2, 2, 3000), dtype=torch.bfloat16)
    target[0, 0, [5, 1500, 2999]] = 3.0
    target[1, 0, [2998, 2999]] = 3.0
    assert check_verify(target, None, [[5], [2999]], [[0.5, 0.5], [0.5, 0.5]], T=[0.0, 0.0]) == [1, 0]


def test_verify_large_calls_look_at_the_first_rows_first():
    """Above 2^26 logits a third of the rows is looked at first: sequences that end there and
    behind it, counts on both sides, greedy ones, and a drafter whose tokens are all kept."""
    n, drafts, V = 16, 15, 151936
    g = torch.Generator(device="cuda").manual_seed(1)
    target = (2.0 * torch.randn((n, drafts + 1, V), device="cuda", generator=g)).to(torch.bfloat16)
    draft = (target[:, :drafts].float() + 0.3 * torch.randn((n, drafts, V), device="cuda", generator=g)).to(torch.bfloat16)
    draft[5], draft[9] = target[5, :drafts], target[9, :drafts]
    drafted = (draft.float() - torch.empty_like(draft, dtype=torch.float32).exponential_(generator=g).log()).argmax(2)
    T = [1.0, 0.0, 0.9, 1.3, 0.0, 1.0, 1.0, 0.8, 1.0, 1.0, 1.0, 0.7, 1.0, 1.0, 0.0, 1.0]
    drafted[1] = target[1, :drafts].argmax(1)
    drafted = drafted.tolist()
    u = np.random.default_rng(2).random((n, drafts + 1)).astype(np.float32).tolist()
    count = [15] * 10 + [4, 5, 6, 0, 15, 5]
    assert n * (2 * drafts + 1) * V >= 1 << 26
    acc = check_verify(target, draft, drafted, u, T=T, count=count)
    assert max(acc) == 15 and min(acc) < 5
    target2 = torch.cat([target, target])                               # without draft logits: 2^26 again
    best = target2[:, :drafts].argmax(2)
    best[::2, 3:] = 7
    assert 2 * n * (drafts + 1) * V >= 1 << 26
    acc = check_verify(target2, None, best.tolist(), u + u, T=[0.0] * n + [0.2] * n, count=count + count)
    assert max(acc) >= 5


# ---------------------------------------------------------------- together


def test_two_streams_at_once():
    """The operators on two streams at the same time, each with scratch of its own."""
    new, length = [16, 3], [3000, 700]
    c = Cache("heads", length, 2, 1)
    q = [rand(i, (19, 8, HEAD), 2.0).cuda() for i in (2, 3)]
    v = [verify_case(4, 7, 50257, s) for s in (1, 2)]
    v = [(t.cuda(), i32(x), torch.tensor(u, device="cuda"), d.cuda()) for t, d, x, u in v]
    b = dict(new_start=i32(starts(new)), max_new=16, **c.kwargs())
    alone = [(qlin.causal_attention(q[i], *c.dev, **b).clone(), *[t.clone() for t in qlin.verify_draft(*v[i][:3], draft=v[i][3])]) for i in (0, 1)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in (0, 1)], [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((qlin.causal_attention(q[i], *c.dev, **b), *qlin.verify_draft(*v[i][:3], draft=v[i][3])))
    torch.cuda.synchronize()
    for i in (0, 1):
        for out, acc, tok in got[i]:
            assert torch.equal(out.view(torch.int16), alone[i][0].view(torch.int16))
            assert torch.equal(acc, alone[i][1]) and torch.equal(tok, alone[i][2])


def test_graphs_that_share_a_workspace():
    """Two captured graphs over one workspace, replayed in turn on one stream between eager calls:
    attention split over keys, single tokens and blocks, and the decision with draft logits."""
    c = Cache("heads", [4000, 3100], 2, 1)
    logits, draft, tokens, u = verify_case(3, 7, 50257, 5)
    v = (logits.cuda(), i32(tokens), torch.tensor(u, device="cuda"))
    draft = draft.cuda()
    cases = []
    for seed, new in enumerate(([1, 1], [16, 9])):
        b = dict(new_start=i32(starts(new)), max_new=max(new), **c.kwargs())
        cases.append((rand(seed, (sum(new), 8, HEAD), 2.0).cuda(), b))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step(i):
        q, b = cases[i]
        return (qlin.causal_attention(q, *c.dev, workspace=ws, **b), *qlin.verify_draft(*v, draft=draft if i else None, workspace=ws))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = [step(i) for i in (0, 1)]
        s.synchronize()
        graphs, got = [], []
        for i in (0, 1):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[i], stream=s):
                got.append(step(i))
        for k in range(4):
            for i in (k & 1, 1, 0):
                for t in got[i]:
                    t.zero_()
                graphs[i].replay()
                step(1 - i)
                s.synchronize()
                for x, y in zip(got[i], want[i]):
                    assert torch.equal(x, y)


def test_a_layer_between_quantized_linears():
    """q|k|v of a quantized layer in one launch, norms, rotation and append of their outputs,
    attention, and the o projection on its output: each stage against the oracle on what the
    stage before it left on the device."""
    from oracle import qlin_ref
    from synth import gen
    Hq, Hkv, K, M, L = 8, 2, 512, 16, 140
    ws = [gen.random_case(60 + i, M, K, n * HEAD) for i, n in enumerate((Hq, Hkv, Hkv))]
    o = gen.random_case(70, M, Hq * HEAD, K)
    lins = [qlin.QLinear(w["packed"], w["scales"], w["zeros"]) for w in ws + [o]]
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    x = torch.from_numpy(ws[0]["x"].view(np.int16)).view(torch.bfloat16).cuda()
    c = Cache("heads", [L], Hkv, 3)
    w = (1 + rand(1, (HEAD,), 0.1))
    freq = 1e6 ** (-torch.arange(64, dtype=torch.float64) / 64)
    batch = dict(new_start=i32([0, M]), max_new=M, **c.kwargs())
    need = max(qlin.group_plan(lins[:3], M)[0], qlin.group_plan(lins[3:], M)[0])
    wsb = qlin.new_workspace(need)
    q, k, v = qlin.forward_group(lins[:3], x, workspace=wsb)
    kc, vc = c.dev
    qr = qlin.norm_rope_append(q, k, v, kc, vc, q_norm=w.cuda(), k_norm=w.cuda(), inv_freq=freq.cuda(), **batch)
    att = qlin.causal_attention(qr, kc, vc, **batch)
    y = qlin.forward_group(lins[3:], att.view(M, Hq * HEAD), workspace=wsb)[0]
    torch.cuda.synchronize()
    for got, e in zip((q, k, v), ws):
        assert qlin_ref.compare(bits(got), qlin_ref.forward(ws[0]["x"], e["packed"], e["scales"], e["zeros"]))["ok"]
    for i in range(M):
        for got, src, heads in ((f64(qr[i]), q, Hq), (f64(kc[0, :, L - M + i]), k, Hkv)):
            want = ref.rotate(ref.norm(f64(src[i]).reshape(heads, HEAD), f64(w), 1e-6), L - M + i, freq.numpy(), False)
            assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -17)      # values of size 4 and below
    assert torch.equal(vc[0, :, L - M:L].transpose(0, 1).reshape(M, -1).view(torch.int16), v.view(torch.int16))
    want, A = ref.causal_attention(f64(qr), f64(kc[0, :, :L].transpose(0, 1)), f64(vc[0, :, :L].transpose(0, 1)), HEAD ** -0.5)
    assert np.all(np.abs(f64(att) - want) <= 2.0 ** -7 * (A + np.abs(want)))
    assert qlin_ref.compare(bits(y), qlin_ref.forward(bits(att.view(M, -1)), o["packed"], o["scales"], o["zeros"]))["ok"]
    for l in lins:
        l.close()


def test_prompt_then_blocks_then_tokens_through_one_cache():
    """A prompt, a draft block that is cut back, and single tokens, each appended and
    attended, against the oracle over the cache the device holds; then the same steps as
    one captured graph whose lengths change between replays."""
    Hq, Hkv, cap = 8, 2, 256
    kc, vc = (torch.zeros((2, Hkv, cap, HEAD), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    freq = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).cuda()
    w = (1 + rand(1, (HEAD,), 0.1)).cuda()

    def step(rows, new_start, length, max_new, out_q, out):
        qlin.norm_rope_append(*rows, kc, vc, new_start, length, max_new=max_new, q_norm=w, k_norm=w, inv_freq=freq, out=out_q)
        return qlin.causal_attention(out_q, kc, vc, new_start, length, max_new=max_new, out=out)

    def check(new, length, out_q, out):
        m = 0
        for b, n in enumerate(new):
            want, A = ref.causal_attention(f64(out_q[m:m + n]), f64(kc[b, :, :length[b]].transpose(0, 1)),
                                           f64(vc[b, :, :length[b]].transpose(0, 1)), HEAD ** -0.5)
            # weights and output rounded (2 x 2^-8, see above); scores of 128 fp32 products are far below
            assert np.all(np.abs(f64(out[m:m + n]) - want) <= 2.0 ** -7 * (A + np.abs(want)))
            m += n

    lengths = [0, 0]
    for seed, (new, cut) in enumerate([([100, 37], [0, 0]), ([16, 16], [9, 3]), ([1, 1], [0, 0]), ([16, 5], [16, 0]), ([1, 1], [0, 0])]):
        lengths = [l + n for l, n in zip(lengths, new)]
        M = sum(new)
        rows = [rand(seed * 3 + i, (M, h * HEAD), 1.5).cuda() for i, h in enumerate((Hq, Hkv, Hkv))]
        out_q, out = (torch.zeros((M, Hq, HEAD), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        step(rows, i32(starts(new)), i32(lengths), max(new), out_q, out)
        torch.cuda.synchronize()
        check(new, lengths, out_q, out)
        lengths = [l - c for l, c in zip(lengths, cut)]

    new = [16, 16]
    rows = [torch.zeros((32, h * HEAD), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    new_start, length = i32(starts(new)), i32([16, 16])
    out_q, out = (torch.zeros((32, Hq, HEAD), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    logits = rand(50, (2, 16, 3001), 2.0).cuda()
    drafted, u = i32([[1] * 15] * 2), torch.full((2, 16), 0.5, device="cuda")
    step(rows, new_start, length, 16, out_q, out)
    qlin.verify_draft(logits, drafted, u)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(rows, new_start, length, 16, out_q, out)
        acc, tok = qlin.verify_draft(logits, drafted, u)
    for i, L in enumerate([[60, 200], [16, 17], [256, 100], [90, 255]]):
        for j, r in enumerate(rows):
            r.copy_(rand(100 + 3 * i + j, tuple(r.shape), 1.5))
        length.copy_(i32(L))
        x = rand(200 + i, (2, 16, 3001), 2.0)
        logits.copy_(x)
        best = x[:, :15].float().argmax(2).to(torch.int32)
        drafted.copy_(best)
        graph.replay()
        torch.cuda.synchronize()
        check(new, L, out_q, out)
        for b in range(2):
            a, nxt = ref.verify(f64(x[b]), None, best[b].tolist(), [0.5] * 16, 1.0)
            assert (int(acc[b]), tok[b].tolist()) == (a, best[b, :a].tolist() + [nxt] + [-1] * (15 - a))


def test_python_refusals():
    q, c = rand(0, (4, 512)).cuda(), Cache("heads", [4], 2, 1)
    kv = q[:, :256]
    ok = dict(new_start=i32([0, 4]), length=i32([4]))
    with pytest.raises(ValueError):
        qlin.norm_rope_append(q.float(), kv, kv, *c.dev, **ok)
    with pytest.raises(ValueError):
        qlin.norm_rope_append(q, kv[:, :128], kv, *c.dev, **ok)
    with pytest.raises(ValueError):
        qlin.norm_rope_append(q, kv, kv, *c.dev, new_start=i32([0, 4]).long(), length=i32([4]))
    with pytest.raises(ValueError):
        qlin.norm_rope_append(q, kv, kv, *c.dev, new_start=i32([0, 4]), length=i32([4, 4]))
    with pytest.raises(ValueError):
        qlin.norm_rope_append(q, kv, kv, c.dev[0], c.dev[1].transpose(1, 2), **ok)
    with pytest.raises(ValueError):
        qlin.norm_rope_append(q, kv, kv, *c.dev, inv_freq=torch.ones(64, device="cuda"), **ok)
    q3 = q.view(4, 4, HEAD)
    with pytest.raises(ValueError):
        qlin.causal_attention(q3.cpu(), *c.dev, **ok)
    with pytest.raises(ValueError):
        qlin.causal_attention(q3, *[t.cpu() for t in c.dev], **ok)
    with pytest.raises(ValueError):                                    # two sequences, a cache of one
        qlin.causal_attention(q3, *c.dev, new_start=i32([0, 2, 4]), length=i32([4, 4]))
    with pytest.raises(qlin.QlinError):
        qlin.causal_attention(q3, *c.dev, out=q3, **ok)
    t = rand(0, (2, 3, 50)).cuda()
    x, u = i32([[1, 2], [3, 4]]), torch.rand((2, 3), device="cuda")
    with pytest.raises(ValueError):
        qlin.verify_draft(t, x[:, :1], u)
    with pytest.raises(ValueError):
        qlin.verify_draft(t, x, u.double())
    with pytest.raises(ValueError):
        qlin.verify_draft(t, x, u, draft=t)
    with pytest.raises(ValueError):
        qlin.verify_draft(t.transpose(0, 1).contiguous().transpose(0, 1), x, u)
    with pytest.raises(ValueError):
        qlin.verify_draft(t, x, u, n_draft=torch.zeros(2, device="cuda"))
