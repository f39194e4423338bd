"""The target's operators between its linears, at the sizes they are used at.

Three operators of one speculative-decoding loop: the norms and rotation of
queries and keys with the append to the key/value cache (``append``), the causal
attention that reads the cache (``attention``), and the decision on the drafted
tokens (``verify``).  Where ``own`` is true a pass calls the public entry points of
``paper_2607_04244_amd.qlin``; where it is false it computes the same in plain torch
operations.  The head layout is that of the 4B decoder of ``synth/gen.py``: 32
query and 8 key/value heads of dimension 128, a draft block of 16 tokens.

A batch is described by two texts, the new tokens and the cached length (with the
new tokens) of each sequence.  The cache is ``[sequences, heads, capacity, 128]``
or, ``packed``, ``[tokens, heads, 128]`` with one sequence behind the other.
"""

import math

import torch

own = False

HEAD = 128
EPS = 1e-6
THETA = 1e6

# What a drawn case may hold at most: the listed prompt's products, and the
# plain form's padded scores.
MOST_SCORES = 32 * 8192 * 8192


def _text(values):
    return ",".join(str(v) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def _spread(count, low, high):
    """``count`` lengths between low and high, odd ones among them, in mixed order."""
    return [low + (high - low) * ((7 * i + 3) % count) // max(count - 1, 1) for i in range(count)]


def _append(name, new, length, capacity=0, Hq=32, Hkv=8, pad=0, norm=True, rotary=HEAD, interleaved=False):
    return dict(name=name, kind="append", Hq=Hq, Hkv=Hkv, new=_text(new), length=_text(length), capacity=capacity,
                pad=pad, norm=norm, rotary=rotary, interleaved=interleaved)


def _attend(name, new, length, capacity=0, Hq=32, Hkv=8):
    return dict(name=name, kind="attention", Hq=Hq, Hkv=Hkv, new=_text(new), length=_text(length), capacity=capacity)


def listed():
    prompts = [1537, 64, 803, 2048, 1, 1290, 333, 912]
    return [
        # Plain decoding of one sequence: one token's heads, the smallest call.
        _append("append_one", [1], [4097], capacity=8448),
        # Verification of 16-token draft blocks of a batch of requests, padded
        # to a fixed number of rows for a captured step.
        _append("append_blocks", [16] * 23, _spread(23, 40, 2000), capacity=2048, pad=16),
        # A long prompt in one chunk, keys and values packed as they come.
        _append("append_prompt", [8192], [8192]),
        # Plain decoding of one sequence with a long context.
        _attend("decode_one", [1], [8191], capacity=8448),
        # Verification of one 16-token draft block, the loop's own call.
        _attend("verify_block", [16], [8192], capacity=8448),
        # Plain decoding of a batch of requests of many lengths: bound by the
        # key/value cache that has to be read.
        _attend("decode_batch", [1] * 64, _spread(64, 130, 8190), capacity=8448),
        # Prompts of different lengths packed into one call.
        _attend("prompts_packed", prompts, prompts),
        # A chunk of a prompt behind a cached prefix.
        _attend("prompt_chunk", [500], [7900], capacity=8448),
        # The longest prompt in one call: the largest product.
        _attend("prompt_long", [8192], [8192]),
        # The decision on one block of a drafter that proposes its most likely
        # tokens: no draft probabilities.
        dict(name="verify_one", kind="verify", B=1, n=15, V=151936, drafts=False, greedy=False, ragged=False),
        # A batch of requests against a sampling drafter.
        dict(name="verify_batch", kind="verify", B=32, n=15, V=151936, drafts=True, greedy=False, ragged=False),
        # Short blocks of different lengths, greedy requests among them, an odd
        # vocabulary.
        dict(name="verify_odd", kind="verify", B=7, n=5, V=50257, drafts=True, greedy=True, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_batch(rng):
    """(new, length, capacity, Hq, Hkv) of a batch within the listed costs."""
    Hkv, G = rng.choice((1, 2, 4, 8, 8)), rng.choice((1, 2, 3, 4, 4, 5, 7, 8))
    use = rng.choice(("decode", "block", "prompts", "chunk"))
    if use == "decode":
        B, longest = _log_int(rng, 1, 96), _log_int(rng, 64, 8192)
        length = [rng.randint(1, longest) for _ in range(B)]
        return [1] * B, length, longest + rng.randint(0, 256), Hkv * G, Hkv
    if use == "block":
        B, longest = _log_int(rng, 1, 24), _log_int(rng, 64, 8192)
        new = [rng.randint(2, 16) for _ in range(B)]
        return new, [max(n, rng.randint(16, longest)) for n in new], longest + rng.randint(0, 256), Hkv * G, Hkv
    if use == "prompts":
        new = [_log_int(rng, 1, 4096) for _ in range(rng.randint(1, 6))]
        return new, new, 0, Hkv * G, Hkv
    B, longest = rng.randint(1, 3), _log_int(rng, 512, 8192)
    new = [rng.randint(17, 512) for _ in range(B)]
    return new, [rng.randint(n, max(n, longest)) for n in new], max(longest, 512) + rng.randint(0, 256), Hkv * G, Hkv


def draw(rng):
    kind = rng.choice(("append", "attention", "attention", "verify"))
    if kind == "verify":
        drafts = rng.random() < 0.6
        return dict(kind=kind, B=_log_int(rng, 1, 24), n=rng.randint(1, 15), V=_log_int(rng, 4000, 151936), drafts=drafts,
                    greedy=rng.random() < 0.4, ragged=rng.random() < 0.5)
    new, length, capacity, Hq, Hkv = _draw_batch(rng)
    while Hq * len(new) * max(new) * max(length) > MOST_SCORES:
        Hq //= 2
        Hkv = math.gcd(Hq, Hkv)
    case = dict(kind=kind, Hq=Hq, Hkv=Hkv, new=_text(new), length=_text(length), capacity=capacity)
    if kind == "append":
        case.update(pad=rng.choice((0, 0, 5, 16)), norm=rng.random() < 0.7, rotary=rng.choice((128, 128, 64, 32)),
                    interleaved=rng.random() < 0.3)
    return case


# ---------------------------------------------------------------- inputs


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, sigma=1.0):
    return (sigma * torch.randn(shape, device="cuda", generator=g)).to(torch.bfloat16)


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _batch(case):
    """What a program holds of a batch: the device arrays and the host's bounds."""
    new, length = _ints(case["new"]), _ints(case["length"])
    start = None if case["capacity"] else torch.tensor(_starts(length)[:-1], dtype=torch.int64, device="cuda")
    return dict(new_start=torch.tensor(_starts(new), dtype=torch.int32, device="cuda"),
                length=torch.tensor(length, dtype=torch.int32, device="cuda"), cache_start=start, max_new=max(new),
                max_len=max(length))


def _cache(g, case):
    length = _ints(case["length"])
    shape = (len(length), case["Hkv"], case["capacity"], HEAD) if case["capacity"] else (sum(length), case["Hkv"], HEAD)
    return _normal(g, shape), _normal(g, shape)


def _inputs(case, seed):
    g = _generator(seed)
    if case["kind"] == "append":
        rows = sum(_ints(case["new"])) + case["pad"]
        q, k, v = (_normal(g, (rows, h * HEAD), 1.5) for h in (case["Hq"], case["Hkv"], case["Hkv"]))
        wq, wk = ((1.0 + 0.2 * torch.randn(HEAD, device="cuda", generator=g)).to(torch.bfloat16) for _ in range(2))
        half = case["rotary"] // 2
        freq = THETA ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        kc, vc = _cache(g, case)
        out = _normal(g, (rows, case["Hq"], HEAD))
        return dict(q=q, k=k, v=v, wq=wq if case["norm"] else None, wk=wk if case["norm"] else None, freq=freq, kc=kc,
                    vc=vc, out=out)
    if case["kind"] == "attention":
        q = _normal(g, (sum(_ints(case["new"])), case["Hq"], HEAD), 2.0)
        kc, vc = _cache(g, case)
        return dict(q=q, kc=kc, vc=vc)
    B, n, V = case["B"], case["n"], case["V"]
    target = _normal(g, (B, n + 1, V), 2.5)
    # a drafter that is near its target: its tokens are often kept
    draft = (target[:, :n].float() + 0.4 * torch.randn((B, n, V), device="cuda", generator=g)).to(torch.bfloat16)
    at = draft.float()
    if case["drafts"]:
        noise = torch.empty((B, n, V), device="cuda").exponential_(generator=g)
        at = at - noise.clamp_min(1e-30).log()
    drafted = at.argmax(2).to(torch.int32)
    u = torch.rand((B, n + 1), device="cuda", generator=g)
    temperature = 0.7 + 0.5 * torch.rand(B, device="cuda", generator=g)
    if case["greedy"]:
        temperature[::2] = 0.0
    return dict(target=target, draft=draft if case["drafts"] else None, drafted=drafted, u=u, temperature=temperature)


def _n_draft(case):
    return [max(0, case["n"] - (b % 3 if case["ragged"] else 0)) for b in range(case["B"])]


def prepare(case, seed):
    state = dict(case, **_inputs(case, seed))
    if case["kind"] == "verify":
        state["n_draft"] = torch.tensor(_n_draft(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
    else:
        state.update(batch=_batch(case), rows=sum(_ints(case["new"])))
    return state


# ---------------------------------------------------------------- one pass


def run(state):
    if own:
        return _run_own(state)
    if state["kind"] == "append":
        return _plain_append(state)
    if state["kind"] == "attention":
        return _plain_attention(state)
    return _plain_verify(state)


def _run_own(state):
    from paper_2607_04244_amd import qlin
    if state["kind"] == "append":
        out = qlin.norm_rope_append(state["q"], state["k"], state["v"], state["kc"], state["vc"], **state["batch"],
                                    q_norm=state["wq"], k_norm=state["wk"], eps=EPS, inv_freq=state["freq"],
                                    interleaved=state["interleaved"], out=state["out"])
        return out, state["kc"], state["vc"]
    if state["kind"] == "attention":
        return qlin.causal_attention(state["q"], state["kc"], state["vc"], **state["batch"])
    return qlin.verify_draft(state["target"], state["drafted"], state["u"], draft=state["draft"],
                             n_draft=state["n_draft"], temperature=state["temperature"])


def _rows(batch, rows):
    """(sequence, index in it, position) of each row."""
    m = torch.arange(rows, device="cuda")
    b = torch.searchsorted(batch["new_start"][1:].contiguous(), m, right=True)
    i = m - batch["new_start"][b]
    new = batch["new_start"][b + 1] - batch["new_start"][b]
    return b, i, batch["length"][b] - new + i


def _norm(x, w):
    if w is None:
        return x
    return x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * w.float()


def _rotate(x, cos, sin, interleaved):
    half = cos.shape[2]
    r, rest = x[:, :, :2 * half], x[:, :, 2 * half:]
    if interleaved:
        a, b = r[:, :, 0::2], r[:, :, 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), 3).flatten(2)
    else:
        a, b = r[:, :, :half], r[:, :, half:]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), 2)
    return torch.cat((turned, rest), 2).to(torch.bfloat16)


def _plain_append(state):
    n, batch = state["rows"], state["batch"]
    b, _, position = _rows(batch, n)
    angle = position.double()[:, None] * state["freq"][None]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q, k, v = (state[s][:n].view(n, -1, HEAD) for s in "qkv")
    state["out"][:n] = _rotate(_norm(q.float(), state["wq"]), cos, sin, state["interleaved"])
    k = _rotate(_norm(k.float(), state["wk"]), cos, sin, state["interleaved"])
    if state["capacity"]:
        state["kc"][b, :, position] = k
        state["vc"][b, :, position] = v
    else:
        slot = batch["cache_start"][b] + position
        state["kc"][slot] = k
        state["vc"][slot] = v
    return state["out"], state["kc"], state["vc"]


def _keys(state, cache):
    """[sequences, heads, longest, 128] in 32 bits."""
    L = state["batch"]["max_len"]
    if state["capacity"]:
        return cache[:, :, :L].float()
    at = state["batch"]["cache_start"][:, None] + torch.arange(L, device="cuda")
    return cache[at.clamp_max(cache.shape[0] - 1)].permute(0, 2, 1, 3).float().contiguous()


def _plain_attention(state):
    batch, q = state["batch"], state["q"]
    M, Hq, Hkv = state["rows"], state["Hq"], state["Hkv"]
    G, B, N, L = Hq // Hkv, batch["length"].shape[0], batch["max_new"], batch["max_len"]
    start, length = batch["new_start"].long(), batch["length"].long()
    i = torch.arange(N, device="cuda")
    at = (start[:-1, None] + i).clamp_max(M - 1)
    rows = q[at].view(B, N, Hkv, G, HEAD).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, HEAD).float()
    s = torch.matmul(rows, _keys(state, state["kc"]).transpose(2, 3).contiguous()).view(B, Hkv, G, N, L)
    position = (length - (start[1:] - start[:-1]))[:, None] + i
    hidden = torch.arange(L, device="cuda") > position[:, :, None]
    s = (s / math.sqrt(HEAD)).masked_fill_(hidden[:, None, None], -math.inf)
    s = torch.exp(s - s.amax(4, keepdim=True).clamp_min(-3e38))
    total = s.sum(4)[..., None]
    o = torch.matmul(s.view(B, Hkv, G * N, L), _keys(state, state["vc"])).view(B, Hkv, G, N, HEAD)
    o = torch.where(total > 0, o / total, 0.0)
    b, i, _ = _rows(batch, M)
    return o[b, :, :, i].reshape(M, Hq, HEAD).to(torch.bfloat16)


def _softmax64(logits, temperature):
    """Probabilities in 64 bits; temperature 0 is the lowest index of the largest."""
    x = logits.double()
    t = temperature.double()[:, None, None]
    e = torch.exp((x - x.amax(2, keepdim=True)) / torch.where(t > 0, t, 1.0))
    top = torch.zeros_like(e).scatter_(2, logits.float().argmax(2, keepdim=True), 1.0)
    return torch.where(t > 0, e / e.sum(2, keepdim=True), top)


def _plain_verify(state):
    B, n = state["B"], state["n"]
    u, t, drafted = state["u"].double(), state["temperature"], state["drafted"]
    x = drafted.long()[:, :, None]
    p = _softmax64(state["target"], t)
    q = torch.zeros_like(p[:, :n]).scatter_(2, x, 1.0)
    if state["draft"] is not None:
        q = torch.where(t[:, None, None] > 0, _softmax64(state["draft"], t), q)
    keep = u[:, :n] * q.gather(2, x)[:, :, 0] < p[:, :n].gather(2, x)[:, :, 0]
    count = torch.full((B,), n, device="cuda") if state["n_draft"] is None else state["n_draft"].long()
    i = torch.arange(n, device="cuda")
    keep = keep & (i < count[:, None])
    kept = keep.long().cumprod(1).sum(1)
    seq = torch.arange(B, device="cuda")
    w = p[seq, kept]
    rest = (w - torch.where((kept < count)[:, None], q[seq, kept.clamp_max(n - 1)], 0.0)).clamp_min(0.0)
    w = torch.where(rest.sum(1, keepdim=True) > 0, rest, w)
    run_sum = w.cumsum(1)
    last = (w > 0).long().cumsum(1).argmax(1)
    after = run_sum > u[:, n:] * run_sum[:, -1:]
    chosen = torch.where(after.any(1), after.to(torch.int32).argmax(1), last)
    tokens = torch.full((B, n + 1), -1, dtype=torch.int32, device="cuda")
    tokens[:, :n] = torch.where(i < kept[:, None], drafted, -1)
    return kept.to(torch.int32), tokens.scatter(1, kept[:, None], chosen.to(torch.int32)[:, None])


# ---------------------------------------------------------------- work


def work(case):
    if case["kind"] == "verify":
        drafts = _n_draft(case)
        rows = sum(n + 1 for n in drafts) + (sum(drafts) if case["drafts"] else 0)
        return {"bytes": 2 * case["V"] * rows + 8 * case["B"] * (2 * case["n"] + 1), "flops": 4 * case["V"] * rows}
    new, length, Hq, Hkv = _ints(case["new"]), _ints(case["length"]), case["Hq"], case["Hkv"]
    rows = sum(new)
    if case["kind"] == "append":
        return {"bytes": 2 * HEAD * rows * (2 * Hq + 4 * Hkv), "flops": 8 * HEAD * rows * (Hq + Hkv)}
    keys = sum(t for n, t in zip(new, length) if n)
    pairs = sum(n * t - n * (n - 1) // 2 for n, t in zip(new, length))
    return {"bytes": 2 * HEAD * (2 * Hkv * keys + 2 * Hq * rows), "flops": 4 * HEAD * Hq * pairs}


# ---------------------------------------------------------------- the same in 64 bits


def _exact_heads(x, w, positions, freq, interleaved):
    """Heads [rows, heads, 128] normalised and rotated, as complex numbers."""
    x = x.double().clone()
    if w is not None:
        x = x / (x.square().sum(2, keepdim=True) / HEAD + EPS).sqrt() * w.double()
    half = freq.numel()
    if interleaved:
        first, second = range(0, 2 * half, 2), range(1, 2 * half, 2)
    else:
        first, second = range(half), range(half, 2 * half)
    pair = torch.complex(x[:, :, list(first)], x[:, :, list(second)])
    turn = torch.polar(torch.ones(len(positions), half, dtype=torch.float64, device="cuda"),
                       torch.outer(positions.double(), freq))
    pair = pair * turn[:, None]
    x[:, :, list(first)], x[:, :, list(second)] = pair.real, pair.imag
    return x


def _exact_append(case, d):
    out, kc, vc = d["out"].double(), d["kc"].double(), d["vc"].double()
    m, slot = 0, 0
    for b, (n, t) in enumerate(zip(_ints(case["new"]), _ints(case["length"]))):
        at = torch.arange(t - n, t, device="cuda")
        q, k, v = (d[s][m:m + n].view(n, -1, HEAD) for s in "qkv")
        out[m:m + n] = _exact_heads(q, d["wq"], at, d["freq"], case["interleaved"])
        k = _exact_heads(k, d["wk"], at, d["freq"], case["interleaved"])
        if case["capacity"]:
            kc[b, :, t - n:t] = k.transpose(0, 1)
            vc[b, :, t - n:t] = v.double().transpose(0, 1)
        else:
            kc[slot + t - n:slot + t] = k
            vc[slot + t - n:slot + t] = v.double()
        m, slot = m + n, slot + t
    return out, kc, vc


def _exact_attention(case, d):
    parts, m, slot = [], 0, 0
    G = case["Hq"] // case["Hkv"]
    for b, (n, t) in enumerate(zip(_ints(case["new"]), _ints(case["length"]))):
        future = torch.ones((n, t), dtype=torch.bool, device="cuda").triu(t - n + 1)
        heads = []
        for h in range(case["Hq"]):
            if case["capacity"]:
                k, v = (d[s][b, h // G, :t].double() for s in ("kc", "vc"))
            else:
                k, v = (d[s][slot:slot + t, h // G].double() for s in ("kc", "vc"))
            s = d["q"][m:m + n, h].double() @ k.t().contiguous() * HEAD ** -0.5
            heads.append(torch.softmax(s.masked_fill(future, -math.inf), 1) @ v)
        parts.append(torch.stack(heads, 1))
        m, slot = m + n, slot + t
    return torch.cat(parts)


def _exact_verify(case, d):
    n = case["n"]
    kept = torch.zeros(case["B"], dtype=torch.int32)
    tokens = torch.full((case["B"], n + 1), -1, dtype=torch.int32)
    for b, count in enumerate(_n_draft(case)):
        t = float(d["temperature"][b])
        u, x = d["u"][b].double().tolist(), d["drafted"][b].tolist()

        def probabilities(logits):
            if t == 0:
                p = torch.zeros(case["V"], dtype=torch.float64, device="cuda")
                p[int((logits == logits.max()).nonzero()[0])] = 1.0
                return p
            return torch.softmax(logits.double() / t, 0)

        a, w = 0, None
        while a < count:
            p = probabilities(d["target"][b, a])
            if d["draft"] is not None and t > 0:
                q = probabilities(d["draft"][b, a])
            else:
                q = torch.zeros_like(p)
                q[x[a]] = 1.0
            if not u[a] * float(q[x[a]]) < float(p[x[a]]):
                w = (p - q).clamp_min(0.0)
                w = w if float(w.sum()) > 0 else p
                break
            tokens[b, a] = x[a]
            a += 1
        if w is None:
            w = probabilities(d["target"][b, a])
        total = w.cumsum(0)
        over = (total > u[n] * total[-1]).nonzero()
        tokens[b, a] = int(over[0]) if len(over) else int((w > 0).nonzero()[-1])
        kept[b] = a
    return kept.cuda(), tokens.cuda()


def exact(case, seed):
    d = _inputs(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "verify": _exact_verify}[case["kind"]](case, d)
