"""The operators of the 4-bit paged cache as measurable cases: appending tokens (quantised as they are written) and reading
them back, reading a stretch of the cache back, and attention over it -- single new tokens, drafts, prompt chunks, sliding
windows with first tokens that stay visible -- on ragged batches.

A case is a dict:
  op         "write":  append the new rows, read them back           (a step's or a prompt's K and V, as the cache holds them)
             "read":   read the last `new` rows of every sequence    (a prefix handed to another program)
             "attend": attention of the new rows over the cache      (they are in the cache already)
  batch, kv_heads, q_heads, dim
  tokens     length of the longest sequence, the new rows included
  new        rows of the longest sequence that the call is about
  ragged     sequences of different lengths; ragged_new: of different numbers of new rows
  window     0, or how many tokens back a row sees; sinks: first tokens that stay visible all the same
  dtype      "fp16" or "bf16" of the rows that go in and come out

The cache holds, for every 32 channels of a token and kv-head, a power of two 2^e (e the least integer with the largest
magnitude <= 7 * 2^e, within -23 .. 13) and for every channel the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign.
"""
import math

import torch

own = False

PAGE = 64
GROUP = 32
E_LEAST, E_MOST = -23, 13
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DEVICE = "cuda:0"


def _case(name, op, batch, kv_heads, q_heads, tokens, new=1, dim=128, ragged=False, ragged_new=False, window=0, sinks=0,
          dtype="fp16"):
    c = dict(op=op, batch=batch, kv_heads=kv_heads, q_heads=q_heads, dim=dim, tokens=tokens, new=new, ragged=ragged,
             ragged_new=ragged_new, window=window, sinks=sinks, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one head and a short context with a ragged end: the smallest step, all latency
        _case("attend_1x1_1k", "attend", 1, 1, 1, 1000),
        # interactive decoding of one sequence, 32 heads, just past a page edge
        _case("attend_1x32_4k", "attend", 1, 32, 32, 4100),
        # a small batch with grouped queries, sequences of different lengths up to the usual long context
        _case("attend_4x8x4_32k_ragged", "attend", 4, 8, 32, 32788, ragged=True, dtype="bf16"),
        # a serving batch of a 52-head model at 32 000 tokens: sustained streaming
        _case("attend_8x52_32k", "attend", 8, 52, 52, 32000),
        # one very long document through a window with four first tokens
        _case("window_1x8x4_128k", "attend", 1, 8, 32, 131079, window=4096, sinks=4),
        # drafts of up to five tokens checked at once, heads of 64 in groups of three
        _case("draft_3x10x3_9k_d64", "attend", 3, 10, 30, 8999, new=5, dim=64, ragged=True, ragged_new=True, dtype="bf16"),
        # a chunk of a long prompt against everything before it
        _case("chunk_1x8x4_2k_at_12k", "attend", 1, 8, 32, 14336, new=2048),
        # whole prompts of different lengths in one call, windowed
        _case("prompts_4x8x4_4k_window", "attend", 4, 8, 32, 4097, new=4097, ragged=True, ragged_new=True, window=1000,
              sinks=4, dtype="bf16"),
        # a long context read back for another program
        _case("read_1x8_128k", "read", 1, 8, 32, 131072, new=131072),
        # short prefixes of several sequences read back, heads of 64
        _case("read_4x10_700_d64", "read", 4, 10, 30, 1500, new=700, dim=64, ragged=True, ragged_new=True, dtype="bf16"),
        # a decode step of the serving batch: one token of every sequence
        _case("write_step_8x52", "write", 8, 52, 52, 4095, ragged=True),
        # prompts of several sequences
        _case("write_prompts_4x32_8k", "write", 4, 32, 32, 8190, new=8190, ragged=True, ragged_new=True, dtype="bf16"),
    ]


MOST_ROWS = 8 * 52 * 32000          # (sequence, kv-head, token) of the largest listed cache
MOST_PAIRS = 2048 * 14336 * 32      # (query head row, token) of the largest listed chunk


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["step", "step", "window", "draft", "chunk", "prompts", "read", "write", "write_step"])
    batch = rng.choice([1, 1, 2, 3, 4, 8])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 10, 32, 40, 52])
    group = rng.choice([1, 2, 3, 4, 4, 5, 8, 12, 16]) if kv_heads <= 10 else 1
    q_heads = kv_heads * group
    dim = rng.choice([128, 128, 128, 64])
    dtype = rng.choice(["fp16", "bf16"])
    ragged = batch > 1 and rng.random() < 0.6
    most = min(131072, MOST_ROWS // (batch * kv_heads))
    window, sinks, new = 0, 0, 1
    if kind in ("step", "window"):
        tokens = _log(rng, 1, most)
    elif kind == "draft":
        new = rng.randint(2, 16)
        tokens = _log(rng, new, min(most, MOST_PAIRS // (batch * q_heads * new)))
    elif kind == "chunk":
        new = _log(rng, 17, 2048)
        tokens = _log(rng, new, max(new, min(32768, most, MOST_PAIRS // (batch * q_heads * new))))
    elif kind == "prompts":
        tokens = new = _log(rng, 17, min(5000, most, int(math.sqrt(MOST_PAIRS / (batch * q_heads)))))
    elif kind == "write_step":
        tokens, new = _log(rng, 1, 30000), 1
    else:
        tokens = _log(rng, 20, min(most, 2 * 131072 // (batch * max(1, kv_heads // 8))))
        new = tokens if kind == "write" and rng.random() < 0.7 else _log(rng, 1, tokens)
    if kind == "window" or kind in ("chunk", "prompts") and rng.random() < 0.4:
        window = _log(rng, 1, 8192)
        sinks = rng.choice([0, 1, 4, 4, 16, 100])
    op = "write" if kind.startswith("write") else "read" if kind == "read" else "attend"
    return _case(None, op, batch, kv_heads, q_heads, tokens, new, dim, ragged, ragged and new > 1 and rng.random() < 0.7,
                 window, sinks, dtype)


def _sizes(case):
    """Lengths of the sequences and how many new rows each has."""
    lens, new = [], []
    for b in range(case["batch"]):
        part = 5 * b / (8 * case["batch"]) if case["ragged"] else 0.0
        length = max(1, case["tokens"] - int(part * case["tokens"]) - (b if case["ragged"] else 0))
        n = max(1, case["new"] - int(5 * b * case["new"] / (8 * case["batch"]))) if case["ragged_new"] else case["new"]
        lens.append(length)
        new.append(min(n, length))
    return lens, new


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _rows(gen, n, heads, dim, gain=None):
    """N(0, 1) rows; gain: of each channel."""
    x = torch.empty(n, heads, dim, dtype=torch.float32, device=DEVICE)
    step = max(1, (1 << 28) // (heads * dim))
    for i in range(0, n, step):
        part = torch.randn(min(step, n - i), heads, dim, generator=gen, device=DEVICE)
        x[i:i + step] = part if gain is None else part * gain
    return x


def _inputs(case, seed):
    """K and V rows of every sequence back to back (K with four channels of ten times the size in each kv-head), q rows."""
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(77000 + seed)
    lens, new = _sizes(case)
    H, D = case["kv_heads"], case["dim"]
    gain = torch.ones(H, D, device=DEVICE)
    gain.scatter_(1, torch.rand(H, D, generator=gen, device=DEVICE).argsort(1)[:, :4], 10.0)
    n = sum(new) if case["op"] == "write" else sum(lens)
    k = _rows(gen, n, H, D, gain).to(_type(case))
    v = _rows(gen, n, H, D).to(_type(case))
    q = _rows(gen, sum(new), case["q_heads"], D).to(_type(case)) if case["op"] == "attend" else None
    return k, v, q


# ---- the plain form -----------------------------------------------------------------------------------------------

def _quantise(x):
    """x [n, H, D] -> its codes two to a byte [n, H, D / 2] (the even channel in the low half) and exponents [n, H, D / 32]."""
    n, H, D = x.shape
    codes = torch.empty(n, H, D // 2, dtype=torch.uint8, device=x.device)
    exps = torch.empty(n, H, D // GROUP, dtype=torch.int32, device=x.device)
    step = max(1, (1 << 26) // (H * D))
    for i in range(0, n, step):
        g = x[i:i + step].float().unflatten(2, (D // GROUP, GROUP))
        m, e = torch.frexp(g.abs().amax(3))
        e = torch.where(m <= 0.875, e - 3, e - 2)                    # 7 * 2^e = 0.875 * 2^(e + 3)
        e = torch.where(m == 0, E_LEAST, e).clamp(E_LEAST, E_MOST).to(torch.int32)
        y = torch.ldexp(g, -e[..., None])
        a = y.abs()
        c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
        c = (c | ((y < 0).to(torch.uint8) << 3)).flatten(2)
        codes[i:i + step] = c[..., 0::2] | (c[..., 1::2] << 4)
        exps[i:i + step] = e
    return codes, exps


def _values(codes, exps):
    """What they stand for, fp32."""
    lut = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float32, device=codes.device)
    nibbles = torch.stack((codes & 15, codes >> 4), -1).flatten(2).int()
    x = lut[nibbles].unflatten(2, (-1, GROUP))
    return torch.ldexp(x, exps[..., None]).flatten(2)


def _visible(case, length, n):
    """Positions that some new row sees, and for each new row which of them."""
    pos = torch.arange(length - n, length, device=DEVICE)
    seen = torch.arange(length, device=DEVICE)
    if case["window"]:
        seen = seen[(seen > length - n - case["window"]) | (seen < case["sinks"])]
    ok = seen[None, :] <= pos[:, None]
    if case["window"]:
        ok &= (seen[None, :] > pos[:, None] - case["window"]) | (seen[None, :] < case["sinks"])
    return seen, ok


def _attend_plain(case, state):
    H, G, D = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    out = torch.empty_like(state["q"])
    row = at = 0
    for length, n in zip(*_sizes(case)):
        seen, ok = _visible(case, length, n)
        k, v = (_values(c[at:at + length][seen], e[at:at + length][seen]) for c, e in state["held"])
        q = state["q"][row:row + n].float().unflatten(1, (H, G)).permute(1, 0, 2, 3).reshape(H, n * G, D)
        step = max(1, (1 << 28) // (n * G * len(seen)))
        for h in range(0, H, step):
            s = torch.matmul(q[h:h + step], k[:, h:h + step].permute(1, 2, 0).contiguous()) * state["scale"]
            s = s.unflatten(1, (n, G)).masked_fill(~ok[None, :, None, :], -math.inf)
            s = torch.exp(s - s.amax(-1, keepdim=True))
            s = (s / s.sum(-1, keepdim=True)).flatten(1, 2)
            o = torch.matmul(s, v[:, h:h + step].transpose(0, 1).contiguous())
            out[row:row + n, h * G:(h + step) * G] = (o.unflatten(1, (n, G)).permute(1, 0, 2, 3).flatten(1, 2).to(out.dtype))
        row, at = row + n, at + length
    return out


def _last_rows(case):
    """Index of the last new rows of every sequence among the rows of all."""
    lens, new = _sizes(case)
    ends = torch.tensor(lens).cumsum(0).tolist()
    return torch.cat([torch.arange(e - n, e, device=DEVICE) for e, n in zip(ends, new)])


def _plain(case, state):
    if case["op"] == "attend":
        return _attend_plain(case, state)
    if case["op"] == "write":
        return [_values(*_quantise(x)).to(_type(case)) for x in state["new"]]
    rows = state["rows"]
    return [_values(c[rows], e[rows]).to(_type(case)) for c, e in state["held"]]


# ---- preparation and one pass ---------------------------------------------------------------------------------------

def prepare(case, seed):
    k, v, q = _inputs(case, seed)
    state = dict(case=case, scale=1.0 / math.sqrt(case["dim"]))
    if q is not None:
        state["q"] = q
    if case["op"] == "write":
        state["new"] = (k, v)
    if own:
        return _prepare_own(case, state, k, v, seed)
    if case["op"] != "write":
        state["held"] = [_quantise(x) for x in (k, v)]
    if case["op"] == "read":
        state["rows"] = _last_rows(case)
    return state


def _prepare_own(case, state, k, v, seed):
    from paper_2512_24449_amd import binding
    lens, new = _sizes(case)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=DEVICE)

    def starts(x):
        return ints([sum(x[:i]) for i in range(len(x))])

    # every sequence's pages lie anywhere among the pages of the cache, as after a while of serving
    pages = [-(-n // PAGE) for n in lens]
    order = torch.randperm(sum(pages) + 3, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((case["batch"], max(pages)), -1, dtype=torch.int32)
    for b, n in enumerate(pages):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)])
    table = table.to(DEVICE)
    state["cache"] = cache = binding.FP4KVCache(sum(pages) + 3, case["kv_heads"], case["q_heads"], case["dim"], device=DEVICE)
    if case["op"] != "write":
        cache.kv_fp4_append(k, v, binding.FP4Batch(ints(lens), max(lens), table, new_rows=ints(lens), first_row=starts(lens)))
    state["batch"] = binding.FP4Batch(ints(lens), max(new), table, new_rows=ints(new), first_row=starts(new))
    state["n_rows"] = sum(new)
    return state


def run(state):
    case = state["case"]
    if not own:
        return _plain(case, state)
    cache, batch = state["cache"], state["batch"]
    if case["op"] == "attend":
        return cache.kv_fp4_attention(state["q"], batch, state["scale"], window=case["window"], sinks=case["sinks"])
    if case["op"] == "write":
        cache.kv_fp4_append(*state["new"], batch)
    return list(cache.kv_fp4_read(batch, state["n_rows"], _type(case)))


def _pairs(length, n, window, sinks):
    """(row, token) pairs that are visible, and tokens that some row sees."""
    pairs = 0
    for p in range(length - n, length):
        seen = p + 1
        if window and seen > window:
            seen = window + min(sinks, seen - window)
        pairs += seen
    union = length
    if window:
        first = max(0, length - n - window + 1)
        union = length - first + min(sinks, first)
    return pairs, union


def work(case):
    lens, new = _sizes(case)
    H, Hq, D = case["kv_heads"], case["q_heads"], case["dim"]
    held = H * 2 * (D // 2 + D // GROUP)     # bytes of a token in the cache
    plain = H * 2 * D * 2                    # and of its K and V rows
    if case["op"] == "write":                # rows in, cache out, and back
        return {"bytes": sum(new) * (2 * plain + 2 * held), "flops": 0}
    if case["op"] == "read":
        return {"bytes": sum(new) * (plain + held), "flops": 0}
    pairs = [_pairs(length, n, case["window"], case["sinks"]) for length, n in zip(lens, new)]
    return {"bytes": sum(u for _, u in pairs) * held + 2 * sum(new) * Hq * D * 2, "flops": 4 * D * Hq * sum(p for p, _ in pairs)}


# ---- from the definition, in 64 bits -------------------------------------------------------------------------------

def _exact_values(x):
    g = x.double().unflatten(2, (-1, GROUP))
    top = g.abs().amax(3, keepdim=True)
    e = torch.ceil(torch.log2(top / 7.0)).clamp(E_LEAST, E_MOST)     # (log2(0) is -inf)
    y = g / torch.exp2(e)
    size = y.abs()
    # spacing of the representable values around |y|; round() takes ties to even multiples, which are the even codes
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0)).to(torch.float64)
    near = (torch.round(size / step) * step).clamp(max=6.0) * torch.sign(y)
    return (near * torch.exp2(e)).flatten(2)


def exact(case, seed):
    k, v, q = _inputs(case, seed)
    if case["op"] == "write":
        return [_exact_values(x) for x in (k, v)]
    if case["op"] == "read":
        rows = _last_rows(case)
        return [_exact_values(x[rows]) for x in (k, v)]
    H, G, D = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["dim"]
    result, row, at = [], 0, 0
    for length, n in zip(*_sizes(case)):
        heads = []
        for h in range(H):
            kh, vh = (_exact_values(x[at:at + length, h:h + 1])[:, 0] for x in (k, v))
            blocks = []
            for i in range(0, n, 512):
                qh = q[row + i:min(row + i + 512, row + n), h * G:(h + 1) * G].double()
                p = torch.arange(length - n + i, length - n + i + len(qh), device=DEVICE)[:, None]
                j = torch.arange(length, device=DEVICE)[None, :]
                hidden = j > p
                if case["window"]:
                    hidden |= (p - j >= case["window"]) & (j >= case["sinks"])
                s = (qh.flatten(0, 1) @ kh.T).unflatten(0, (len(qh), G)) / math.sqrt(D)
                s[hidden[:, None, :].expand_as(s)] = -math.inf
                w = torch.softmax(s, -1)
                blocks.append((w.flatten(0, 1) @ vh).unflatten(0, (len(qh), G)))
            heads.append(torch.cat(blocks))
        result.append(torch.cat(heads, 1))
        row, at = row + n, at + length
    return torch.cat(result)
