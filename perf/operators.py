"""Timed cases of the operators around a bounded key/value cache, and each operator's plain form.

  rotary    positions with several axes turn the channel pairs of queries and keys: forward and backward pass
  append    the same for new tokens in serving: turned queries out, turned keys and values into the pages of the cache
  decode    the newest rows of every sequence attend to the paged cache, and each cached key adds up the weight it gets
  chunk     the weight that a chunk of prompt rows gives to each cached key, from the rows' saved log-sum-exp
  evict     the keys of most accumulated weight move to fresh pages, the others are left behind

`own` says what run() does: False, plain torch operations in fp32, rounded once at the end; True, the calls of
`paper_2511_02043_amd.functional`.  Layouts are those of that module: q [B, H, T, D], caches [pages, page_size, Hkv, D],
int32 lengths and block tables, fp32 weights [B, Hkv, capacity].
"""
import numpy as np
import torch

own = False

DEVICE = "cuda:0"
_MOST_FLOPS = 2.8e11                  # no drawn case costs more than the largest listed one,
_MOST_BYTES = 1.7e9                   # ... moves more than the listed decode batch,
_MOST_SCORES = 2.2e9                  # ... nor has more scores than the listed prompt


def listed():
    return [
        # a training step of a decoder layer on video: text, then frames of 16 x 16 patches, three axes over D = 128
        dict(name="rotary_train_video", kind="rotary", dtype="bf16", B=2, S=8192, H=32, Hkv=8, D=128, sections="16,24,24", interleaved=False),
        # fp32 training on a small image of odd size, neighbouring channels paired, a quarter of the channels not turned
        dict(name="rotary_train_f32", kind="rotary", dtype="f32", B=1, S=333, H=8, Hkv=8, D=64, sections="12,12", interleaved=True),
        # the token being generated, a full serving batch: bound by latency
        dict(name="append_token", kind="append", B=64, T=1, H=32, Hkv=8, D=128, page=16, lo=1024, hi=4096, sections="16,24,24", interleaved=False),
        # a chunk of prompt tokens per sequence enters the cache
        dict(name="append_chunk", kind="append", B=8, T=512, H=32, Hkv=8, D=128, page=16, lo=512, hi=4096, sections="64", interleaved=False),
        # one decode step of a full serving batch over long caches
        dict(name="decode_batch", kind="decode", variant="plain", B=64, T=1, H=32, Hkv=8, D=128, lo=4096, hi=8192, page=16),
        # one decode step of a single short conversation: latency
        dict(name="decode_single", kind="decode", variant="plain", B=1, T=1, H=32, Hkv=8, D=64, lo=1500, hi=2000, page=16),
        # a speculative step: four rows verified at once, soft-capped scores
        dict(name="decode_speculative", kind="decode", variant="softcap", B=16, T=4, H=32, Hkv=8, D=128, lo=2048, hi=4096, page=16),
        # a chunk of prompt rows per sequence over what is cached (chunked prefill)
        dict(name="chunk_512", kind="chunk", variant="plain", B=8, Sq=512, H=32, Hkv=8, D=128, lo=4096, hi=8192, page=16),
        # a whole long prompt at once
        dict(name="chunk_prompt", kind="chunk", variant="plain", B=1, Sq=8192, H=32, Hkv=8, D=128, lo=8192, hi=8192, page=16),
        # long prompts cut to a small budget before decoding starts
        dict(name="evict_prompt", kind="evict", B=8, Hkv=8, D=128, lo=16384, hi=32768, page=16, budget=2048, sinks=4, recent=256),
        # a serving batch back to its budget after some tokens of decoding
        dict(name="evict_batch", kind="evict", B=64, Hkv=8, D=128, lo=2049, hi=2304, page=16, budget=2048, sinks=4, recent=512),
        # one short conversation of a small model
        dict(name="evict_small", kind="evict", B=1, Hkv=8, D=64, lo=500, hi=700, page=16, budget=255, sinks=1, recent=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and _scores(case) <= _MOST_SCORES:
            return case


_SECTIONS = {32: ["16", "8,8", "4,6,6"], 64: ["32", "16,16", "8,12,12", "12,12"], 80: ["40", "20,20"], 128: ["64", "32,32", "16,24,24", "32"]}


def _draw(rng):
    kind = rng.choice(["rotary", "rotary", "append", "decode", "decode", "chunk", "chunk", "evict", "evict"])
    H, Hkv = rng.choice([(8, 8), (16, 16), (16, 2), (32, 8)])
    if kind == "rotary":
        dtype, D = rng.choice(["bf16", "bf16", "f32"]), rng.choice([32, 64, 80, 128])
        S = _log_int(rng, 1, 1024 if dtype == "f32" else 16384)
        return dict(kind=kind, dtype=dtype, B=_log_int(rng, 1, max(1, 16384 // S)), S=S, H=H, Hkv=Hkv, D=D,
                    sections=rng.choice(_SECTIONS[D]), interleaved=rng.choice([False, True]))
    D, page = rng.choice([64, 128]), rng.choice([16, 16, 32, 64])
    if kind == "append":
        T = rng.choice([1, _log_int(rng, 1, 1024)])
        hi = _log_int(rng, max(T, 64), 4096)
        return dict(kind=kind, B=_log_int(rng, 1, 64 if T <= 64 else 8), T=T, H=H, Hkv=Hkv, D=D, page=page, lo=max(1, hi // 2), hi=hi,
                    sections=rng.choice(_SECTIONS[D]), interleaved=rng.choice([False, True]))
    variant = rng.choice(["plain", "plain", "softcap", "alibi", "window"])
    if kind == "decode":
        hi = _log_int(rng, 64, 32768)
        return dict(kind=kind, variant=variant, B=_log_int(rng, 1, 64), T=rng.choice([1, 1, 1, 2, 4]), H=H, Hkv=Hkv, D=D, lo=max(1, hi // 2),
                    hi=hi, page=page)
    if kind == "chunk":
        Sq = _log_int(rng, 16, 4096)
        hi = _log_int(rng, Sq, 16384)
        return dict(kind=kind, variant=variant, B=_log_int(rng, 1, 8), Sq=Sq, H=H, Hkv=Hkv, D=D, lo=max(1, hi // 2), hi=hi, page=page)
    hi = _log_int(rng, 64, 65536)
    budget = _log_int(rng, 16, hi)
    return dict(kind="evict", B=_log_int(rng, 1, 64), Hkv=Hkv, D=D, lo=max(1, hi // 2), hi=hi, page=page, budget=budget,
                sinks=min(4, budget // 8), recent=budget // rng.choice([4, 8, 16]))


# ---- inputs -----------------------------------------------------------------------------------------------------------

_CAP, _WINDOW, _BASE, _GRID = 30.0, 512, 10000.0, 16


def _normal(gen, *shape, dtype=torch.bfloat16):
    """N(0, 1), drawn in fp32 and rounded to the storage type."""
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)


def _sections(case):
    return tuple(int(n) for n in case["sections"].split(","))


def _inv_freq(case):
    """One frequency per channel pair, falling from 1 to 1 / base over all axes."""
    n = sum(_sections(case))
    return (_BASE ** (-torch.arange(n, dtype=torch.float64) / n)).to(DEVICE, torch.float32)


def _positions(case, first, tokens):
    """int32 [B, tokens, axes]: one axis counts tokens; several hold an eighth of text, where all axes count alike, then
    frames of 16 x 16 patches (three axes: frame, row, column; two: row, column).  first: each sequence's first position."""
    axes, n = len(_sections(case)), torch.arange(tokens, device=DEVICE)
    text = tokens // 8
    patch = (n - text).clamp(min=0)
    grid = torch.stack([patch // _GRID ** 2, patch // _GRID % _GRID, patch % _GRID])[3 - axes:] if axes > 1 else patch[None]
    p = torch.where(n < text, n, text + grid)
    return (first[:, None, None] + p.t()[None]).to(torch.int32).contiguous()


def _cache(case, seed, gen, extra=0):
    """Lengths, a pool of pages handed out in arbitrary order, as a serving system's allocator does, and block tables;
    `extra` more pages per sequence come as a second table."""
    B, Hkv, D, page = (case[n] for n in ("B", "Hkv", "D", "page"))
    rng = np.random.default_rng(seed)
    lens = rng.integers(case["lo"], case["hi"] + 1, size=B).astype(np.int32)
    per = -(-case["hi"] // page)
    tables = rng.permutation(B * (per + extra)).astype(np.int32).reshape(B, per + extra)
    k_cache, v_cache = (_normal(gen, B * (per + extra), page, Hkv, D) for _ in range(2))
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEVICE)
    return dict(k_cache=k_cache, v_cache=v_cache, lens=up(lens), table=up(tables[:, :per]), spare=up(tables[:, per:]), max_len=case["hi"])


def _accumulated(gen, *shape):
    """Attention weight summed over some rows: positive, over several decades, some keys never looked at."""
    x = torch.exp(2.0 * torch.randn(shape, generator=gen, device=DEVICE) - 5.0)
    return torch.where(torch.rand(shape, generator=gen, device=DEVICE) < 0.02, torch.zeros_like(x), x)


def _variant(case):
    H, variant = case["H"], case["variant"]
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=DEVICE)
    return dict(softcap=_CAP if variant == "softcap" else None, alibi_slopes=slopes if variant == "alibi" else None,
                window=_WINDOW if variant == "window" else None)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, rng = case["kind"], np.random.default_rng(seed)
    if kind in ("rotary", "append"):
        B, H, Hkv, D = (case[n] for n in ("B", "H", "Hkv", "D"))
        S = case["S"] if kind == "rotary" else case["T"]
        dtype = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
        proj = _normal(gen, B, S, H + 2 * Hkv, D, dtype=dtype).transpose(1, 2)      # one projection: [B, S, heads, D] in memory
        q, k, v = proj[:, :H], proj[:, H:H + Hkv], proj[:, H + Hkv:]
        state = dict(inv_freq=_inv_freq(case), sections=_sections(case), interleaved=case["interleaved"])
    if kind == "rotary":
        first = torch.from_numpy(rng.integers(0, 64, size=B)).to(DEVICE)
        state.update(q=q.detach().requires_grad_(True), k=k.detach().requires_grad_(True), positions=_positions(case, first, S),
                     dq=_normal(gen, B, H, S, D, dtype=dtype), dk=_normal(gen, B, Hkv, S, D, dtype=dtype))
    elif kind == "append":
        state.update(_cache(case, seed, gen))
        # positions go on where the sequence is, whatever was evicted before
        first = state["lens"].long() - S + torch.from_numpy(rng.integers(S, 4096 + S, size=B)).to(DEVICE)
        state.update(q=q, k=k, v=v, positions=_positions(case, first, S))
    elif kind == "evict":
        state = _cache(case, seed, gen, extra=-(-case["budget"] // case["page"]))
        state.update(weights=_accumulated(gen, case["B"], case["Hkv"], case["hi"]), budget=case["budget"], sinks=case["sinks"], recent=case["recent"])
    else:
        state = _cache(case, seed, gen)
        rows = case["T"] if kind == "decode" else case["Sq"]
        state.update(q=_normal(gen, case["B"], case["H"], rows, case["D"]), weights=_accumulated(gen, case["B"], case["Hkv"], case["hi"]),
                     scale=case["D"] ** -0.5, **_variant(case))
        if kind == "chunk":                        # what the chunk's own attention has left behind
            state["lse"] = torch.logsumexp(_plain_scores(state), -1).reshape(state["q"].shape[:3])
    state["kind"] = kind
    return state


# ---- one pass: plain forms ----------------------------------------------------------------------------------------------

def _plain_turn(x, positions, inv_freq, sections, interleaved, back):
    """Each pair (a, b) of channels becomes (a cos - b sin, b cos + a sin) at the angle position * frequency of its axis
    (back: at the negative angle); channels beyond the pairs stay."""
    n = inv_freq.numel()
    axis = torch.repeat_interleave(torch.arange(len(sections), device=x.device), torch.tensor(sections, device=x.device))
    angle = (positions[:, :, axis].float() * inv_freq)[:, None]                     # [B, 1, S, pairs]
    cos, sin = torch.cos(angle), torch.sin(angle) * (-1.0 if back else 1.0)
    y = x.detach().float()
    if interleaved:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., 2 * n:]], -1).to(x.dtype)


def _plain_rotary(s):
    how = (s["positions"], s["inv_freq"], s["sections"], s["interleaved"])
    return (_plain_turn(s["q"], *how, False), _plain_turn(s["k"], *how, False), _plain_turn(s["dq"], *how, True), _plain_turn(s["dk"], *how, True))


def _plain_append(s):
    how = (s["positions"], s["inv_freq"], s["sections"], s["interleaved"], False)
    q, k = _plain_turn(s["q"], *how), _plain_turn(s["k"], *how)
    T, page = q.shape[2], s["k_cache"].shape[1]
    slot = s["lens"].long()[:, None] - T + torch.arange(T, device=q.device)         # [B, T]; below 0: not a token of the sequence
    b, t = torch.nonzero(slot >= 0, as_tuple=True)
    at = slot[b, t]
    pages = s["table"].long()[b, at // page]
    s["k_cache"][pages, at % page] = k[b, :, t]
    s["v_cache"][pages, at % page] = s["v"][b, :, t]
    return q, s["k_cache"], s["v_cache"]


def _gathered(cache, table, max_len):
    """[B, Hkv, max_len, D] rows of a paged cache in fp32."""
    B, Hkv, D = table.shape[0], cache.shape[2], cache.shape[3]
    return cache[table.long()].reshape(B, -1, Hkv, D)[:, :max_len].transpose(1, 2).float()


def _plain_scores(s):
    """Masked scores [B, Hkv, group * rows, max_len] of the newest rows, -inf where hidden."""
    q, lens = s["q"], s["lens"].long()
    B, H, T, D = q.shape
    k = _gathered(s["k_cache"], s["table"], s["max_len"])
    Hkv, L = k.shape[1], k.shape[2]
    x = torch.matmul(q.float().reshape(B, Hkv, -1, D), k.transpose(2, 3)).mul_(s["scale"])
    if s["softcap"] is not None:
        x = torch.tanh(x.div_(s["softcap"])).mul_(s["softcap"])
    x = x.view(B, Hkv, H // Hkv, T, L)
    pos = (lens[:, None] - T + torch.arange(T, device=q.device)).view(B, 1, 1, T, 1)
    j = torch.arange(L, device=q.device)
    if s["alibi_slopes"] is not None:
        x -= s["alibi_slopes"].view(1, Hkv, -1, 1, 1) * (pos - j).float()
    hidden = j > pos
    if s["window"] is not None:
        hidden = hidden | (j < pos - s["window"])
    return x.masked_fill_(hidden, float("-inf")).view(B, Hkv, -1, L)


def _plain_gain(s, rows, gained):
    """Weights of the keys: those of the newest `rows` tokens start here, older ones grow, slots past the length stay."""
    w, lens = s["weights"], s["lens"].long()[:, None, None]
    j = torch.arange(s["max_len"], device=w.device)
    old = torch.where(j < lens - rows, w[..., :s["max_len"]], torch.zeros_like(gained))
    w[..., :s["max_len"]] = torch.where(j < lens, old + gained, w[..., :s["max_len"]])
    return w


def _plain_decode(s):
    q = s["q"]
    x = _plain_scores(s)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    out = torch.matmul(p, _gathered(s["v_cache"], s["table"], s["max_len"]))
    return out.reshape(q.shape).to(q.dtype), _plain_gain(s, q.shape[2], p.sum(2))


def _plain_chunk(s):
    q = s["q"]
    x = _plain_scores(s)
    lse = s["lse"].reshape(x.shape[:3])[..., None]
    p = x.sub_(torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)).exp_()
    return _plain_gain(s, q.shape[2], p.sum(2))


def _plain_evict(s):
    w, lens, L = s["weights"], s["lens"].long()[:, None, None], s["max_len"]
    budget, page = s["budget"], s["k_cache"].shape[1]
    B, Hkv = w.shape[:2]
    j = torch.arange(L, device=w.device)
    rank = ((j < s["sinks"]) | (j >= lens - s["recent"])).int() + 1                 # kept whatever their weight, the rest, no token
    rank = torch.where(j < lens, rank, torch.zeros_like(rank)).expand(B, Hkv, L)
    order = torch.sort(w[..., :L], dim=-1, descending=True, stable=True).indices    # the heaviest, of equal ones the oldest first
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, descending=True, stable=True).indices)
    new_lens = torch.clamp(s["lens"], max=budget)
    live = torch.arange(budget, device=w.device) < new_lens[:, None, None]          # [B, 1, budget]
    first = torch.nn.functional.pad(order, (0, max(0, budget - L)))[..., :budget]
    kept = torch.where(live, first, torch.full_like(first, L)).sort(-1).values      # slot order
    src = torch.where(live, kept, torch.zeros_like(kept))
    new_w = torch.where(live, w.gather(-1, src), torch.zeros((), device=w.device))
    b, h, r = torch.nonzero(live.expand(B, Hkv, budget), as_tuple=True)
    at = src[b, h, r]
    from_page, to_page = s["table"].long()[b, at // page], s["spare"].long()[b, r // page]
    s["k_cache"][to_page, r % page, h] = s["k_cache"][from_page, at % page, h]
    s["v_cache"][to_page, r % page, h] = s["v_cache"][from_page, at % page, h]
    return s["k_cache"], s["v_cache"], new_lens, new_w, torch.where(live, kept, torch.full_like(kept, -1)).int()


_PLAIN = dict(rotary=_plain_rotary, append=_plain_append, decode=_plain_decode, chunk=_plain_chunk, evict=_plain_evict)


# ---- one pass: the framework's calls ------------------------------------------------------------------------------------

def _own_rotary(fn, s):
    q, k = fn.rotary(s["q"], s["k"], s["positions"], s["inv_freq"], sections=s["sections"], interleaved=s["interleaved"])
    return (q, k) + torch.autograd.grad((q, k), (s["q"], s["k"]), (s["dq"], s["dk"]))


def _own_append(fn, s):
    q = fn.rotary_append(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["k_cache"], s["v_cache"], s["lens"], s["table"],
                         max_seq_len=s["max_len"], sections=s["sections"], interleaved=s["interleaved"])
    return q, s["k_cache"], s["v_cache"]


def _own_decode(fn, s):
    out = fn.decode_attention_weights(s["q"], s["k_cache"], s["v_cache"], s["weights"], s["lens"], s["table"], max_seq_len=s["max_len"],
                                      scale=s["scale"], softcap=s["softcap"], alibi_slopes=s["alibi_slopes"], window=s["window"])
    return out, s["weights"]


def _own_chunk(fn, s):
    return fn.prefill_key_weights(s["q"], s["k_cache"], s["lse"], s["weights"], s["lens"], s["table"], max_seq_len=s["max_len"],
                                  scale=s["scale"], softcap=s["softcap"], alibi_slopes=s["alibi_slopes"], window=s["window"])


def _own_evict(fn, s):
    new_lens, new_w, kept = fn.evict_cache(s["weights"], s["k_cache"], s["v_cache"], s["lens"], s["table"], s["spare"], s["budget"],
                                           sinks=s["sinks"], recent=s["recent"], max_seq_len=s["max_len"])
    return s["k_cache"], s["v_cache"], new_lens, new_w, kept


_OWN = dict(rotary=_own_rotary, append=_own_append, decode=_own_decode, chunk=_own_chunk, evict=_own_evict)


def run(state):
    if own:
        from paper_2511_02043_amd import functional
        return _OWN[state["kind"]](functional, state)
    with torch.no_grad():
        return _PLAIN[state["kind"]](state)


# ---- 64 bits ------------------------------------------------------------------------------------------------------------

def _exact_turn(x, s, sign):
    """x [B, heads, S, D] as complex numbers, one per channel pair, times exp(i angle)."""
    n, y = s["inv_freq"].numel(), x.detach().double().clone()
    at = torch.arange(n, device=DEVICE)
    re, im = (2 * at, 2 * at + 1) if s["interleaved"] else (at, at + n)
    first = 0
    for a, count in enumerate(s["sections"]):
        pair = slice(first, first + count)
        angle = s["positions"][..., a].double()[..., None] * s["inv_freq"][pair].double()       # [B, S, count]
        z = torch.complex(y[..., re[pair]], y[..., im[pair]]) * torch.exp(1j * sign * angle)[:, None]
        y[..., re[pair]], y[..., im[pair]] = z.real, z.imag
        first += count
    return y


def _exact_rows(cache, table, b, n):
    page = cache.shape[1]
    j = torch.arange(n, device=DEVICE)
    return cache[table[b].long()[j // page], j % page].double()                      # [n, Hkv, D]


def _exact_softmax(s, b, h, k):
    """Probabilities [rows, n] of query head h of sequence b over its n cached keys k [n, D], and which rows see a key."""
    T, n = s["q"].shape[2], k.shape[0]
    x = s["scale"] * (s["q"][b, h].double() @ k.t())
    if s["softcap"] is not None:
        x = s["softcap"] * torch.tanh(x / s["softcap"])
    i, j = torch.arange(n - T, n, device=DEVICE)[:, None], torch.arange(n, device=DEVICE)[None]
    if s["alibi_slopes"] is not None:
        x = x - float(s["alibi_slopes"][h]) * (i - j)
    seen = j <= i
    if s["window"] is not None:
        seen = seen & (i - j <= s["window"])
    x = x.masked_fill(~seen, float("-inf"))
    if s["kind"] == "chunk":
        lse = s["lse"][b, h].double()[:, None]
        return torch.where(seen, torch.exp(x - torch.where(lse.isinf(), torch.zeros_like(lse), lse)), torch.zeros_like(x))
    return torch.nan_to_num(torch.softmax(x, -1), nan=0.0)


def _exact_attention(s):
    q, weights = s["q"], s["weights"].double()
    B, H, T, D = q.shape
    Hkv = s["k_cache"].shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lens"].tolist()):
        k, v = _exact_rows(s["k_cache"], s["table"], b, n), _exact_rows(s["v_cache"], s["table"], b, n)
        weights[b, :, max(0, n - T):n] = 0.0
        for h in range(H):
            hk = h // (H // Hkv)
            p = _exact_softmax(s, b, h, k[:, hk])
            weights[b, hk, :n] += p.sum(0)
            if s["kind"] == "decode":
                out[b, h] = p @ v[:, hk]
    return weights if s["kind"] == "chunk" else (out, weights)


def _exact_append(s):
    q, k, cache = _exact_turn(s["q"], s, 1.0), _exact_turn(s["k"], s, 1.0), s["k_cache"].double()
    T, page = q.shape[2], cache.shape[1]
    for b, n in enumerate(s["lens"].tolist()):
        j = torch.arange(max(0, n - T), n, device=DEVICE)
        cache[s["table"][b].long()[j // page], j % page] = k[b, :, j - n + T].transpose(0, 1)
    return q, cache, None


def _exact_evict(s):
    """The weights that stay; what else comes back is copied or whole."""
    w, kept_w = s["weights"].cpu().numpy(), np.zeros(s["weights"].shape[:2] + (s["budget"],))
    for b, n in enumerate(s["lens"].tolist()):
        free = np.arange(min(s["sinks"], n), max(min(s["sinks"], n), n - s["recent"]))
        for h in range(w.shape[1]):
            lost = free[np.lexsort((-free, w[b, h, free]))][:max(0, n - s["budget"])]
            stay = np.delete(np.arange(n), lost)
            kept_w[b, h, :len(stay)] = w[b, h, stay]
    return None, None, None, torch.from_numpy(kept_w).to(DEVICE), None


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_turn(s["q"], s, 1.0), _exact_turn(s["k"], s, 1.0), _exact_turn(s["dq"], s, -1.0), _exact_turn(s["dk"], s, -1.0)
    if case["kind"] == "append":
        return _exact_append(s)
    if case["kind"] == "evict":
        return _exact_evict(s)
    return _exact_attention(s)


# ---- work ---------------------------------------------------------------------------------------------------------------

def _mean_len(case):
    return (case["lo"] + case["hi"]) / 2


def _seen(case, rows):
    """Visible keys per head and sequence, summed over the rows, at the mean length."""
    n, reach = _mean_len(case), _WINDOW + 1 if case["variant"] == "window" else float("inf")
    rows = min(rows, n)
    if reach >= n:
        return rows * (n - (rows - 1) / 2)
    ramp = max(0.0, min(rows, reach - (n - rows)))       # rows that see less than a window
    return (rows - ramp) * reach + ramp * (n - rows) + ramp * (ramp + 1) / 2


def _reached(case, rows):
    """Keys that any of the rows sees."""
    n = _mean_len(case)
    return min(n, _WINDOW + rows) if case["variant"] == "window" else n


def _scores(case):
    """Scores that the plain form holds at once."""
    if case["kind"] not in ("decode", "chunk"):
        return 0
    return case["B"] * case["H"] * case.get("T", case.get("Sq")) * case["hi"]


def work(case):
    """Each input read once and each output written once; one contraction per visible score for the keys' weights, two where
    the rows' outputs are computed too."""
    kind, B, Hkv, D = case["kind"], case["B"], case["Hkv"], case["D"]
    if kind == "rotary":
        size, heads, pairs = 4 if case["dtype"] == "f32" else 2, case["H"] + Hkv, sum(_sections(case))
        tokens = B * case["S"]
        return dict(bytes=4 * size * tokens * heads * D + 4 * tokens * len(_sections(case)), flops=2 * 6 * tokens * heads * pairs)
    if kind == "append":
        tokens, heads = B * case["T"], case["H"] + Hkv
        return dict(bytes=2 * 2 * tokens * (heads + Hkv) * D + 4 * tokens * len(_sections(case)), flops=6 * tokens * heads * sum(_sections(case)))
    if kind == "evict":
        n = _mean_len(case)
        kept = min(case["budget"], n)
        return dict(bytes=B * Hkv * (4 * n + kept * (2 * 2 * 2 * D + 4 + 4)), flops=B * Hkv * n)
    H, rows = case["H"], case["T"] if kind == "decode" else case["Sq"]
    qo, cached, w = 2 * B * H * rows * D, 2 * B * Hkv * _reached(case, rows) * D, 4 * B * Hkv * _reached(case, rows)
    if kind == "decode":
        return dict(bytes=2 * qo + 2 * cached + 2 * w, flops=4 * D * B * H * _seen(case, rows))
    return dict(bytes=qo + 4 * B * H * rows + cached + 2 * w, flops=2 * D * B * H * _seen(case, rows))
