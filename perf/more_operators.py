"""Timed cases of normalised, turned heads and of a key/value cache in 4 bits, and each operator's plain form.

  norm     queries and keys: every head's row is normalised, weighted and turned by its position, forward and backward pass
  append   the same for new tokens in serving: queries out, keys and values into the pages of a bf16 cache or of a 4-bit cache
  decode   the newest rows of every sequence attend to a 4-bit paged cache
  chunk    a chunk of prompt rows per sequence attends to a 4-bit paged cache

`own` says what run() does: False, plain torch operations; True, the calls of `paper_2511_02043_amd.functional`.  Layouts are
those of that module: q [B, H, T, D], bf16 caches [pages, page_size, Hkv, D], int32 lengths and block tables, and 4-bit caches uint8
[pages, Hkv, page_size * (D / 2 + D / 32)]: for each page and kv head the codes [page_size, D / 2] of its tokens (byte i holds channel 2 i in its low
half and 2 i + 1 in its high half), then the scales [D / 32, page_size].  A code is a sign and an index into 0, 0.5, 1, 1.5, 2, 3, 4, 6; a
scale byte E stands for 2^(E - 127) and belongs to 32 channels of one token: the smallest with every magnitude below 7 of it, from 1 to 252.
"""
import numpy as np
import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
_MOST_FLOPS = 5.6e11                  # no drawn case costs more than the largest listed one,
_MOST_BYTES = 1.4e9                   # ... moves more than the listed training step,
_MOST_SCORES = 2.2e9                  # ... nor has more scores than the listed prompt,
_MOST_HELD = 1.1e9                    # ... nor holds more values than the listed decode batch


def listed():
    return [
        # a training step of a decoder layer on video: text, then frames of 16 x 16 patches, three axes over D = 128
        dict(name="norm_train_video", kind="norm", dtype="bf16", B=2, S=8192, H=32, Hkv=8, D=128, sections="16,24,24", interleaved=False),
        # fp32 training on a small image of odd size, neighbouring channels paired, a quarter of the channels not turned
        dict(name="norm_train_f32", kind="norm", dtype="f32", B=1, S=333, H=8, Hkv=8, D=64, sections="12,12", interleaved=True),
        # the token being generated, a full serving batch: bound by latency
        dict(name="append4_token", kind="append", cache="mx4", B=64, T=1, H=32, Hkv=8, D=128, page=16, lo=1024, hi=4096, sections="16,24,24", interleaved=False),
        # a chunk of prompt tokens per sequence enters the 4-bit cache
        dict(name="append4_chunk", kind="append", cache="mx4", B=8, T=512, H=32, Hkv=8, D=128, page=16, lo=512, hi=4096, sections="64", interleaved=False),
        # the token being generated of a smaller model with a bf16 cache
        dict(name="append_token", kind="append", cache="bf16", B=16, T=1, H=16, Hkv=2, D=64, page=32, lo=300, hi=900, sections="32", interleaved=True),
        # one decode step of a full serving batch over long caches
        dict(name="decode4_batch", kind="decode", variant="plain", B=64, T=1, H=32, Hkv=8, D=128, lo=4096, hi=8192, page=16),
        # one decode step of a single short conversation: latency
        dict(name="decode4_single", kind="decode", variant="plain", B=1, T=1, H=32, Hkv=8, D=64, lo=1500, hi=2000, page=16),
        # a speculative step: four rows verified at once, soft-capped scores
        dict(name="decode4_speculative", kind="decode", variant="softcap", B=16, T=4, H=32, Hkv=8, D=128, lo=2048, hi=4096, page=16),
        # two whole books in the cache
        dict(name="decode4_long", kind="decode", variant="plain", B=2, T=1, H=32, Hkv=8, D=128, lo=100000, hi=131072, page=64),
        # a chunk of prompt rows per sequence over what is cached (chunked prefill)
        dict(name="chunk4_512", kind="chunk", variant="plain", B=8, T=512, H=32, Hkv=8, D=128, lo=4096, hi=8192, page=16),
        # a whole long prompt at once
        dict(name="chunk4_prompt", kind="chunk", variant="plain", B=1, T=8192, H=32, Hkv=8, D=128, lo=8192, hi=8192, page=16),
        # the odd rest of a prompt over a window of a small model's cache
        dict(name="chunk4_rest", kind="chunk", variant="window", B=4, T=77, H=16, Hkv=2, D=64, lo=700, hi=1500, page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and _scores(case) <= _MOST_SCORES and _held(case) <= _MOST_HELD:
            return case


_SECTIONS = {32: ["16", "8,8", "4,6,6"], 64: ["32", "16,16", "8,12,12", "12,12"], 80: ["40", "20,20"], 128: ["64", "32,32", "16,24,24", "32"]}


def _draw(rng):
    kind = rng.choice(["norm", "norm", "append", "append", "decode", "decode", "decode", "chunk", "chunk"])
    H, Hkv = rng.choice([(8, 8), (16, 16), (16, 2), (32, 8)])
    if kind == "norm":
        dtype, D = rng.choice(["bf16", "bf16", "f32"]), rng.choice([32, 64, 80, 128])
        S = _log_int(rng, 1, 1024 if dtype == "f32" else 16384)
        return dict(kind=kind, dtype=dtype, B=_log_int(rng, 1, max(1, 16384 // S)), S=S, H=H, Hkv=Hkv, D=D,
                    sections=rng.choice(_SECTIONS[D]), interleaved=rng.choice([False, True]))
    D, page = rng.choice([64, 128]), rng.choice([8, 16, 16, 32, 64])
    if kind == "append":
        T = rng.choice([1, _log_int(rng, 1, 1024)])
        hi = _log_int(rng, max(T, 64), 4096)
        return dict(kind=kind, cache=rng.choice(["mx4", "mx4", "bf16"]), B=_log_int(rng, 1, 64 if T <= 64 else 8), T=T, H=H, Hkv=Hkv, D=D, page=page,
                    lo=hi // 2, hi=hi, sections=rng.choice(_SECTIONS[D]), interleaved=rng.choice([False, True]))
    variant = rng.choice(["plain", "plain", "softcap", "alibi", "window"])
    if kind == "decode":
        hi = _log_int(rng, 2, 131072)
        return dict(kind=kind, variant=variant, B=_log_int(rng, 1, 64), T=rng.choice([1, 1, 1, 2, 4]), H=H, Hkv=Hkv, D=D, lo=hi // 2,
                    hi=hi, page=page)
    T = _log_int(rng, 9, 4096)
    hi = _log_int(rng, T, 16384)
    return dict(kind=kind, variant=variant, B=_log_int(rng, 1, 8), T=T, H=H, Hkv=Hkv, D=D, lo=hi // 2, hi=hi, page=page)


# ---- inputs -----------------------------------------------------------------------------------------------------------

_CAP, _WINDOW, _BASE, _GRID = 30.0, 512, 10000.0, 16


def _normal(gen, *shape, dtype=torch.bfloat16):
    """N(0, 1), drawn in fp32 and rounded to the storage type."""
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)


def _gains(gen, D):
    """Channels of a head differ in size: most within a factor of two, some far out."""
    return torch.exp(0.5 * torch.randn(D, generator=gen, device=DEVICE))


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


def _to_mx4(x):
    """Rows [..., D] -> codes uint8 [..., D / 2] and scales uint8 [..., D / 32]."""
    D = x.shape[-1]
    b = x.unflatten(-1, (D // 32, 32))
    half, power = torch.frexp(b.abs().amax(-1))                                     # amax = half * 2^power, half in [0.5, 1)
    e = (power + 124 + (half >= 0.875).int()).clamp(1, 252)
    t = torch.ldexp(b.abs(), (127 - e)[..., None])
    code = (t > 0.25).byte() + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.0) + 8 * torch.signbit(b).byte()
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], e.byte()


def _pages(x):
    """Pages of rows [pages, Hkv, page, D] as a 4-bit cache."""
    codes, scales = _to_mx4(x)
    return torch.cat([codes.flatten(2), scales.transpose(2, 3).flatten(2)], -1).contiguous()


def _cache(case, seed, gen):
    """Lengths, a pool of pages handed out in arbitrary order, as a serving system's allocator does, and block tables."""
    B, Hkv, D, page = (case[n] for n in ("B", "Hkv", "D", "page"))
    rng = np.random.default_rng(seed)
    lens = rng.integers(case["lo"], case["hi"] + 1, size=B).astype(np.int32)
    per = -(-case["hi"] // page)
    table = rng.permutation(B * per).astype(np.int32).reshape(B, per)
    if case.get("cache") == "bf16":
        k_cache, v_cache = (_normal(gen, B * per, page, Hkv, D) for _ in range(2))
    else:
        k_cache, v_cache = (_pages(_normal(gen, B * per, Hkv, page, D, dtype=torch.float32).mul_(_gains(gen, D))) for _ in range(2))
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEVICE)
    return dict(k_cache=k_cache, v_cache=v_cache, lens=up(lens), table=up(table), max_len=case["hi"], page=page)


def _variant(case):
    H, variant = case["H"], case["variant"]
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], dtype=torch.float32, device=DEVICE)
    return dict(softcap=_CAP if variant == "softcap" else None, alibi_slopes=slopes if variant == "alibi" else None,
                window=_WINDOW if variant == "window" else None)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    kind, rng = case["kind"], np.random.default_rng(seed)
    B, H, Hkv, D = (case[n] for n in ("B", "H", "Hkv", "D"))
    if kind in ("norm", "append"):
        S = case["S"] if kind == "norm" else case["T"]
        dtype = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
        proj = _normal(gen, B, S, H + 2 * Hkv, D, dtype=dtype).transpose(1, 2)      # one projection: [B, S, heads, D] in memory
        q, k, v = proj[:, :H], proj[:, H:H + Hkv], proj[:, H + Hkv:]
        state = dict(q_weight=_gains(gen, D), k_weight=_gains(gen, D), inv_freq=_inv_freq(case), sections=_sections(case), interleaved=case["interleaved"])
    if kind == "norm":
        first = torch.from_numpy(rng.integers(0, 64, size=B)).to(DEVICE)
        leaf = lambda x: x.detach().requires_grad_(True)
        state.update(q=leaf(q), k=leaf(k), q_weight=leaf(state["q_weight"]), k_weight=leaf(state["k_weight"]), positions=_positions(case, first, S),
                     dq=_normal(gen, B, H, S, D, dtype=dtype), dk=_normal(gen, B, Hkv, S, D, dtype=dtype))
    elif kind == "append":
        state.update(_cache(case, seed, gen))
        # positions go on where the sequence is, whatever was evicted before
        first = state["lens"].long() - S + torch.from_numpy(rng.integers(S, 4096 + S, size=B)).to(DEVICE)
        state.update(q=q, k=k, v=v, positions=_positions(case, first, S), mx4=case["cache"] == "mx4")
    else:
        state = _cache(case, seed, gen)
        state.update(q=_normal(gen, B, H, case["T"], D), scale=D ** -0.5, **_variant(case))
    state["kind"] = kind
    return state


# ---- one pass: plain forms ----------------------------------------------------------------------------------------------

def _plain_turn(y, s, back):
    """Each pair (a, b) of channels becomes (a cos - b sin, b cos + a sin) at the angle position * frequency of its axis, formed in 64 bits for far
    positions (back: at the negative angle); channels beyond the pairs stay."""
    n, sections = s["inv_freq"].numel(), s["sections"]
    axis = torch.repeat_interleave(torch.arange(len(sections), device=y.device), torch.tensor(sections, device=y.device))
    angle = (s["positions"][:, :, axis].double() * s["inv_freq"].double())[:, None]  # [B, 1, S, pairs]
    cos, sin = torch.cos(angle).to(y.dtype), (torch.sin(angle) * (-1.0 if back else 1.0)).to(y.dtype)
    if s["interleaved"]:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, y[..., 2 * n:]], -1)


def _plain_heads(x, weight, s):
    """x [B, heads, S, D] normalised, weighted and turned."""
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return _plain_turn(x * r * weight, s, False)


def _plain_gradient(x, weight, dy, s):
    """The gradients of _plain_heads with respect to x and weight."""
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    dz = _plain_turn(dy, s, True)
    g = dz * weight
    dx = r * g - x * (r * r * r * (x * g).mean(-1, keepdim=True))
    return dx, (dz * x * r).sum((0, 1, 2), dtype=torch.float64)


def _plain_norm(s):
    out = []
    for x, w, dy in ((s["q"], s["q_weight"], s["dq"]), (s["k"], s["k_weight"], s["dk"])):
        x, w = x.detach(), w.detach()
        dx, dw = _plain_gradient(x.float(), w, dy.float(), s)
        out.append((_plain_heads(x.float(), w, s).to(x.dtype), dx.to(x.dtype), dw.float()))
    return tuple(zip(*out))


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _from_mx4(codes, scales):
    """Codes uint8 [..., D / 2] and scales uint8 [..., D / 32] -> fp32 [..., D]."""
    table = torch.tensor(_VALUES, device=codes.device)
    x = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * torch.ldexp(torch.ones((), device=codes.device), scales.int() - 127)[..., None]).flatten(-2)


def _plain_append(s):
    k_cache, v_cache, page = s["k_cache"], s["v_cache"], s["page"]
    q = _plain_heads(s["q"].float(), s["q_weight"], s).to(s["q"].dtype)
    T = q.shape[2]
    slot = s["lens"].long()[:, None] - T + torch.arange(T, device=q.device)         # [B, T]; below 0: not a token of the sequence
    b, t = torch.nonzero(slot >= 0, as_tuple=True)
    at = slot[b, t]
    pages, at = s["table"].long()[b, at // page], at % page
    if not s["mx4"]:
        k_cache[pages, at] = _plain_heads(s["k"].float(), s["k_weight"], s).to(q.dtype)[b, :, t]
        v_cache[pages, at] = s["v"][b, :, t]
        return q, k_cache, v_cache
    D, out = q.shape[-1], [q]
    # keys in 64 bits: a value next to the border of two codes
    for x, cache in ((_plain_heads(s["k"].double(), s["k_weight"].double(), s), k_cache), (s["v"].float(), v_cache)):
        codes, scales = _to_mx4(x)
        split = page * (D // 2)
        cache[..., :split].unflatten(-1, (page, D // 2))[pages, :, at] = codes[b, :, t]
        cache[..., split:].unflatten(-1, (D // 32, page))[pages, :, :, at] = scales[b, :, t]
        out += [cache, _from_mx4(codes, scales).to(q.dtype)]
    return tuple(out)


def _gathered(cache, s):
    """[B, Hkv, max_len, D] rows of a paged 4-bit cache in fp32."""
    D, page, table = s["q"].shape[-1], s["page"], s["table"].long()
    x, split = cache[table].transpose(1, 2), page * (D // 2)                        # [B, Hkv, pages, bytes]
    rows = _from_mx4(x[..., :split].unflatten(-1, (page, D // 2)), x[..., split:].unflatten(-1, (D // 32, page)).transpose(-1, -2))
    return rows.flatten(2, 3)[:, :, :s["max_len"]]


def _plain_scores(s):
    """Masked scores [B, Hkv, group * rows, max_len] of the newest rows, -inf where hidden."""
    q, lens = s["q"], s["lens"].long()
    B, H, T, D = q.shape
    k = _gathered(s["k_cache"], s)
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


def _plain_attention(s):
    q = s["q"]
    x = _plain_scores(s)
    m = x.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + m).reshape(q.shape[:3])
    out = torch.matmul(p, _gathered(s["v_cache"], s))
    out = torch.where(total > 0, out / total, torch.zeros_like(out))
    return out.reshape(q.shape).to(q.dtype), lse


_PLAIN = dict(norm=_plain_norm, append=_plain_append, decode=_plain_attention, chunk=_plain_attention)


# ---- one pass: the framework's calls ------------------------------------------------------------------------------------

def _own_norm(fn, s):
    leaves = s["q"], s["k"], s["q_weight"], s["k_weight"]
    q, k = fn.norm_rotary(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_weight"], s["k_weight"], eps=EPS, sections=s["sections"],
                          interleaved=s["interleaved"])
    dq, dk, dqw, dkw = torch.autograd.grad((q, k), leaves, (s["dq"], s["dk"]))
    return (q, k), (dq, dk), (dqw, dkw)


def _own_append(fn, s):
    got = fn.norm_rotary_append(s["q"], s["k"], s["v"], s["positions"], s["inv_freq"], s["k_cache"], s["v_cache"], s["lens"], s["table"], s["q_weight"],
                                s["k_weight"], eps=EPS, max_seq_len=s["max_len"], sections=s["sections"], interleaved=s["interleaved"],
                                return_held=s["mx4"])
    if not s["mx4"]:
        return got, s["k_cache"], s["v_cache"]
    q, k_held, v_held = got
    return q, s["k_cache"], k_held, s["v_cache"], v_held


def _own_attention(call, s):
    return call(s["q"], s["k_cache"], s["v_cache"], s["lens"], s["table"], max_seq_len=s["max_len"], scale=s["scale"], softcap=s["softcap"],
                alibi_slopes=s["alibi_slopes"], window=s["window"], return_lse=True)


_OWN = dict(norm=_own_norm, append=_own_append, decode=lambda fn, s: _own_attention(fn.decode_attention_mx4, s),
            chunk=lambda fn, s: _own_attention(fn.paged_prefill_attention_mx4, s))


def run(state):
    if own:
        from paper_2511_02043_amd import functional
        return _OWN[state["kind"]](functional, state)
    with torch.no_grad():
        return _PLAIN[state["kind"]](state)


# ---- 64 bits ------------------------------------------------------------------------------------------------------------

def _exact_turn(x, s, sign):
    """x [B, heads, S, D] as complex numbers, one per channel pair, times exp(i angle)."""
    n, y = s["inv_freq"].numel(), x.clone()
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


def _exact_heads(x, weight, s):
    x = x.detach().double()
    length = torch.linalg.vector_norm(x, dim=-1, keepdim=True)
    return _exact_turn(x / torch.sqrt(length ** 2 / x.shape[-1] + EPS) * weight.detach().double(), s, 1.0)


def _exact_norm(s):
    out = []
    for x, w, dy in ((s["q"], s["q_weight"], s["dq"]), (s["k"], s["k_weight"], s["dk"])):
        y = _exact_heads(x, w, s)
        x, w, dz = x.detach().double(), w.detach().double(), _exact_turn(dy.double(), s, -1.0)
        D = x.shape[-1]
        size = torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS)
        unit = x / size                            # d unit / dx = (1 - unit unit^T / D) / size
        g = dz * w
        out.append((y, (g - unit * (unit * g).sum(-1, keepdim=True) / D) / size, (dz * unit).flatten(0, 2).sum(0)))
    return tuple(zip(*out))


def _exact_held(x):
    """Each value of the rows x [..., D] as a 4-bit cache holds it: the nearest of its block's sixteen (halfway: the even code)."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEVICE)
    b = x.double().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(most > 0, most, torch.ones_like(most)))) - 3
    for _ in range(4):                             # up from below the one that is wanted
        e = e + (most >= 7.0 * 2.0 ** e)
    unit = 2.0 ** e.clamp(-126, 125)
    size = (b.abs() / unit)[..., None]
    off = (size - grid).abs()
    off[..., 1::2] *= 1 + 1e-15                    # a tie between neighbours goes to the even one
    return (torch.sign(b) * grid[off.argmin(-1)] * unit).flatten(-2)


def _exact_append(s):
    q, k = _exact_heads(s["q"], s["q_weight"], s), _exact_heads(s["k"], s["k_weight"], s)
    if s["mx4"]:
        return q, None, _exact_held(k), None, _exact_held(s["v"])
    T, page, cache = q.shape[2], s["page"], s["k_cache"].double()
    for b, n in enumerate(s["lens"].tolist()):
        j = torch.arange(max(0, n - T), n, device=DEVICE)
        cache[s["table"][b].long()[j // page], j % page] = k[b, :, j - n + T].transpose(0, 1)
    return q, cache, None


def _exact_rows(cache, s, b, n):
    """[n, Hkv, D] values of sequence b's cached tokens."""
    page, D = s["page"], s["q"].shape[-1]
    j = torch.arange(n, device=DEVICE)
    at, within = s["table"][b].long()[j // page], j % page
    c = torch.arange(D, device=DEVICE)
    byte = cache[at[:, None], :, (within * (D // 2))[:, None] + c // 2].long()       # [n, D, Hkv]
    code = torch.where((c % 2 == 1)[None, :, None], byte // 16, byte % 16)
    e = cache[at[:, None], :, page * (D // 2) + (c // 32) * page + within[:, None]].double()
    size = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEVICE)[code % 8]
    return (torch.where(code >= 8, -size, size) * torch.exp2(e - 127)).transpose(1, 2)


def _exact_attention(s):
    q = s["q"]
    B, H, T, D = q.shape
    group = H // s["k_cache"].shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(q.shape[:3], float("-inf"), dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lens"].tolist()):
        if n == 0:
            continue
        k, v = _exact_rows(s["k_cache"], s, b, n), _exact_rows(s["v_cache"], s, b, n)
        i, j = torch.arange(n - T, n, device=DEVICE)[:, None], torch.arange(n, device=DEVICE)[None]
        seen = j <= i
        if s["window"] is not None:
            seen = seen & (i - j <= s["window"])
        for h in range(H):
            x = s["scale"] * (q[b, h].double() @ k[:, h // group].t())
            if s["softcap"] is not None:
                x = s["softcap"] * torch.tanh(x / s["softcap"])
            if s["alibi_slopes"] is not None:
                x = x - float(s["alibi_slopes"][h]) * (i - j)
            x = x.masked_fill(~seen, float("-inf"))
            lse[b, h] = torch.logsumexp(x, -1)
            out[b, h] = torch.nan_to_num(torch.softmax(x, -1), nan=0.0) @ v[:, h // group]
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    return dict(norm=_exact_norm, append=_exact_append, decode=_exact_attention, chunk=_exact_attention)[case["kind"]](s)


# ---- work ---------------------------------------------------------------------------------------------------------------

def _mean_len(case):
    return (case["lo"] + case["hi"]) / 2


def _seen(case):
    """Visible keys per head and sequence, summed over the rows, at the mean length."""
    n, reach = _mean_len(case), _WINDOW + 1 if case["variant"] == "window" else float("inf")
    rows = min(case["T"], n)
    if reach >= n:
        return rows * (n - (rows - 1) / 2)
    ramp = max(0.0, min(rows, reach - (n - rows)))       # rows that see less than a window
    return (rows - ramp) * reach + ramp * (n - rows) + ramp * (ramp + 1) / 2


def _scores(case):
    """Scores that the plain form holds at once."""
    return case["B"] * case["H"] * case["T"] * case["hi"] if case["kind"] in ("decode", "chunk") else 0


def _held(case):
    """Values in the caches."""
    return 2 * case["B"] * case["hi"] * case["Hkv"] * case["D"] if case["kind"] != "norm" else 0


def _row_bytes(case):
    """Of one token and kv head in a cache."""
    return 2 * case["D"] if case.get("cache") == "bf16" else case["D"] // 2 + case["D"] // 32


def work(case):
    """Each input read once and each output written once; two contractions per visible score."""
    kind, B, H, Hkv, D = (case[n] for n in ("kind", "B", "H", "Hkv", "D"))
    if kind == "norm":
        size, heads, pairs = 4 if case["dtype"] == "f32" else 2, H + Hkv, sum(_sections(case))
        tokens = B * case["S"]
        # forward: x in, y out; backward: x and dy in, dx out
        return dict(bytes=5 * size * tokens * heads * D + 4 * tokens * len(_sections(case)) + 16 * D, flops=tokens * heads * (12 * pairs + 14 * D))
    if kind == "append":
        tokens = B * case["T"]
        held = 2 * 2 * Hkv * D if case["cache"] == "mx4" else 0                      # k and v as they are held, for the caller
        return dict(bytes=tokens * (2 * 2 * H * D + 2 * 2 * Hkv * D + 2 * Hkv * _row_bytes(case) + held + 4 * len(_sections(case))) + 8 * D,
                    flops=tokens * (H + Hkv) * (6 * sum(_sections(case)) + 5 * D))
    reached = min(_mean_len(case), _WINDOW + case["T"]) if case["variant"] == "window" else _mean_len(case)
    rows = B * H * case["T"]
    return dict(bytes=2 * 2 * rows * D + 4 * rows + 2 * B * Hkv * reached * _row_bytes(case), flops=4 * D * B * H * _seen(case))
