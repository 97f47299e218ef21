"""A paged cache in the model's own type as a serving program has it: what is timed when the speed of its operators is
looked at, and their plain forms.  A case is a plain dict; `prepare` builds what the program holds before the call, `run`
makes one pass.

Operators (public entry points in paper_2503_19950_amd.binding: Rope, rotate, class DeviceCachePaged)
  rotate  rotary positions of queries and keys: pairs of the first `dims` channels turn by position * freq[pair]
  write   append: keys (rotated on the way) and values go to pages of P tokens that a table names for every row
  token   the same, one token per row
  attn    decode_attn: one query token per sequence attends through the table; scores may be capped by a tanh, get a bias
          that falls with distance, and be cut off behind a window of the newest tokens
  step    decode_step: one token is rotated and written and its rotated query, of the cache's type as well, attends; a
          cache that keeps weights adds up the attention that every token has had
  evict   evict: of every row longer than `keep`, the newest `recent` tokens and those others with the largest weights
          move to pages of their own, in order
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
CACHED = ("write", "token", "attn", "step", "evict")


def _case(kind, B, Hq, Hkv, d, L, dtype, P=64, ragged=False, dims=0, interleaved=False, scaled=False, start=0, cap=0.0, window=0,
          bias=False, weighted=False, keep=0, recent=0):
    """B rows, Hq query and Hkv kv heads of dimension d, L tokens (the longest row's with `ragged`): those that a prompt
    brings (`rotate`, `write`), else those that the cache holds before the call.  P: tokens of a page.  dims: rotated
    channels, 0 for none; `scaled`: frequencies stretched for eight times the length; `start`: position of the first token."""
    return dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, d=d, L=L, dtype=dtype, P=P, ragged=ragged, dims=dims, interleaved=interleaved,
                scaled=scaled, start=start, cap=cap, window=window, bias=bias, weighted=weighted, keep=keep, recent=recent)


def listed():
    gqa = dict(Hq=32, Hkv=8, d=128)
    return [
        # queries and keys of a serving batch's new tokens, one a row: all latency
        dict(name="rotate_token_b64", **_case("rotate", 64, L=1, dtype="f16", dims=128, start=4095, **gqa)),
        # the last quarter of a very long document, positions scaled
        dict(name="rotate_prompt_b1_32k", **_case("rotate", 1, L=32768, dtype="bf16", dims=128, scaled=True, start=98304, **gqa)),
        # a small batch of prompts of different lengths becomes a cache
        dict(name="write_ragged_b8_8k", **_case("write", 8, L=8191, dtype="f16", P=64, ragged=True, dims=128, **gqa)),
        # a serving batch, one token per row; half of the head is rotated, in pairs of neighbours
        dict(name="write_token_b64_4k", **_case("token", 64, L=4095, dtype="bf16", P=32, ragged=True, dims=64, interleaved=True, **gqa)),
        # one user, short chat: all latency
        dict(name="attn_b1_512", **_case("attn", 1, L=512, dtype="f16", P=32, **gqa)),
        # one very long document, spread over the whole GPU
        dict(name="attn_b1_128k", **_case("attn", 1, L=131072, dtype="bf16", P=64, **gqa)),
        # a full serving batch whose rows have different ages, one of them empty; capped scores
        dict(name="attn_capped_ragged_b64_4k", **_case("attn", 64, L=4096, dtype="f16", P=32, ragged=True, cap=30.0, **gqa)),
        # multi-head attention, head dimension 96, with a bias by distance and a window
        dict(name="attn_window_mha_b16_16k", **_case("attn", 16, 32, 32, 96, 16384, "bf16", 64, bias=True, window=4096)),
        # the decode step of one short chat: rotate, write and attend
        dict(name="step_b1_520", **_case("step", 1, L=520, dtype="bf16", P=64, dims=128, **gqa)),
        # the decode step of a full serving batch of rows of different ages whose cache keeps weights
        dict(name="step_weighted_ragged_b64_4k", **_case("step", 64, L=4096, dtype="f16", P=32, ragged=True, dims=128, weighted=True, **gqa)),
        # the serving batch gives up half of its longest rows' room
        dict(name="evict_ragged_b64_4k", **_case("evict", 64, L=4096, dtype="f16", P=32, ragged=True, weighted=True, keep=2048, recent=256, **gqa)),
        # a very long document gives up half of its tokens
        dict(name="evict_b1_128k", **_case("evict", 1, L=131072, dtype="bf16", P=64, weighted=True, keep=65536, recent=4096, **gqa)),
    ]


MOST_VALUES = 16 * 32 * 16384 * 96     # of a cache's K (or V): the largest listed case


def draw(rng):
    kind = rng.choice(["rotate", "write", "token", "attn", "attn", "attn", "step", "step", "evict"])
    d = rng.choice([64, 96, 128, 128])
    Hkv, gh = rng.choice([(8, 4), (8, 4), (8, 1), (32, 1), (2, 8), (4, 2), (1, 16), (8, 8), (4, 5), (2, 3), (1, 24)])
    B = round(2 ** rng.uniform(0, 6))
    L = round(2 ** rng.uniform(0, 17))
    most = MOST_VALUES // {"attn": 4, "token": 8, "step": 8}.get(kind, 16)
    wide = gh if kind == "rotate" else 1
    while B * Hkv * wide * L * d > most and L > 300:
        L = L * 2 // 3
    while B * Hkv * wide * L * d > most:
        B = (B + 1) // 2
    rotates = kind == "rotate" or (kind in ("write", "token", "step") and rng.random() < 0.8)
    dims = 2 * rng.choice([d // 2, d // 2, d // 4, rng.randint(1, d // 2)]) if rotates else 0
    scores = kind in ("attn", "step")
    window = rng.choice([0, 0, rng.randint(1, L)]) if scores else 0
    keep = rng.randint(1, L) if kind == "evict" else 0
    return _case(kind, B, Hkv * gh, Hkv, d, L, rng.choice(["f16", "bf16"]), rng.choice([32, 32, 64, 128]),
                 ragged=kind != "rotate" and B > 1 and rng.random() < 0.5, dims=dims, interleaved=rotates and rng.random() < 0.4,
                 scaled=rotates and rng.random() < 0.3, start=rng.choice([0, rng.randint(0, 1 << 20)]) if rotates else 0,
                 cap=rng.choice([0.0, 0.0, 30.0, 50.0]) if scores else 0.0, window=window, bias=scores and rng.random() < 0.3,
                 weighted=kind == "evict" or (scores and rng.random() < 0.3), keep=keep,
                 recent=rng.choice([0, rng.randint(0, keep)]) if kind == "evict" else 0)


# ---- sizes ---------------------------------------------------------------------------------
def _lengths(c):
    """Tokens of each row: with `ragged`, spread evenly over (0, L] in a scattered order, the last of several rows empty."""
    if not c["ragged"]:
        return [c["L"]] * c["B"]
    rows = [c["L"] - int(c["L"] * (b * 0.6180339887 % 1.0)) for b in range(c["B"])]
    if c["B"] > 3:
        rows[-1] = 0
    return rows


def _after(c):
    """Tokens of each row behind the call."""
    return [n + (c["kind"] in ("token", "step")) for n in _lengths(c)]


def _pages(c, n):
    return -(-n // c["P"])


def _max_pages(c):
    return max(1, _pages(c, max(_after(c))))


def _evicted(c):
    """Rows that lose tokens."""
    return [b for b, n in enumerate(_lengths(c)) if n > c["keep"]]


# ---- layout --------------------------------------------------------------------------------
# A page of a kv head lies as 16-bit matrix operands.  Keys: [tile of 16 tokens][channel / 32][octet of channels][token % 16]
# [channel % 8]; values, with 16 b + 4 a + e the token within its unit of 32: [unit][channel / 16][a][channel % 16][b][e].
def _k_place(t, ch, d):
    return ((t // 16 * (d // 32) + ch // 32) * 64 + 16 * (ch % 32 // 8) + t % 16) * 8 + ch % 8


def _v_place(t, ch, d):
    return ((t // 32 * (d // 16) + ch // 16) * 64 + 16 * (t % 16 // 4) + ch % 16) * 8 + 4 * (t % 32 // 16) + t % 4


PLACES = {"k": _k_place, "v": _v_place}


def _to_pages(which, x):
    """[..][P][d] rows as pages [..][P * d]."""
    d = x.shape[-1]
    if which == "k":
        x = x.unflatten(-2, (-1, 16)).unflatten(-1, (d // 32, 4, 8))            # .. tile, token, chunk, octet, channel
        return x.permute(*range(x.dim() - 5), -5, -3, -2, -4, -1).flatten(-5)
    x = x.unflatten(-2, (-1, 2, 4, 4)).unflatten(-1, (d // 16, 16))             # .. unit, b, a, e, tile, channel
    return x.permute(*range(x.dim() - 6), -6, -2, -4, -1, -5, -3).flatten(-6)


def _to_rows(which, x, d):
    """And back."""
    if which == "k":
        x = x.unflatten(-1, (-1, d // 32, 4, 16, 8))                            # .. tile, chunk, octet, token, channel
        return x.permute(*range(x.dim() - 5), -5, -2, -4, -3, -1).flatten(-3).flatten(-3, -2)
    x = x.unflatten(-1, (-1, d // 16, 4, 16, 2, 4))                             # .. unit, tile, a, channel, b, e
    return x.permute(*range(x.dim() - 6), -6, -2, -4, -1, -5, -3).flatten(-2).flatten(-5, -2)


# ---- plain forms ---------------------------------------------------------------------------
def _turned(c, x, positions, freq):
    """x [B][H][L][d] turned by positions [B][L], in fp32; angles in 64 bits."""
    angle = positions.double()[..., None] * freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    x, dims = x.float(), c["dims"]
    first, second = (x[..., 0:dims:2], x[..., 1:dims:2]) if c["interleaved"] else (x[..., :dims // 2], x[..., dims // 2:dims])
    turned = [first * cos - second * sin, second * cos + first * sin]
    turned = torch.stack(turned, -1).flatten(-2) if c["interleaved"] else torch.cat(turned, -1)
    return torch.cat([turned, x[..., dims:]], -1)


def _plain_rotate(state, x):
    c = state["case"]
    return _turned(c, x, state["positions"], state["freq"]).to(TYPES[c["dtype"]])


def _put(state, which, x, slots, valid):
    """Rows x [B][Hkv][L][d] to slots [B][L] of the pool where `valid` [B][L]."""
    c = state["case"]
    pool, d, P, Hkv = state[which + "_pages"], c["d"], c["P"], c["Hkv"]
    b, i = valid.nonzero(as_tuple=True)
    slot = slots[b, i]
    page = slot // P * Hkv
    at = (page[:, None] + torch.arange(Hkv, device=DEVICE))[..., None] * (P * d) + PLACES[which](slot[:, None] % P, torch.arange(d, device=DEVICE), d)[:, None]
    pool.view(-1)[at.flatten()] = x[b, :, i].flatten()


def _slots(table, t, P):
    """Physical slots of tokens t [B][..] of every row."""
    return table.long().gather(1, t // P) * P + t % P


def _plain_append(state):
    """New rows behind what each row holds: n_new of them of each row."""
    c = state["case"]
    k_new = _plain_rotate(state, state["k_new"]) if c["dims"] else state["k_new"]
    i = torch.arange(k_new.shape[2], device=DEVICE)[None]
    valid = i < state["n_new"][:, None]
    t = (state["n"][:, None] + i).clamp(max=_max_pages(c) * c["P"] - 1)
    slots = _slots(state["table"][0], t, c["P"])
    _put(state, "k", k_new, slots, valid)
    _put(state, "v", state["v_new"], slots, valid)
    if c["weighted"]:
        live = state["weights"][0]
        b, at = valid.nonzero(as_tuple=True)
        live[b, :, t[b, at]] = 0.0


def _plain_attention(state, n, q):
    c = state["case"]
    B, Hkv, d, P = c["B"], c["Hkv"], c["d"], c["P"]
    k, v = (_to_rows(w, state[w + "_pages"][state["table"][0].long()], d).transpose(1, 2).flatten(2, 3).float() for w in "kv")
    q = q.float().reshape(B, Hkv, -1, d)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * d ** -0.5
    if c["cap"]:
        s = c["cap"] * torch.tanh(s / c["cap"])
    ahead = n[:, None] - 1 - torch.arange(_max_pages(c) * P, device=DEVICE)[None]     # distance of every slot
    if c["bias"]:
        s = s - state["slopes"].reshape(1, Hkv, -1, 1) * ahead.float()[:, None, None]
    seen = (ahead >= 0) & ((ahead < c["window"]) if c["window"] else True)
    s = s.masked_fill(~seen[:, None, None], float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-3e38))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    v = torch.where((ahead >= 0)[:, None, :, None], v, torch.zeros((), device=DEVICE))
    out = torch.matmul(p, v).reshape(B, c["Hq"], d).to(TYPES[c["dtype"]])
    if not c["weighted"]:
        return {"out": out}
    state["weights"][0] += p.sum(2)
    return {"out": out, "weights": state["weights"]}


def _plain_evict(state):
    c = state["case"]
    P, keep, recent = c["P"], c["keep"], c["recent"]
    rows = state["evicted"]
    if len(rows):
        n, w = state["n"][rows], state["weights"][0, rows]
        t = torch.arange(w.shape[-1], device=DEVICE)
        inside, newest = t < n[:, None], t >= n[:, None] - recent
        w = torch.where(newest[:, None], torch.full_like(w, float("inf")), torch.where(inside[:, None], w, torch.full_like(w, -1.0)))
        w = torch.where((inside & newest | ~newest)[:, None], w, torch.full_like(w, -1.0))
        kept = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :keep].sort(-1).values      # [rows][Hkv][keep]
        state["weights"][1, rows, :, :keep] = state["weights"][0, rows].gather(-1, kept)
        src = _slots(state["table"][0][rows], kept.flatten(1), P).reshape(kept.shape)
        dst = _slots(state["table"][1][rows], t[None, :keep].expand(len(rows), -1), P)
        head = torch.arange(c["Hkv"], device=DEVICE)[None, :, None]
        ch = torch.arange(c["d"], device=DEVICE)
        for_head = lambda slot, which: ((slot // P * c["Hkv"] + head) * (P * c["d"]))[..., None] + PLACES[which](slot[..., None] % P, ch, c["d"])  # noqa: E731
        flat = {x: state[x + "_pages"].view(-1) for x in "kv"}
        flat["k"][for_head(dst[:, None], "k")] = flat["k"][for_head(src, "k")]
        flat["v"][for_head(dst[:, None], "v")] = flat["v"][for_head(src, "v")]
    return {"k_pages": state["k_pages"], "v_pages": state["v_pages"], "weights": state["weights"]}


# ---- inputs --------------------------------------------------------------------------------
def _frequencies(c):
    """Radians a position of every pair: base ** (-2 i / dims); `scaled`: pairs that turn less than once in the first 8192
    positions eight times slower, those that turn more than four times as they are, between them in proportion."""
    f = [10000.0 ** (-2 * i / c["dims"]) for i in range(c["dims"] // 2)]
    if c["scaled"]:
        for i, x in enumerate(f):
            part = min(max((8192 * x / (2 * math.pi) - 1) / 3, 0.0), 1.0)
            f[i] = part * x + (1 - part) * x / 8
    return f


def _normal(shape, gen, dtype, outliers=None):
    """Normal values; four channels of every kv head (axis 1) ten times larger."""
    x = torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(generator=gen)
    if outliers is not None:
        boost = torch.ones((shape[1], shape[-1]), device=DEVICE).scatter_(1, outliers, 10.0)
        x *= boost[:, None]
    return x.to(dtype)


def _handle(state):
    """The framework's cache with these contents: what a serving program holds."""
    from paper_2503_19950_amd import binding
    c = state["case"]
    cfg = binding.make_config_paged(c["B"], c["Hq"], c["Hkv"], c["d"], c["P"], c["dtype"], state["k_pages"].shape[0], _max_pages(c), c["weighted"])
    cache = binding.DeviceCachePaged(cfg, DEVICE)
    cache.k_pages.copy_(state["k_pages"].view(-1).view(torch.uint8))
    cache.v_pages.copy_(state["v_pages"].view(-1).view(torch.uint8))
    for spare in (False, True):
        for b, ids in enumerate(state["ids"][spare]):
            if ids:
                cache.set_pages(b, ids, spare=spare)
    if c["weighted"]:
        cache.weights.copy_(state["weights"])
    state["k_pages"], state["v_pages"] = (getattr(cache, w + "_pages").view(TYPES[c["dtype"]]).view(state[w + "_pages"].shape) for w in "kv")
    state["weights"] = cache.weights
    return cache


def prepare(case, seed):
    c = case
    B, Hq, Hkv, d, P, L, kind = (c[x] for x in ("B", "Hq", "Hkv", "d", "P", "L", "kind"))
    gen = torch.Generator(DEVICE)
    gen.manual_seed(seed)
    pick = random.Random(seed)
    outliers = torch.tensor([pick.sample(range(d), 4) for _ in range(Hkv)], device=DEVICE)
    lengths, dt = _lengths(c), TYPES[c["dtype"]]
    state = dict(case=c, lengths=lengths)
    if c["dims"]:
        state["freq_list"] = _frequencies(c)
        state["freq"] = torch.tensor(state["freq_list"], dtype=torch.float64, device=DEVICE)
        ahead = torch.tensor([pick.randint(0, 63) for _ in range(B)], device=DEVICE)
        state["positions"] = (c["start"] + ahead[:, None] + torch.arange(L if kind in ("rotate", "write") else 1, device=DEVICE)).int()
    if kind == "rotate":
        state["q"], state["k"] = _normal((B, Hq, L, d), gen, dt), _normal((B, Hkv, L, d), gen, dt, outliers)
        state["q_out"], state["k_out"] = torch.empty_like(state["q"]), torch.empty_like(state["k"])
    else:
        # pages in a scattered order, as a pool that has served other requests gives them out
        need = [_pages(c, n) for n in _after(c)]
        spare = [_pages(c, c["keep"]) if n > c["keep"] and kind == "evict" else 0 for n in lengths]
        order = list(range(sum(need) + sum(spare) + 3))
        pick.shuffle(order)
        state["ids"] = [[[order.pop() for _ in range(x)] for x in counts] for counts in (need, spare)]
        flat = [ids + [0] * (_max_pages(c) - len(ids)) for part in state["ids"] for ids in part]
        state["table"] = torch.tensor(flat, dtype=torch.int32, device=DEVICE).reshape(2, B, _max_pages(c))
        shape = (sum(need) + sum(spare) + 3, Hkv, P, d)
        held = kind not in ("write", "token")
        for w in "kv":
            state[w + "_pages"] = _to_pages(w, _normal(shape, gen, dt, outliers if w == "k" else None)) if held else torch.zeros((*shape[:2], P * d), dtype=dt, device=DEVICE)
        state["weights"] = None
        if c["weighted"]:
            # what a thousand steps leave: most tokens little, some much, the newest of each row nothing yet (equal weights)
            w = torch.empty((2, B, Hkv, _max_pages(c) * P), device=DEVICE).exponential_(0.2, generator=gen).pow_(3.0)
            state["weights"] = torch.where(w < 1e-2, torch.zeros_like(w), w)
        state["n"] = torch.tensor([0 if kind == "write" else n for n in lengths], device=DEVICE)
        state["counts"], state["halves"] = state["n"].tolist(), [0] * B        # tokens of each row, which table of two is its
        state["n_new"] = torch.tensor(lengths if kind == "write" else [1] * B, device=DEVICE)
        state["evicted"] = torch.tensor(_evicted(c), dtype=torch.long, device=DEVICE)
        if kind in ("write", "token", "step"):
            new = (B, Hkv, L if kind == "write" else 1, d)
            state["k_new"], state["v_new"] = _normal(new, gen, dt, outliers), _normal(new, gen, dt)
        if kind in ("attn", "step"):
            state["q"] = (_normal((B, Hq, d), gen, torch.float32) * (4 if c["cap"] else 1)).to(dt)
            state["out"] = torch.empty_like(state["q"])
            state["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device=DEVICE) / Hq).float() if c["bias"] else None
    if own:
        from paper_2503_19950_amd import binding
        state["rope"] = binding.Rope(state["freq_list"], c["interleaved"], device=DEVICE) if c["dims"] else None
        state["cache"] = _handle(state) if kind != "rotate" else None
    return state


# ---- one pass ------------------------------------------------------------------------------
def _run_own(state):
    c = state["case"]
    kind, cache = c["kind"], state["cache"]
    turn = dict(rope=state["rope"], positions=state["positions"]) if c["dims"] else {}
    if kind == "rotate":
        from paper_2503_19950_amd import binding
        binding.rotate(state["rope"], state["positions"], state["q"], state["k"], state["q_out"], state["k_out"])
        return {"q": state["q_out"], "k": state["k_out"]}
    cache.set_counts(state["counts"], state["halves"])
    if kind == "write":
        cache.append(state["k_new"], state["v_new"], state["lengths"], **turn)
    if kind == "token":
        cache.append(state["k_new"], state["v_new"], **turn)
    if kind == "evict":
        cache.evict(c["keep"], c["recent"])
    result = {}
    if kind in ("attn", "step"):
        scores = dict(softcap=c["cap"], window=c["window"], slopes=state["slopes"])
        if kind == "attn":
            cache.decode_attn(state["q"], state["out"], **scores)
        else:
            cache.decode_step(state["k_new"], state["v_new"], state["q"], state["out"], **turn, **scores)
        result["out"] = state["out"]
    if c["weighted"]:
        result["weights"] = state["weights"]
    if kind != "attn":
        result.update(k_pages=state["k_pages"], v_pages=state["v_pages"])
    return result


def run(state):
    """One pass.  The counts go back to where `prepare` left them first, so that a pass can be repeated: the pages that it
    writes are the same again; weights go on adding up."""
    if own:
        return _run_own(state)
    c = state["case"]
    kind = c["kind"]
    if kind == "rotate":
        return {"q": _plain_rotate(state, state["q"]), "k": _plain_rotate(state, state["k"])}
    if kind == "evict":
        return _plain_evict(state)
    if kind == "attn":
        return _plain_attention(state, state["n"], state["q"])
    _plain_append(state)
    result = {"k_pages": state["k_pages"], "v_pages": state["v_pages"]}
    if kind == "step":
        q = _plain_rotate(state, state["q"][:, :, None])[:, :, 0] if c["dims"] else state["q"]
        result.update(_plain_attention(state, state["n"] + 1, q))
    return result


# ---- what a pass cannot do without -----------------------------------------------------------
def work(case):
    c = case
    B, Hq, Hkv, d, kind = (c[x] for x in ("B", "Hq", "Hkv", "d", "kind"))
    lengths = _lengths(c)
    angles = 8 * (c["dims"] // 2)
    if kind == "rotate":
        rows = B * c["L"] * (Hq + Hkv)
        return {"bytes": 4 * d * rows + 4 * B * c["L"] + angles, "flops": 3 * c["dims"] * rows}
    nbytes, flops = angles, 0
    for b, n in enumerate(lengths):
        if kind in ("write", "token", "step"):
            new = n if kind == "write" else 1
            nbytes += Hkv * new * 8 * d + 4 * (_pages(c, new) + new * (c["dims"] > 0))
            flops += 3 * c["dims"] * Hkv * new
        if kind in ("attn", "step"):
            all_of = n + (kind == "step")
            seen = min(all_of, c["window"] or all_of)
            nbytes += Hkv * 4 * d * (seen - (kind == "step")) + 4 * _pages(c, seen) + 4 * Hq * d
            nbytes += 8 * Hkv * seen if c["weighted"] else 0
            flops += 4 * Hq * d * seen
        if kind == "evict" and n > c["keep"]:
            nbytes += Hkv * (4 * n + 4 * c["keep"] + 8 * d * c["keep"]) + 4 * (_pages(c, n) + _pages(c, c["keep"]))
    return {"bytes": nbytes, "flops": flops}


# ---- the definition in 64 bits -----------------------------------------------------------------
def _exact_turn(c, x, positions):
    """x [..][L][d] in 64 bits: every pair as a complex number times e^(i position freq)."""
    dims = c["dims"]
    angle = positions.double()[:, None] * torch.tensor(_frequencies(c), dtype=torch.float64, device=DEVICE)
    first = torch.arange(dims // 2, device=DEVICE) * (2 if c["interleaved"] else 1)
    second = first + (1 if c["interleaved"] else dims // 2)
    x = x.double().clone()
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones_like(angle), angle)
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_rows(state, which, b, h, n, spare=0):
    """Addresses [n][d] in the pool of what row b has in its first n slots."""
    c = state["case"]
    t = torch.arange(n, device=DEVICE)
    page = torch.tensor(state["ids"][spare][b], dtype=torch.long, device=DEVICE)[t // c["P"]]
    inside = PLACES[which]((t % c["P"])[:, None], torch.arange(c["d"], device=DEVICE)[None], c["d"])
    return (page * c["Hkv"] + h)[:, None] * (c["P"] * c["d"]) + inside


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    c = case
    B, Hq, Hkv, d, kind = (c[x] for x in ("B", "Hq", "Hkv", "d", "kind"))
    if kind == "rotate":
        return {w: torch.stack([_exact_turn(c, state[w][b], state["positions"][b]) for b in range(B)]) for w in "qk"}
    lengths = state["lengths"]
    result = {}
    pools = {w: state[w + "_pages"].double() for w in "kv"}
    flat = {w: pools[w].view(-1) for w in "kv"}
    if kind in ("write", "token", "step"):
        for b, n in enumerate(lengths):
            new = n if kind == "write" else 1
            for w in "kv":
                x = state[w + "_new"][b, :, :new].double()
                if w == "k" and c["dims"] and new:
                    x = _exact_turn(c, x, state["positions"][b, :new])
                for h in range(Hkv):
                    flat[w][_exact_rows(state, w, b, h, n if kind == "write" else n + 1)[-new:] if new else torch.zeros((0, d), dtype=torch.long, device=DEVICE)] = x[h]
    if kind != "attn":
        result = {w + "_pages": pools[w] for w in "kv"}
    weights = state["weights"].double() if c["weighted"] else None
    if kind in ("attn", "step"):
        out = torch.zeros((B, Hq, d), dtype=torch.float64, device=DEVICE)
        gh = Hq // Hkv
        for b, n in enumerate(_after(c)):
            q = state["q"][b].double()
            if kind == "step" and c["dims"]:
                q = _exact_turn(c, q[:, None], state["positions"][b, :1])[:, 0].to(TYPES[c["dtype"]]).double()
            first = max(0, n - c["window"]) if c["window"] else 0
            if kind == "step" and weights is not None:
                weights[0, b, :, n - 1] = 0.0
            for h in range(Hkv if n else 0):
                at = slice(h * gh, (h + 1) * gh)
                # (what attends and is attended to are values of the cache's type, those of the call's own turned key too)
                k, v = (flat[w][_exact_rows(state, w, b, h, n)[first:]].to(TYPES[c["dtype"]]).double() for w in "kv")
                s = torch.matmul(q[at], k.t().contiguous()) / math.sqrt(d)
                if c["cap"]:
                    s = torch.tanh(s / c["cap"]) * c["cap"]
                if c["bias"]:
                    s = s + state["slopes"][at, None].double() * (torch.arange(first, n, device=DEVICE) - (n - 1))
                p = torch.softmax(s, -1)
                out[b, at] = torch.matmul(p, v)
                if weights is not None:
                    weights[0, b, h, first:n] += p.sum(0)
        result["out"] = out
    if kind == "evict":
        keep, recent = c["keep"], c["recent"]
        for b in _evicted(c):
            n = lengths[b]
            for h in range(Hkv):
                w = weights[0, b, h, :n - recent]
                count = keep - recent
                if count:
                    border = torch.topk(w, count).values[-1]
                    over, equal = w > border, w == border
                    chosen = over | (equal & (equal.cumsum(0) <= count - over.sum()))
                else:
                    chosen = torch.zeros_like(w, dtype=torch.bool)
                kept = torch.cat([chosen.nonzero()[:, 0], torch.arange(n - recent, n, device=DEVICE)])
                weights[1, b, h, :keep] = weights[0, b, h, kept]
                for x in "kv":
                    flat[x][_exact_rows(state, x, b, h, keep, spare=1)] = flat[x][_exact_rows(state, x, b, h, n)[kept]]
    if weights is not None:
        result["weights"] = weights
    return result
