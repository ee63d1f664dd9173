"""Performance cases of the 4-bit cache: appending to it, attending over it, managing its pages.

What a program does with the cache between two prompts: it quantises the keys and values of new tokens into
pages, attends from the newest tokens over all that a sequence holds, branches sequences (beams, samples of
one prompt) by sharing their pages, and packs the pool when many sequences have left it.  Kinds:

  append   sa_cache_append, then sa_cache_read of the same tokens: what later steps will see of them
  attend   sa_cache_attend
  branch   sa_cache_free, sa_cache_fork, sa_cache_reserve: sequences leave, others branch, all get room
  compact  sa_cache_compact

The cache: ``pool`` is uint8 [layers, pages, Hkv, 2, P * (d/2 + d/16)].  A page holds P tokens; for each KV head and
side (0 = K, 1 = V) first P rows of d/2 bytes of codes (dimension 2i in the low half of byte i), then P rows of d/16
scale bytes.  A value is e2m1(code) * e4m3(scale) * t with a power of two t for each side.  ``table`` is int32
[slots, row]: the pages of a sequence in order, -1 where it holds none; ``lens`` int32 [slots] its tokens; ``refs``
int32 [pages] how many table entries name a page.

``listed()`` names the sizes; ``draw()`` gives further ones of the same kinds and ranges.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # One token each of 64 running sequences, 8 KV heads of 128 (configuration 3's heads): every decode step.
        dict(name="append_step_64", kind="append", dtype="bf16", B=64, T=1, Hkv=8, d=128, P=64, past=4000, ragged=False, token_major=True, k_log2=-4, v_log2=-4),
        # Four prompts of uneven length in fp32, 12 heads of 64 (the pre-training model's attention), cache empty.
        dict(name="append_prompts_f32", kind="append", dtype="f32", B=4, T=2047, Hkv=12, d=64, P=32, past=0, ragged=True, token_major=False, k_log2=-4, v_log2=-5),
        # The keys and values of a 32768-token prompt after its prefill: the largest append.
        dict(name="append_prompt_32k", kind="append", dtype="bf16", B=1, T=32768, Hkv=8, d=128, P=64, past=0, ragged=False, token_major=False, k_log2=-4, v_log2=-4),
        # One user's next token after a short prompt (32/8 heads of 128): latency is everything.
        dict(name="attend_700", kind="attend", dtype="bf16", B=1, T=1, Hq=32, Hkv=8, d=128, P=64, keys=700, ragged=False, w=0, causal=True, k_log2=-4, v_log2=-4),
        # A serving batch of 64 sequences of very uneven length: the ordinary decode step.
        dict(name="attend_batch_64", kind="attend", dtype="bf16", B=64, T=1, Hq=32, Hkv=8, d=128, P=64, keys=8191, ragged=True, w=0, causal=True, k_log2=-4, v_log2=-4),
        # One sequence of 131072 tokens, 32/4 heads (configuration 4's prompt): few rows, one long axis.
        dict(name="attend_131072", kind="attend", dtype="bf16", B=1, T=1, Hq=32, Hkv=4, d=128, P=64, keys=131072, ragged=False, w=0, causal=True, k_log2=-4, v_log2=-4),
        # A chunk of new tokens over the cached prefix in fp32, 16 heads of 64: joined with the chunk's own attention through lse.
        dict(name="attend_prefix_f32", kind="attend", dtype="f32", B=9, T=37, Hq=16, Hkv=16, d=64, P=16, keys=2500, ragged=True, w=0, causal=False, k_log2=-4, v_log2=-4),
        # 32 sequences of 32768 tokens, 32/8 heads: the largest step.
        dict(name="attend_32x32768", kind="attend", dtype="bf16", B=32, T=1, Hq=32, Hkv=8, d=128, P=128, keys=32768, ragged=False, w=0, causal=True, k_log2=-4, v_log2=-4),
        # Two more samples of one prompt, 12 layers (the pre-training model): books and a few pages.
        dict(name="branch_3_samples", kind="branch", layers=12, Hkv=12, d=64, P=32, slots=8, row=64, pages=512, keys=1500, parents=1, children=2, leave=2),
        # Beams of 64 sequences, three children each, through 24 layers: every child and parent writes next.
        dict(name="branch_64x4_beams", kind="branch", layers=24, Hkv=8, d=128, P=64, slots=512, row=64, pages=3000, keys=1900, parents=64, children=3, leave=100),
        # A small pool after one of its sequences left.
        dict(name="compact_small", kind="compact", layers=4, Hkv=4, d=128, P=16, slots=8, row=32, pages=250, live=120, moves=35),
        # A large pool packed after half of its sequences left: the largest move of pages.
        dict(name="compact_large", kind="compact", layers=12, Hkv=8, d=128, P=64, slots=256, row=64, pages=8000, live=4100, moves=2000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "append", "attend", "attend", "attend", "branch", "compact"))
    d = rng.choice((64, 64, 128, 128, 128, 256, 96, 80))
    P = rng.choice((16, 32, 64, 64, 128))
    scales = dict(k_log2=rng.choice((-5, -4, -3)), v_log2=rng.choice((-6, -5, -4)))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind == "append":
        Hkv = rng.choice((1, 2, 4, 8, 12, 16))
        most = 32768 * 8 * 128 // (Hkv * d)
        B = _log(rng, 1, 200)
        T = _log(rng, 1, max(1, min(40000, most // B))) if rng.random() < 0.7 else 1
        return dict(kind=kind, dtype=dtype, B=B, T=T, Hkv=Hkv, d=d, P=P, past=_log(rng, 1, 5000) - 1,
                    ragged=rng.random() < 0.5, token_major=rng.random() < 0.5, **scales)
    if kind == "attend":
        Hkv = rng.choice((1, 2, 4, 8, 12))
        G = rng.choice((1, 2, 4, 5, 8, 16))
        T = 1 if rng.random() < 0.6 else _log(rng, 2, 48)
        B = _log(rng, 1, 200)
        # Bounded by keys, and by rows times keys, whichever the plain form's memory feels first.
        most = min(32 * 32768 * 8 * 128 // (B * Hkv * d), (1 << 29) // (B * Hkv * G * T))
        keys = _log(rng, 1, max(1, min(131072, most)))
        return dict(kind=kind, dtype=dtype, B=B, T=T, Hq=Hkv * G, Hkv=Hkv, d=d, P=P, keys=keys,
                    ragged=rng.random() < 0.6, w=_log(rng, 1, 4096) if rng.random() < 0.3 else 0,
                    causal=rng.random() < 0.7, **scales)
    Hkv, layers = rng.choice((1, 2, 4, 8)), rng.randint(1, 24)
    page = layers * Hkv * 2 * P * (d // 2 + d // 16)
    most = max(64, min(20000, (3 << 30) // page))
    if kind == "branch":
        parents, children, row = _log(rng, 1, 48), rng.randint(1, 4), _log(rng, 8, 100)
        leave = rng.randint(0, 60)
        pages = parents * (row + children + 1) + leave * row + 20
        if pages > most:
            parents, leave, row = 1, 2, 8
            pages = parents * (row + children + 1) + leave * row + 20
        return dict(kind=kind, layers=layers, Hkv=Hkv, d=d, P=P, slots=parents * (children + 1) + leave + rng.randint(0, 30),
                    row=row, pages=pages, keys=rng.randint(2, (row - 1) * P), parents=parents, children=children, leave=leave)
    pages = _log(rng, 60, most)
    live, slots = rng.randint(pages // 4, 3 * pages // 4), _log(rng, 1, 256)
    row = -(-live // slots) + rng.randint(0, 50)
    return dict(kind=kind, layers=layers, Hkv=Hkv, d=d, P=P, slots=slots, row=row, pages=pages,
                live=live, moves=rng.randint(0, min(live, pages - live)))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _kv(shape, dtype, gen):
    """Keys (a few channels stand out, as they do after training) and values, [B, Hkv, n, d]."""
    k = torch.randn(shape, generator=gen, device="cuda")
    k = k * (1 + 3 * (torch.rand(1, shape[1], 1, shape[3], generator=gen, device="cuda") < 0.05))
    v = torch.randn(shape, generator=gen, device="cuda") * 0.7
    return k.to(dtype), v.to(dtype)


def _quantise(x, t):
    """Codes (uint8 [..., d/2]) and scales (uint8 [..., d/16]) of x [..., d]."""
    y = x.float() / t
    y = y.reshape(*y.shape[:-1], -1, 16)
    s = (y.abs().amax(-1, keepdim=True) / 6).clamp(max=448).to(torch.float8_e4m3fn)
    f = s.float()
    q = torch.where(f > 0, y.abs() / f, 0)
    c = (q > 0.25).to(torch.uint8) + (q >= 0.75) + (q > 1.25) + (q >= 1.75) + (q > 2.5) + (q >= 3.5) + (q > 5)
    c = (c + 8 * (y < 0)).to(torch.uint8).reshape(x.shape)
    return c[..., ::2] | (c[..., 1::2] << 4), s.view(torch.uint8).reshape(*x.shape[:-1], -1)


def _dequantise(codes, scales, t):
    """fp32 [..., d] of what codes and scales stand for."""
    lut = torch.tensor(E2M1 + tuple(-e for e in E2M1), device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).to(torch.int32)
    v = lut[c].reshape(*scales.shape, 16)
    return (v * (scales.view(torch.float8_e4m3fn).float() * t).unsqueeze(-1)).flatten(-2)


def _sides(pool, P, d):
    """Views of a layer's codes [pages, Hkv, 2, P, d/2] and scales [pages, Hkv, 2, P, d/16]."""
    at = P * d // 2
    return pool[..., :at].unflatten(-1, (P, d // 2)), pool[..., at:].unflatten(-1, (P, d // 16))


def _room(slots, need, row, gen):
    """A table [slots, row] that gives slot b need[b] pages in random order, and how many pages that takes."""
    held = torch.arange(row, device="cuda") < need.unsqueeze(1)
    total = int(held.sum())
    pages = total + 3
    table = torch.full((slots, row), -1, dtype=torch.int32, device="cuda")
    table[held] = torch.randperm(pages, generator=gen, device="cuda")[:total].int()
    return table, pages


def _prepare_append(c, gen):
    B, T, P, d = c["B"], c["T"], c["P"], c["d"]
    dtype = DTYPES[c["dtype"]]
    slots = B + 2
    lens = torch.randint(0, c["past"] + 1, (slots,), generator=gen, device="cuda", dtype=torch.int32)
    counts = torch.full((B,), T, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        counts = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    row = (c["past"] + T + P - 1) // P
    table, pages = _room(slots, (lens.long() + T + P - 1) // P, row, gen)
    pool = torch.zeros(1, pages, c["Hkv"], 2, P * (d // 2 + d // 16), dtype=torch.uint8, device="cuda")
    k, v = _kv((B, c["Hkv"], T, d), dtype, gen)
    if c["token_major"]:
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    ids = torch.randperm(slots, generator=gen, device="cuda")[:B].int()
    return dict(pool=pool, table=table, lens=lens, slots=ids, starts=lens[ids.long()], counts=counts, k=k, v=v,
                k_out=torch.zeros_like(k), v_out=torch.zeros_like(v))


def _prepare_attend(c, gen):
    B, T, P, d, Hkv = c["B"], c["T"], c["P"], c["d"], c["Hkv"]
    dtype = DTYPES[c["dtype"]]
    most = c["keys"]
    total = torch.full((B,), most, dtype=torch.int32, device="cuda")
    if c["ragged"]:
        total = torch.randint(0, most + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    # The step's own tokens stand behind the lens that the cache had before it.
    lens = (total - T).clamp(min=0) if c["causal"] else total
    end = lens + T if c["causal"] else total
    row = (most + T + P - 1) // P
    table, pages = _room(B, (end.long() + P - 1) // P, row, gen)
    pool = torch.zeros(1, pages, Hkv, 2, P * (d // 2 + d // 16), dtype=torch.uint8, device="cuda")
    codes, scales = _sides(pool[0], P, d)
    for at in range(0, pages, 1 << 10):
        m = min(pages, at + (1 << 10)) - at
        k, v = _kv((m, Hkv, P, d), dtype, gen)
        for side, x, t in ((0, k, c["k_log2"]), (1, v, c["v_log2"])):
            codes[at:at + m, :, side], scales[at:at + m, :, side] = _quantise(x, 2.0 ** t)
    q = torch.randn(B, c["Hq"], T, d, generator=gen, device="cuda").to(dtype)
    return dict(pool=pool, table=table, lens=lens, q=q)


def _pages(c, table, lens, refs, gen):
    size = (c["layers"], c["pages"], c["Hkv"], 2, c["P"] * (c["d"] // 2 + c["d"] // 16))
    pool = torch.randint(0, 256, size, generator=gen, device="cuda", dtype=torch.uint8)
    return dict(pool=pool, table=table, lens=lens, refs=refs)


def _prepare_branch(c, gen):
    S, P, row, n = c["slots"], c["P"], c["row"], c["parents"]
    ids = torch.randperm(S, generator=gen, device="cuda").int()
    parents, children = ids[:n], ids[n:n * (c["children"] + 1)]
    leave = ids[n * (c["children"] + 1):][:c["leave"]]
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    some = torch.cat((parents, leave)).long()
    drawn = torch.randint(1, c["keys"] + 1, (len(some),), generator=gen, device="cuda", dtype=torch.int32)
    lens[some] = torch.where(drawn % P == 0, drawn - 1, drawn)          # last pages are part full
    need = (lens.long() + P - 1) // P
    held = torch.arange(row, device="cuda") < need.unsqueeze(1)
    table = torch.full((S, row), -1, dtype=torch.int32, device="cuda")
    table[held] = torch.randperm(c["pages"], generator=gen, device="cuda")[:int(held.sum())].int()
    refs = torch.zeros(c["pages"], dtype=torch.int32, device="cuda")
    refs[table[held].long()] = 1
    add = torch.zeros(S, dtype=torch.int32, device="cuda")
    add[torch.cat((parents, children)).long()] = 1
    return _pages(c, table, lens, refs, gen) | dict(
        leave=leave, parents=parents.repeat(c["children"]), children=children, add=add)


def _prepare_compact(c, gen):
    n, live, m, row = c["pages"], c["live"], c["moves"], c["row"]
    refs = torch.zeros(n, dtype=torch.int32, device="cuda")
    low, high = (torch.randperm(k, generator=gen, device="cuda") for k in (live, n - live))
    refs[low[m:]] = 1
    refs[live + high[:m]] = 1
    held = torch.nonzero(refs).flatten()
    held = held[torch.randperm(live, generator=gen, device="cuda")]
    table = torch.full((c["slots"] * row,), -1, dtype=torch.int32, device="cuda")
    table[:live] = held.int()
    return _pages(c, table.view(c["slots"], row), torch.zeros(c["slots"], dtype=torch.int32, device="cuda"), refs, gen)


def prepare(case, seed):
    make = dict(append=_prepare_append, attend=_prepare_attend, branch=_prepare_branch, compact=_prepare_compact)
    return make[case["kind"]](case, _gen(seed)) | dict(case=case)


def _plain_append(s):
    c = s["case"]
    P, d, T = c["P"], c["d"], c["T"]
    t = torch.arange(T, device="cuda")
    pos = s["starts"].long().unsqueeze(1) + t
    real = t < s["counts"].unsqueeze(1)                                  # [B, T]
    page = s["table"][s["slots"].long()].long().gather(1, pos.div(P, rounding_mode="floor"))
    codes, scales = _sides(s["pool"][0], P, d)
    b, i = real.nonzero(as_tuple=True)
    at, rows = page[b, i], pos[b, i] % P
    k, v = (_quantise(s[x][b, :, i], 2.0 ** c[x + "_log2"]) for x in "kv")
    codes[at, :, 0, rows], scales[at, :, 0, rows] = k
    codes[at, :, 1, rows], scales[at, :, 1, rows] = v
    s["k_out"][b, :, i] = _dequantise(codes[at, :, 0, rows], scales[at, :, 0, rows], 2.0 ** c["k_log2"]).to(s["k"].dtype)
    s["v_out"][b, :, i] = _dequantise(codes[at, :, 1, rows], scales[at, :, 1, rows], 2.0 ** c["v_log2"]).to(s["v"].dtype)
    return s["k_out"], s["v_out"]


def _visible(c, lens, n):
    """[B, T, n]: which of n cached keys each new token sees."""
    pos = lens.long().unsqueeze(1) + torch.arange(c["T"], device="cuda")
    j = torch.arange(n, device="cuda")
    last = pos if c["causal"] else (lens.long() - 1).unsqueeze(1).expand_as(pos)
    seen = j <= last.unsqueeze(2)
    return seen & (pos.unsqueeze(2) - j < c["w"]) if c["w"] else seen


def _plain_attend(s):
    c = s["case"]
    B, T, Hq, Hkv, d, P = (c[x] for x in ("B", "T", "Hq", "Hkv", "d", "P"))
    row = s["table"].shape[1]
    pages = s["pool"][0][s["table"].clamp(min=0).long()]                 # [B, row, Hkv, 2, bytes]
    codes, scales = (x.permute(3, 0, 2, 1, 4, 5).flatten(3, 4) for x in _sides(pages, P, d))
    k = _dequantise(codes[0], scales[0], 2.0 ** c["k_log2"])             # [B, Hkv, row P, d]
    q = s["q"].float().view(B, Hkv, Hq // Hkv * T, d)
    x = torch.matmul(q, k.transpose(2, 3)).view(B, Hkv, Hq // Hkv, T, row * P) / math.sqrt(d)
    del k
    seen = _visible(c, s["lens"], row * P).view(B, 1, 1, T, row * P)
    x = x.masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0, m))
    total = p.sum(-1, keepdim=True)
    v = _dequantise(codes[1], scales[1], 2.0 ** c["v_log2"])
    y = torch.matmul(p.view(B, Hkv, Hq // Hkv * T, row * P), v).view(B, Hkv, Hq // Hkv, T, d)
    y = torch.where(total > 0, y / total, 0).reshape(B, Hq, T, d).to(s["q"].dtype)
    return y, (m + torch.log(total)).reshape(B, Hq, T)


def _plain_branch(s):
    c = s["case"]
    P, row = c["P"], c["row"]
    pool, table, lens, refs = s["pool"], s["table"].clone(), s["lens"].clone(), s["refs"].clone()
    j = torch.arange(row, device="cuda")
    # free
    gone = table[s["leave"].long()]
    refs.index_add_(0, gone.clamp(min=0).flatten().long(), -(gone >= 0).int().flatten())
    table[s["leave"].long()] = -1
    lens[s["leave"].long()] = 0
    # fork
    a, b = s["parents"].long(), s["children"].long()
    rows = torch.where(j < ((lens[a] + P - 1) // P).unsqueeze(1), table[a], -1)
    table[b], lens[b] = rows, lens[a]
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), (rows >= 0).int().flatten())
    # reserve
    need = torch.where(s["add"] > 0, (lens + s["add"] + P - 1) // P, 0).unsqueeze(1)
    shared = (table >= 0) & (refs[table.clamp(min=0).long()] > 1)
    take = (j >= (lens // P).unsqueeze(1)) & (j < need) & ((table < 0) | shared)
    want = take.sum(1)
    free = (refs == 0).nonzero().flatten()
    got = (want.cumsum(0) <= len(free)) & (need.flatten() <= row)
    b, i = (take & got.unsqueeze(1)).nonzero(as_tuple=True)
    new, old = free[:len(b)], table[b, i].long()
    filled = (old >= 0) & (i * P < lens[b])
    pool[:, new[filled]] = pool[:, old[filled]]
    refs.index_add_(0, old.clamp(min=0), -(old >= 0).int())
    refs[new] = 1
    table[b, i] = new.int()
    return pool, table, lens, refs, (got | (want == 0) & (need.flatten() <= row)).int()


def _plain_compact(s):
    pool, table, refs = s["pool"], s["table"], s["refs"]
    live = refs > 0
    n = live.sum(dtype=torch.int32)
    index = torch.arange(len(refs), device="cuda")
    holes, movers = ((~live) & (index < n)).nonzero().flatten(), (live & (index >= n)).nonzero().flatten()
    pool[:, holes] = pool[:, movers]
    to = index.clone()
    to[movers] = holes
    new = refs.clone()
    new[holes], new[movers] = refs[movers], 0
    return pool, torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table), new, n.view(1)


def _own_run(s):
    from paper_2604_00754_b200 import binding as sa
    c = s["case"]
    if c["kind"] == "append":
        t = dict(k_scale=2.0 ** c["k_log2"], v_scale=2.0 ** c["v_log2"])
        sa.sa_cache_append(s["pool"], s["table"], s["lens"], s["k"], s["v"], slots=s["slots"], counts=s["counts"], **t)
        return sa.sa_cache_read(s["pool"], s["table"], s["k_out"], s["v_out"], slots=s["slots"], starts=s["starts"],
                                counts=s["counts"], **t)
    if c["kind"] == "attend":
        return sa.sa_cache_attend(s["pool"], s["table"], s["lens"], s["q"], w=c["w"], flags=sa.CAUSAL if c["causal"] else 0,
                                  k_scale=2.0 ** c["k_log2"], v_scale=2.0 ** c["v_log2"], want_lse=True)
    table, refs = s["table"].clone(), s["refs"].clone()
    if c["kind"] == "branch":
        lens = s["lens"].clone()
        sa.sa_cache_free(table, lens, refs, s["leave"])
        sa.sa_cache_fork(table, lens, refs, s["parents"], s["children"], page=c["P"])
        got = sa.sa_cache_reserve(s["pool"], table, lens, refs, s["add"], page=c["P"])
        return s["pool"], table, lens, refs, got
    live = sa.sa_cache_compact(s["pool"], table, refs)
    return s["pool"], table, refs, live


def run(state):
    if own:
        return _own_run(state)
    plain = dict(append=_plain_append, attend=_plain_attend, branch=_plain_branch, compact=_plain_compact)
    return plain[state["case"]["kind"]](state)


def _mean_keys(c):
    """Visible keys of one new token, averaged over sequences and tokens, and cached keys that any of them sees."""
    total = c["keys"] / 2 if c["ragged"] else c["keys"]
    seen = max(1.0, total - (c["T"] - 1) / 2) if c["causal"] else total
    if c["w"]:
        return min(seen, c["w"]), min(total, c["w"] + c["T"] - 1)
    return seen, max(total, 1.0) if c["causal"] else total


def work(case):
    c = case
    packed = 2 * (c["d"] // 2 + c["d"] // 16)                            # a token's K and V, one head
    if c["kind"] == "append":
        tokens = c["B"] * c["T"] * (0.5 if c["ragged"] else 1.0) * c["Hkv"]
        elt = 2 if c["dtype"] == "bf16" else 4
        # Read in the run's type and written packed, then read packed and written in the run's type.
        return {"bytes": tokens * 2 * (2 * c["d"] * elt + packed), "flops": tokens * 2 * c["d"] * 4.0}
    if c["kind"] == "attend":
        elt = 2 if c["dtype"] == "bf16" else 4
        seen, read = _mean_keys(c)
        rows = c["B"] * c["Hq"] * c["T"]
        return {"bytes": c["B"] * c["Hkv"] * read * packed + rows * (2 * c["d"] * elt + 4), "flops": 4.0 * rows * seen * c["d"]}
    page = c["layers"] * c["Hkv"] * c["P"] * packed
    if c["kind"] == "branch":
        copies = c["parents"] * (c["children"] + 1)
        return {"bytes": 2.0 * page * copies + 8.0 * (c["slots"] * (c["row"] + 1) + c["pages"]), "flops": float(c["slots"] * c["row"])}
    return {"bytes": 2.0 * page * c["moves"] + 8.0 * (c["slots"] * c["row"] + c["pages"]), "flops": float(c["pages"])}


def _exact_values(codes, scales, t):
    """Float64 values, from the formats' definitions: sign, two exponent bits and one of mantissa (bias 1); sign, four
    exponent bits and three of mantissa (bias 7)."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    e, m = c % 8 // 2, (c % 2).double()
    x = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2((e - 1).double())) * (1 - 2 * (c // 8))
    b = scales.long()
    e, m = b % 128 // 8, (b % 8).double()
    s = torch.where(e == 0, m / 512, (1 + m / 8) * torch.exp2((e - 7).double()))
    return x * s.repeat_interleave(16, -1) * 2.0 ** t


def _exact_round(x, t):
    """x [..., d] as the cache gives it back: float64, by nearest entries of the formats' value lists."""
    grid = torch.tensor([0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device=x.device)   # even codes first
    b = torch.arange(0x7f, device=x.device)
    e, m = b // 8, (b % 8).double()
    list_ = torch.where(e == 0, m / 512, (1 + m / 8) * torch.exp2((e - 7).double()))
    y = x.double().unflatten(-1, (-1, 16)) / 2.0 ** t
    top = y.abs().amax(-1, keepdim=True) / 6
    at = torch.searchsorted(list_, top).clamp(max=126)
    below = (at - 1).clamp(min=0)
    up, down = list_[at] - top, top - list_[below]
    s = torch.where((up < down) | (up == down) & (at % 2 == 0) | (top >= 448), list_[at], list_[below])
    q = torch.where(s > 0, y.abs() / s, 0)
    near = grid[(q.unsqueeze(-1) - grid).abs().argmin(-1)]
    return (near * s * torch.sign(y) * 2.0 ** t).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    P, d = c.get("P"), c.get("d")
    if c["kind"] == "append":
        real = torch.arange(c["T"], device="cuda") < s["counts"].view(-1, 1)
        out = []
        for x in "kv":
            y = torch.zeros(s[x].shape, dtype=torch.float64, device="cuda")
            step = max(1, (1 << 22) // (c["B"] * c["Hkv"] * d))
            for at in range(0, c["T"], step):
                y[:, :, at:at + step] = _exact_round(s[x][:, :, at:at + step], c[x + "_log2"])
            out.append(torch.where(real.view(c["B"], 1, -1, 1), y, 0))
        return tuple(out)
    if c["kind"] == "attend":
        B, T, Hq, Hkv = c["B"], c["T"], c["Hq"], c["Hkv"]
        y = torch.zeros(B, Hq, T, d, dtype=torch.float64, device="cuda")
        lse = torch.full((B, Hq, T), -math.inf, dtype=torch.float64, device="cuda")
        codes, scales = _sides(s["pool"][0], P, d)
        held = (s["table"] >= 0).sum(1).tolist()
        for b, n in enumerate(held):
            if not n:
                continue
            at = s["table"][b, :n].long()
            k, v = (_exact_values(codes[at, :, i], scales[at, :, i], c[x + "_log2"]).transpose(0, 1).reshape(Hkv, n * P, d)
                    for i, x in enumerate("kv"))
            j, pos = torch.arange(n * P, device="cuda"), s["lens"][b].long() + torch.arange(T, device="cuda").view(-1, 1)
            seen = (j <= pos) if c["causal"] else (j < s["lens"][b]).expand(T, -1)
            if c["w"]:
                seen = seen & (j > pos - c["w"])
            for h in range(Hq):
                x = s["q"][b, h].double() @ k[h * Hkv // Hq].T / math.sqrt(d)
                x = torch.where(seen, x, -math.inf)
                lse[b, h] = torch.logsumexp(x, -1)
                p = torch.exp(x - torch.where(lse[b, h] == -math.inf, 0, lse[b, h]).unsqueeze(-1))
                y[b, h] = p @ v[h * Hkv // Hq]
        return y, lse
    pool, lens = s["pool"], s["lens"].tolist()
    table, refs = s["table"].tolist(), s["refs"].tolist()
    moves = []
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    if c["kind"] == "compact":
        live = sum(r > 0 for r in refs)
        holes = [p for p in range(live) if refs[p] <= 0]
        moves = list(zip([p for p in range(live, len(refs)) if refs[p] > 0], holes))
        for old, new in moves:
            refs[new], refs[old] = refs[old], 0
        to = dict(moves)
        table = [[to.get(p, p) for p in r] for r in table]
    else:
        for b in s["leave"].tolist():
            for p in table[b]:
                if p >= 0:
                    refs[p] -= 1
            table[b], lens[b] = [-1] * c["row"], 0
        for a, b in zip(s["parents"].tolist(), s["children"].tolist()):
            n = -(-lens[a] // P)
            table[b], lens[b] = table[a][:n] + [-1] * (c["row"] - n), lens[a]
            for p in table[a][:n]:
                refs[p] += 1
        free = [p for p, r in enumerate(refs) if r == 0]
        before, used, got = list(refs), 0, []
        for b, more in enumerate(s["add"].tolist()):
            last = -(-(lens[b] + more) // P) if more else 0
            want = [j for j in range(lens[b] // P, min(last, c["row"])) if table[b][j] < 0 or before[table[b][j]] > 1]
            used += len(want)
            fits = last <= c["row"] and (not want or used <= len(free))
            got.append(int(fits))
            for k, j in enumerate(want if fits else []):
                new, old = free[used - len(want) + k], table[b][j]
                if old >= 0:
                    refs[old] -= 1
                    if j * P < lens[b]:
                        moves.append((old, new))
                refs[new], table[b][j] = 1, new
    for old, new in moves:
        pool[:, new] = pool[:, old]
    if c["kind"] == "compact":
        return pool, as_int(table), as_int(refs), as_int([live])
    return pool, as_int(table), as_int(lens), as_int(refs), as_int(got)
