"""Performance cases of the 4-bit paged cache: filling it from an eviction, growing it token by
token with the position rotation, attending over it, and reading it back.

A case is one pass of a serving program, on inputs and pages it already holds on the GPU:

  load     the eviction's compact cache (bf16 keys, 4-bit value codes and scales) into pages, and the
           loaded tokens read back
  append   new tokens' keys (rotated at their positions) and values into the pages, their queries
           rotated beside them, and the new tokens read back
  attend   causal attention of each sequence's newest tokens over its pages
  step     append, then attend: one decode step of a layer
  read     a range of every sequence's tokens read back as bf16 rows (to evict again)

The cache is one tensor of bytes [L][pages][Hkv][page_tokens / 32][block bytes].  A block holds 32
tokens of one head: the keys' codes (16 d bytes), the values' codes (16 d), the keys' scales (bf16, one
per token and group of 32 channels) and the values' scales (fp32, one per token).  A code c in [-7, 7]
is the 4-bit number c + 8; eight of them make a 32-bit word whose nibbles 0..7 hold elements
0, 2, 4, 6, 1, 3, 5, 7.  Keys: token t's row is d/8 words, word h * (d/32) + s holding channels
32 s + 8 h .. + 7.  Values: a word holds one channel of the eight tokens 4g .. 4g + 3, 16 + 4g ..
16 + 4g + 3; channel 16 j + m, tokens of g: word (j / 4) * 256 + (16 g + m) * 4 + j % 4.
"""
import math
import random

import torch

own = False

ORDER = [0, 2, 4, 6, 1, 3, 5, 7]  # the elements in nibbles 0..7
PLACE = [0, 4, 1, 5, 2, 6, 3, 7]  # the nibbles of elements 0..7


def _case(kind, Hq, Hkv, d, page, lens, new="1", L=1, first="0", rope="halves", table=0, name=None):
    c = {"kind": kind, "L": L, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "lens": lens, "new": new, "first": first,
         "rope": rope, "table": table}
    if name is not None:
        c["name"] = name
    return c


def _text(values):
    return ",".join(str(int(v)) for v in values)


def listed():
    r = random.Random(11)
    ragged = _text(int(math.exp(r.uniform(math.log(6000), math.log(32768)))) for _ in range(64))
    verify = [(r.randint(3000, 9000), r.randint(1, 8)) for _ in range(16)]
    return [
        # the smallest call: one sequence of a small model, bound by launches and latency
        _case("attend", 8, 2, 64, 32, "257", name="attend_tiny"),
        # decoding after a 128K prefill whose eviction kept a tenth, some tokens into the answer
        _case("attend", 32, 8, 128, 64, "13215", name="attend_kept_128k"),
        # a full serving batch of mixed lengths, 64 query heads: the bandwidth of the cache
        _case("attend", 64, 8, 128, 64, ragged, name="attend_ragged64"),
        # two very long sequences that were not evicted
        _case("attend", 64, 8, 128, 256, "262144,131073", name="attend_long"),
        # drafted tokens verified: 1 to 8 query tokens a sequence
        _case("attend", 32, 8, 128, 64, _text(a for a, _ in verify), _text(b for _, b in verify), name="attend_verify"),
        # the next part of a prompt in chunks, over a cache that is already in pages
        _case("attend", 32, 8, 128, 128, "17333,4096", "1024,300", name="attend_chunk"),
        # one decode step's append in a full batch
        _case("append", 32, 8, 128, 64, _text(r.randint(1, 2600) for _ in range(64)), table=131072, name="append_decode"),
        # a prompt's chunk written at once, pairs of neighbours rotated
        _case("append", 64, 8, 128, 64, "9011,4099", "8191,4099", rope="pairs", table=65536, name="append_chunk"),
        # every layer of an 8B model: the kept tenth of a 128K prefill into pages
        _case("load", 32, 8, 128, 64, "13107", L=32, name="load_kept_128k"),
        # a small model's batch under a budget of 512 tokens and shorter sequences
        _case("load", 8, 2, 64, 32, "512,512,77,512,301,1", L=4, name="load_budget_small"),
        # the tokens of a long answer read back to be evicted again
        _case("read", 32, 8, 128, 64, "20011,6000,12345", L=8, first="6553,2048,0", name="read_answers"),
        # one decode step of a layer: append and attention under a budget of 2048 and what was answered since
        _case("step", 32, 8, 128, 64, _text(2048 + r.randint(1, 500) for _ in range(32)), table=131072,
              name="step_budget_2048"),
    ]


def draw(rng):
    """A case of the same kinds over the same ranges; lengths log-uniform."""
    def logint(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        kind = rng.choice(["attend"] * 5 + ["append", "append", "load", "read", "step", "step"])
        Hq, Hkv, d = rng.choice([(8, 2, 64), (32, 8, 128), (32, 8, 128), (64, 8, 128), (16, 2, 128), (12, 4, 64), (5, 5, 128)])
        B = logint(1, 64)
        top = logint(100, 262144)
        lens = [top] + [logint(max(1, top // 8), top) for _ in range(B - 1)]
        new = [1] * B
        how = rng.random()
        if kind in ("attend", "append", "step") and how < 0.5:
            most = logint(2, 16) if how < 0.3 else logint(17, 1500)
            new = [min(n, rng.randint(1, most)) for n in lens]
        L = logint(1, 32) if kind in ("load", "read") else 1
        first = [rng.randint(0, n - 1) if rng.random() < 0.5 else 0 for n in lens] if kind == "read" else [0]
        c = _case(kind, Hq, Hkv, d, rng.choice([32, 64, 128, 256]), _text(lens), _text(new), L, _text(first),
                  rng.choice(["halves", "halves", "pairs"]), rng.choice([32768, 131072]) if kind in ("append", "step") else 0)
        w = work(c)
        # no dearer than the largest listed case, and the plain form's padded scores and keys fit
        if (w["bytes"] <= 1.2e9 and w["flops"] <= 3.0e11 and len(lens) * max(lens) * Hkv * d <= 64 * 32768 * 8 * 128
                and len(lens) * max(lens) * max(new) * Hq <= 2.0e9):
            return c


# ------------------------------------------------------------------------------ inputs
def _ints(text):
    return [int(x) for x in text.split(",")]


def _offsets(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _new(c):
    n = _ints(c["new"])
    return n * len(_ints(c["lens"])) if len(n) == 1 else n


def _first(c):
    n = _ints(c["first"])
    return n * len(_ints(c["lens"])) if len(n) == 1 else n


def _block_bytes(d):
    return 32 * (d + d // 16 + 4)


def _keys(shape, g):
    """Keys: normal, with channels of different strength."""
    strength = torch.empty(shape[-1], device="cuda").normal_(0.0, 0.5, generator=g).exp_()
    return torch.empty(shape, device="cuda").normal_(generator=g).mul_(strength).to(torch.bfloat16)


def _values(shape, g):
    """Values: normal, one token in 200 an outlier 20 times larger."""
    far = torch.rand(shape[:-1] + (1,), device="cuda", generator=g) < 0.005
    return torch.empty(shape, device="cuda").normal_(generator=g).mul_(torch.where(far, 20.0, 1.0)).to(torch.bfloat16)


def _cos_sin(positions, r):
    """fp32 [positions][r]: the cosines of r / 2 angles, then their sines."""
    freq = 500000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    L, Hq, Hkv, d, page = c["L"], c["Hq"], c["Hkv"], c["d"], c["page"]
    lens, new, first = _ints(c["lens"]), _new(c), _first(c)
    B, per = len(lens), page // 32
    need = [-(-n // page) for n in lens]
    num_pages = sum(need) + 3
    order = torch.randperm(num_pages, device="cuda", generator=g)[:sum(need)].to(torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
    at = _offsets(need)
    for b in range(B):
        table[b, :need[b]] = order[at[b]:at[b + 1]]
    pages = torch.empty((L, num_pages, Hkv, per, _block_bytes(d)), dtype=torch.uint8, device="cuda")
    flat = pages.view(-1, _block_bytes(d))
    for i in range(0, flat.shape[0], 65536):  # the tokens that the pages hold, quantised as the operators do
        n = min(65536, flat.shape[0] - i)
        flat[i:i + n] = _pack(*_quantise_keys(_keys((n, 32, d), g)), *_quantise_values(_values((n, 32, d), g)))
    st = {"c": c, "pages": pages, "table": table, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
          "max_len": max(lens), "scale": 1.0 / math.sqrt(d)}

    def touched(start, stop):
        """The blocks that tokens start[b] .. stop[b] - 1 of the sequences lie in, and each token's place."""
        page_of, block_of, token_block, token_slot = [], [], [], []
        base = 0
        for b in range(B):
            j0, j1 = start[b] // 32, -(-stop[b] // 32)
            j = torch.arange(j0, j1, device="cuda")
            page_of.append(table[b, j // per].long())
            block_of.append(j % per)
            t = torch.arange(start[b], stop[b], device="cuda")
            token_block.append(t // 32 - j0 + base)
            token_slot.append(t % 32)
            base += j1 - j0
        st["blocks"] = torch.cat(page_of), torch.cat(block_of)
        st["tokens"] = torch.cat(token_block), torch.cat(token_slot)

    if c["kind"] == "load":
        n = sum(lens)
        st["offsets"] = _offsets(lens)
        st["k"] = _keys((L, Hkv, n, d), g)
        codes, st["v_scales"] = _quantise_values(_values((L, Hkv, n, d), g))
        st["v_codes"] = (codes[..., 0::2] & 15 | codes[..., 1::2] << 4).to(torch.uint8)  # two's complement, even element low
        touched([0] * B, lens)
    elif c["kind"] == "read":
        st["offsets"] = _offsets(n - f for n, f in zip(lens, first))
        st["first"] = first
        touched(first, lens)
    else:
        n = sum(new)
        st["offsets"] = _offsets(new)
        st["new_offsets"] = torch.tensor(st["offsets"], dtype=torch.int32, device="cuda")
        st["max_new"] = max(new)
        st["new_lens"] = torch.tensor(new, dtype=torch.int32, device="cuda")
        st["q"] = torch.empty((n, Hq, d), device="cuda").normal_(generator=g).to(torch.bfloat16)
        if c["kind"] != "attend":
            qkv = torch.empty((n, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")  # one projection's output
            qkv[:, :Hq] = st["q"]
            qkv[:, Hq:Hq + Hkv] = _keys((n, Hkv, d), g)
            qkv[:, Hq + Hkv:] = _values((n, Hkv, d), g)
            st["q"], st["k"], st["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            # a token's position counts what was evicted before it, so it is beyond its place in the cache
            pos = [torch.arange(t, device="cuda") + int(torch.randint(m, c["table"] - t, (1,), device="cuda", generator=g))
                   if c["table"] - t > m else torch.arange(t, device="cuda") + m - t for m, t in zip(lens, new)]
            st["positions"] = torch.cat(pos).to(torch.int32).clamp_(0, c["table"] - 1)
            st["cos_sin"] = _cos_sin(c["table"], d)
            touched([m - t for m, t in zip(lens, new)], lens)
        if c["kind"] != "append":
            back = torch.arange(max(new), device="cuda")
            start = torch.tensor(st["offsets"][:-1], device="cuda")
            st["rows"] = (start[:, None] + back).clamp_(max=n - 1)  # [B][max_new]: each padded row's query
            st["row_of"] = torch.cat([torch.arange(t, device="cuda") + b * max(new) for b, t in enumerate(new)])
    return st


# ------------------------------------------------------------------------------ the plain form
def _quantise_keys(k):
    """bf16 [..., d] -> codes int8 [..., d] and bf16 scales [..., d / 32], one per group of 32 channels."""
    x = k.float().unflatten(-1, (-1, 32))
    scale = (x.abs().amax(-1).double() / 7).float().to(torch.bfloat16)
    s = scale.float()[..., None]
    codes = torch.where(s > 0, torch.round(x / s), 0.0).clamp_(-7, 7)
    return codes.to(torch.int8).flatten(-2), scale


def _quantise_values(v):
    """bf16 [..., d] -> codes int8 [..., d] and fp32 scales [...]."""
    x = v.float()
    scale = (x.abs().amax(-1).double() / 7).float()
    s = scale[..., None]
    codes = torch.where(s > 0, torch.round(x / s), 0.0).clamp_(-7, 7)
    return codes.to(torch.int8), scale


def _words(codes):
    """int8 [..., 8] -> uint8 [..., 4]: eight codes in the nibbles of a word."""
    n = (codes + 8).to(torch.uint8)[..., ORDER]
    return n[..., 0::2] | n[..., 1::2] << 4


def _codes(words):
    """uint8 [..., 4] -> int8 [..., 8]."""
    return (torch.stack([words & 15, words >> 4], -1).flatten(-2)[..., PLACE].to(torch.int8)) - 8


def _pack(kc, ks, vc, vs):
    """Codes [..., 32, d] and scales [..., 32, d / 32], [..., 32] -> blocks [..., bytes]."""
    d = kc.shape[-1]
    lead = kc.shape[:-2]
    n = len(lead)
    k = _words(kc.reshape(*lead, 32, d // 32, 4, 8).transpose(-3, -2)).reshape(*lead, -1)
    v = vc.reshape(*lead, 2, 4, 4, d // 64, 4, 16)  # tokens (u, g, r), channels (j / 4, j % 4, m)
    v = v.permute(*range(n), n + 3, n + 1, n + 5, n + 4, n, n + 2)
    v = _words(v.flatten(-2)).reshape(*lead, -1)
    ks = ks.contiguous().view(torch.uint8).reshape(*lead, -1)
    vs = vs.contiguous().view(torch.uint8).reshape(*lead, -1)
    return torch.cat([k, v, ks, vs], -1)


def _unpack(blocks, d):
    """Blocks [..., bytes] -> codes int8 [..., 32, d], scales, codes, scales."""
    lead = blocks.shape[:-1]
    n = len(lead)
    k, v, ks, vs = blocks.split([16 * d, 16 * d, 2 * d, 128], -1)
    kc = _codes(k.reshape(*lead, 32, 4, d // 32, 4)).transpose(-3, -2).reshape(*lead, 32, d)
    vc = _codes(v.reshape(*lead, d // 64, 4, 16, 4, 4)).unflatten(-1, (2, 4))  # (j / 4, g, m, j % 4, u, r)
    vc = vc.permute(*range(n), n + 4, n + 1, n + 5, n, n + 3, n + 2).reshape(*lead, 32, d)
    return kc, ks.contiguous().view(torch.bfloat16).reshape(*lead, 32, d // 32), vc, vs.contiguous().view(torch.float32)


def _held(blocks, d):
    """Blocks -> the keys and values that they stand for, fp32 [..., 32, d]."""
    kc, ks, vc, vs = _unpack(blocks, d)
    return (kc.float().unflatten(-1, (-1, 32)) * ks.float()[..., None]).flatten(-2), vc.float() * vs[..., None]


def _blocks_first(pages):
    return pages.permute(1, 3, 0, 2, 4)  # [pages][blocks of a page][L][Hkv][bytes]


def _plain_write(st, kc, ks, vc, vs):
    """Tokens' codes [tokens][L][Hkv][..] into the pages; the rest of their blocks keeps what it holds."""
    view = _blocks_first(st["pages"])
    held = list(_unpack(view[st["blocks"]], st["c"]["d"]))
    block, slot = st["tokens"]
    for part, value in zip(held, (kc, ks, vc, vs)):
        part[block, :, :, slot] = value
    view[st["blocks"]] = _pack(*held)


def _plain_read(st):
    k, v = _held(_blocks_first(st["pages"])[st["blocks"]], st["c"]["d"])
    block, slot = st["tokens"]
    return {name: x[block, :, :, slot].permute(1, 2, 0, 3).to(torch.bfloat16) for name, x in (("k", k), ("v", v))}


def _plain_rotate(st, x):
    """bf16 [tokens][heads][d] rotated by their positions: products in 64 bits, rounded once."""
    cs = st["cos_sin"][st["positions"].long()].double()[:, None]
    cos, sin = cs.chunk(2, -1)
    x = x.double()
    a, b = x.chunk(2, -1) if st["c"]["rope"] == "halves" else (x[..., 0::2], x[..., 1::2])
    p, q = a * cos - b * sin, b * cos + a * sin
    return (torch.cat([p, q], -1) if st["c"]["rope"] == "halves" else torch.stack([p, q], -1).flatten(-2)).to(torch.bfloat16)


def _plain_append(st):
    kc, ks = _quantise_keys(_plain_rotate(st, st["k"]))
    vc, vs = _quantise_values(st["v"])
    _plain_write(st, kc[:, None], ks[:, None], vc[:, None], vs[:, None])
    return _plain_rotate(st, st["q"])


def _plain_load(st):
    kc, ks = _quantise_keys(st["k"])
    low, high = (st["v_codes"] << 4).view(torch.int8) >> 4, st["v_codes"].view(torch.int8) >> 4
    vc = torch.stack([low, high], -1).flatten(-2)
    _plain_write(st, *(x.movedim(2, 0) for x in (kc, ks, vc, st["v_scales"])))


def _plain_attend(st, q):
    c = st["c"]
    B, d, Hkv, R, T = st["lens"].numel(), c["d"], c["Hkv"], c["Hq"] // c["Hkv"], st["rows"].shape[1]
    blocks = st["pages"][0][st["table"].long().clamp(min=0)]  # [B][pages][Hkv][blocks][bytes]
    k, v = (x.permute(0, 2, 1, 3, 4, 5).reshape(B, Hkv, -1, d) for x in _held(blocks, d))
    q = q[st["rows"]].float().reshape(B, T, Hkv, R, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * R, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(st["scale"]).view(B, Hkv, T, R, -1)
    seen = (st["lens"] - st["new_lens"])[:, None] + torch.arange(1, T + 1, device=x.device)  # [B][T]
    hidden = torch.arange(x.shape[-1], device=x.device) >= seen[:, None, :, None, None]
    x.masked_fill_(hidden, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp_(x.sub_(m))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.div_(total).view(B, Hkv, T * R, -1), v).view(B, Hkv, T, R, d)
    lse = (m + total.log())[..., 0]
    o = o.permute(0, 2, 1, 3, 4).reshape(B * T, c["Hq"], d)[st["row_of"]]
    lse = lse.permute(1, 3, 0, 2).reshape(c["Hq"], B * T)[:, st["row_of"]]
    return {"o": o.to(torch.bfloat16), "lse": lse}


# ------------------------------------------------------------------------------ the framework's calls
def _handles(st):
    """What a serving program keeps from step to step: dims, the cache's handle, output buffers, workspace."""
    from paper_2608_03276_amd import binding as B

    c = st["c"]
    h = {"B": B, "d": B.dims(c["L"], c["Hq"], c["Hkv"], c["d"])}
    h["cache"] = B.Cache(h["d"], st["pages"], st["table"], st["lens"], c["page"])
    n = st["offsets"][-1]
    if c["kind"] in ("load", "append", "read"):
        h["batch"] = B.Batch(st["offsets"])
        h["first"] = [m - t for m, t in zip(_ints(c["lens"]), _new(c))] if c["kind"] == "append" else st.get("first")
        h["k"] = torch.empty((c["L"], c["Hkv"], n, c["d"]), dtype=torch.bfloat16, device="cuda")
        h["v"] = torch.empty_like(h["k"])
    if c["kind"] in ("append", "attend", "step"):
        h["step"] = B.Step(n, st["max_new"], st["new_offsets"])
    if c["kind"] in ("append", "step"):
        h["rope"] = B.Rope(st["cos_sin"], c["d"], B.TP_ROPE_HALVES if c["rope"] == "halves" else B.TP_ROPE_PAIRS)
        h["q"] = torch.empty((n, c["Hq"], c["d"]), dtype=torch.bfloat16, device="cuda")
    if c["kind"] in ("attend", "step"):
        h["o"] = torch.empty((n, c["Hq"], c["d"]), dtype=torch.bfloat16, device="cuda")
        h["lse"] = torch.empty((c["Hq"], n), device="cuda")
        h["ws"] = torch.empty(B.tp_cache_workspace_size(h["d"], h["cache"], h["step"], st["max_len"]), dtype=torch.uint8,
                              device="cuda")
    return h


def _own_run(st):
    c = st["c"]
    h = st.get("handles") or st.setdefault("handles", _handles(st))
    B, d, cache = h["B"], h["d"], h["cache"]
    if c["kind"] == "load":
        B.tp_cache_load(d, cache, st["offsets"], st["k"], st["v_codes"], st["v_scales"], 4)
    if c["kind"] in ("append", "step"):
        B.tp_cache_append(d, cache, h["step"], st["k"], st["v"], st["positions"], h["rope"], st["q"], h["q"])
    if c["kind"] in ("load", "append", "read"):
        B.tp_cache_read(d, cache, h["batch"], h["k"], h["v"], h["first"])
        out = {"k": h["k"], "v": h["v"]}
        return {**out, "q": h["q"]} if c["kind"] == "append" else out
    q = h["q"] if c["kind"] == "step" else st["q"]
    B.tp_cache_attention(d, cache, h["step"], q, st["scale"], st["max_len"], h["o"], h["lse"], h["ws"])
    out = {"o": h["o"], "lse": h["lse"]}
    return {**out, "q": q} if c["kind"] == "step" else out


def run(st):
    if own:
        return _own_run(st)
    kind = st["c"]["kind"]
    if kind == "load":
        _plain_load(st)
    if kind == "attend":
        return _plain_attend(st, st["q"])
    if kind in ("append", "step"):
        q = _plain_append(st)
        return {**(_plain_attend(st, q) if kind == "step" else _plain_read(st)), "q": q}
    return _plain_read(st)


# ------------------------------------------------------------------------------ accounting
def work(c):
    """Each input read once, each output written once; the flops of the two products (and of the
    quantisation and rotation where there are none)."""
    lens, new, d, segs = _ints(c["lens"]), _new(c), c["d"], c["L"] * c["Hkv"]
    held = d + d // 16 + 4  # bytes of a token of one head in the cache
    if c["kind"] == "load":  # keys, codes and scales in, the pages written and read, two bf16 rows out
        n = segs * sum(lens)
        return {"bytes": n * (2 * d + d // 2 + 4 + 2 * held + 4 * d), "flops": n * d * 4}
    if c["kind"] == "read":
        n = segs * sum(m - f for m, f in zip(lens, _first(c)))
        return {"bytes": n * (held + 4 * d), "flops": n * d * 2}
    q = sum(new) * c["Hq"] * 2 * d
    if c["kind"] == "append":
        n = segs * sum(new)
        return {"bytes": n * (4 * d + 2 * held + 4 * d) + 2 * q + sum(new) * (4 * d + 4), "flops": (n + sum(new) * c["Hq"]) * d * 4}
    seen = sum(t * m - t * (t - 1) // 2 for m, t in zip(lens, new))
    b = c["Hkv"] * sum(lens) * held + 2 * q + sum(new) * c["Hq"] * 4
    if c["kind"] == "step":
        b += segs * sum(new) * 4 * d + q + sum(new) * (4 * d + 4)
    return {"bytes": b, "flops": 4 * c["Hq"] * d * seen}


# ------------------------------------------------------------------------------ in 64 bits
def _exact_places(d):
    """For token t and channel x of a block: the byte and the shift of the key's code, and of the value's."""
    out = [torch.empty((32, d), dtype=torch.int64) for _ in range(4)]
    for t in range(32):
        for x in range(d):
            e = x % 8
            nibble = e // 2 + 4 * (e % 2)
            word = t * (d // 8) + (x % 32) // 8 * (d // 32) + x // 32
            out[0][t, x], out[1][t, x] = 4 * word + nibble // 2, 4 * (nibble % 2)
            e = t // 16 * 4 + t % 4
            nibble = e // 2 + 4 * (e % 2)
            word = x // 64 * 256 + (t // 4 % 4 * 16 + x % 16) * 4 + x // 16 % 4
            out[2][t, x], out[3][t, x] = 16 * d + 4 * word + nibble // 2, 4 * (nibble % 2)
    return [x.cuda() for x in out]


def _exact_tokens(pages, table_row, page, d, start, stop, places):
    """Keys and values of tokens start .. stop - 1 of one sequence, fp64 [L][Hkv][tokens][d]."""
    t = torch.arange(start, stop, device="cuda")
    j = torch.arange(start // 32, (stop + 31) // 32, device="cuda")
    b = pages[:, table_row[j * 32 // page].long(), :, j % (page // 32)]  # [blocks][L][Hkv][bytes]
    out = []
    for byte, shift in ((places[0], places[1]), (places[2], places[3])):
        code = (b[..., byte.reshape(-1)].reshape(*b.shape[:-1], 32, d) >> shift.to(torch.uint8) & 15).double() - 8
        if not out:
            s = b[..., 32 * d:34 * d].contiguous().view(torch.bfloat16).double().reshape(*b.shape[:-1], 32, d // 32)
            code *= s.repeat_interleave(32, -1)
        else:
            code *= b[..., 34 * d:].contiguous().view(torch.float32).double()[..., None]
        x = code.permute(1, 2, 0, 3, 4).reshape(b.shape[1], b.shape[2], -1, d)
        out.append(x[:, :, t - start // 32 * 32])
    return out


def _exact_rotate(st, x):
    r = x.shape[-1]
    cs = st["cos_sin"][st["positions"].long()].double()
    c, s = cs[:, :r // 2], cs[:, r // 2:]
    x, out = x.double(), torch.empty(x.shape, dtype=torch.float64, device="cuda")
    lo, hi = (slice(0, r // 2), slice(r // 2, r)) if st["c"]["rope"] == "halves" else (slice(0, r, 2), slice(1, r, 2))
    for h in range(x.shape[1]):
        out[:, h, lo] = x[:, h, lo] * c - x[:, h, hi] * s
        out[:, h, hi] = x[:, h, hi] * c + x[:, h, lo] * s
    return out


def _exact_keys(k):
    """fp64 values of the 4-bit keys of bf16 rows [..., d]."""
    k = k.double()
    out = torch.empty_like(k)
    for s in range(0, k.shape[-1], 32):
        x = k[..., s:s + 32]
        g = (x.abs().max(-1, keepdim=True).values / 7).float().bfloat16().double()
        out[..., s:s + 32] = torch.where(g > 0, (x / g.clamp(min=1e-300)).round().clamp(-7, 7) * g, 0.0)
    return out


def _exact_values(v):
    v = v.double()
    g = (v.abs().max(-1, keepdim=True).values / 7).float().double()
    return torch.where(g > 0, (v / g.clamp(min=1e-300)).float().round().double().clamp(-7, 7) * g, 0.0)


def exact(c, seed):
    w = work(c)
    if w["flops"] > 4.0e11 or w["bytes"] > 4.0e9:
        return None
    st = prepare(c, seed)
    lens, new, d, R = _ints(c["lens"]), _new(c), c["d"], c["Hq"] // c["Hkv"]
    if c["kind"] == "load":
        codes = torch.stack([st["v_codes"].int() & 15, st["v_codes"].int() >> 4], -1).flatten(-2)
        codes = torch.where(codes > 7, codes - 16, codes)
        return {"k": _exact_keys(st["k"]), "v": codes.double() * st["v_scales"].double()[..., None]}
    places = _exact_places(d)
    if c["kind"] == "read":
        parts = [_exact_tokens(st["pages"], st["table"][b], c["page"], d, f, n, places)
                 for b, (f, n) in enumerate(zip(_first(c), lens))]
        return {"k": torch.cat([p[0] for p in parts], 2), "v": torch.cat([p[1] for p in parts], 2)}
    out = {}
    q = st["q"].double()
    if c["kind"] != "attend":
        out["q"] = _exact_rotate(st, st["q"])
        q = out["q"].float().bfloat16().double()  # the attention takes the rounded queries
        kn = _exact_keys(_exact_rotate(st, st["k"]).float().bfloat16())
        vn = _exact_values(st["v"])
        if c["kind"] == "append":
            return {**out, "k": kn.permute(1, 0, 2)[None], "v": vn.permute(1, 0, 2)[None]}
    o = torch.empty((sum(new), c["Hq"], d), dtype=torch.float64, device="cuda")
    lse = torch.empty((c["Hq"], sum(new)), dtype=torch.float64, device="cuda")
    for b, (n, t) in enumerate(zip(lens, new)):
        k, v = (x[0] for x in _exact_tokens(st["pages"], st["table"][b], c["page"], d, 0, n, places))
        at = st["offsets"][b]
        if c["kind"] == "step":
            k[:, n - t:], v[:, n - t:] = kn[at:at + t].transpose(0, 1), vn[at:at + t].transpose(0, 1)
        unseen = torch.arange(n, device="cuda") > torch.arange(n - t, n, device="cuda")[:, None]
        for h in range(c["Hq"]):
            x = (q[at:at + t, h] @ k[h // R].T / math.sqrt(d)).masked_fill(unseen, -math.inf)
            lse[h, at:at + t] = torch.logsumexp(x, 1)
            o[at:at + t, h] = torch.softmax(x, 1) @ v[h // R]
    return {**out, "o": o, "lse": lse}
