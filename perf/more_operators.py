"""Performance cases of the 8-bit paged cache: filling it from an eviction, growing it token by token with
the position rotation, attending over it, and reading it back.

A case is one pass of a serving program, on inputs and pages it already holds on the GPU:

  load     the eviction's compact cache (bf16 keys, value codes and scales) into pages, and the loaded tokens
           read back
  append   new tokens' keys (rotated at their positions) and values into the pages, their queries rotated
           beside them, and the blocks of 32 tokens that they lie in read back
  attend   causal attention of each sequence's newest tokens over its pages
  step     append, then attend: one decode step of a layer
  read     a range of every sequence's tokens read back as bf16 rows (to evict again)

The cache is one tensor of bytes [L][pages][Hkv][page_tokens / 32][64 d + 144].  A block holds 32 tokens of
one head: the keys' codes (32 d bytes), the values' codes (32 d), the values' scales (fp32, one per token), the
keys' scale (fp32, one for the block) and 12 bytes that nothing uses.  A code c is held as the byte c + 128
("int") or as its OCP E4M3 byte ("fp8").  Bytes of token t, channel x:
  keys     (t / 16) 16 d + (x / 64) 1024 + ((x % 32 / 8) 16 + t % 16) 16 + (x / 32 % 2) 8 + x % 8
  values   32 d + (x / 32) 1024 + ((t % 16 / 4) 16 + x % 16) 16 + (x / 16 % 2) 8 + (t / 16) 4 + t % 4

The keys' scale: absmax / qmax of the block's tokens that one call writes; a later token beyond it raises it
by a power of two, and the codes that the block holds are rounded again.
"""
import math
import random

import torch

own = False


def _case(kind, fmt, Hq, Hkv, d, page, lens, new="1", L=1, first="0", rope="halves", table=0, bits=8, name=None):
    c = {"kind": kind, "fmt": fmt, "L": L, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "lens": lens, "new": new,
         "first": first, "rope": rope, "table": table, "bits": bits}
    if name is not None:
        c["name"] = name
    return c


def _text(values):
    return ",".join(str(int(v)) for v in values)


def listed():
    r = random.Random(23)
    ragged = _text(int(math.exp(r.uniform(math.log(5000), math.log(24576)))) for _ in range(48))
    drafts = [(r.randint(2000, 12000), r.randint(1, 8)) for _ in range(16)]
    return [
        # the smallest call: one sequence of a small model, bound by launches and latency
        _case("attend", "int", 8, 2, 64, 32, "321", name="attend_one"),
        # a full serving batch of mixed lengths, 64 query heads: the bandwidth of the cache
        _case("attend", "fp8", 64, 8, 128, 64, ragged, name="attend_ragged48"),
        # two very long sequences that were not evicted
        _case("attend", "int", 64, 8, 128, 256, "200003,98305", name="attend_long"),
        # drafted tokens verified: 1 to 8 query tokens a sequence
        _case("attend", "int", 32, 8, 128, 64, _text(a for a, _ in drafts), _text(b for _, b in drafts), name="attend_drafts"),
        # the next part of a prompt in chunks, over a cache that is already in pages
        _case("attend", "fp8", 32, 8, 128, 128, "14001,4096", "1024,300", name="attend_chunk"),
        # one decode step's append in a full batch
        _case("append", "int", 32, 8, 128, 64, _text(r.randint(1, 2600) for _ in range(64)), table=131072, name="append_decode"),
        # a prompt's chunk written at once, pairs of neighbours rotated
        _case("append", "fp8", 64, 8, 128, 64, "10007,5003", "8191,5003", rope="pairs", table=65536, name="append_chunk"),
        # every layer of an 8B model: the kept tenth of a 128K prefill into pages
        _case("load", "fp8", 32, 8, 128, 64, "13107", L=32, name="load_kept_128k"),
        # a small model's batch under a budget of 512 tokens and shorter sequences
        _case("load", "int", 8, 2, 64, 32, "512,512,77,512,301,1", L=4, name="load_budget_small"),
        # the tokens of a long answer read back to be evicted again
        _case("read", "int", 32, 8, 128, 64, "20011,6000,12345", L=8, first="6553,2048,0", name="read_answers"),
        # the same for a small model and one answer
        _case("read", "fp8", 8, 2, 64, 32, "1500", L=4, first="413", name="read_one"),
        # one decode step of a layer: append and attention under a budget of 2048 and what was answered since
        _case("step", "fp8", 32, 8, 128, 64, _text(2048 + r.randint(1, 500) for _ in range(32)), table=131072,
              name="step_budget_2048"),
    ]


def draw(rng):
    """A case of the same kinds over the same ranges; lengths log-uniform."""
    def logint(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    while True:
        kind = rng.choice(["attend"] * 5 + ["append", "append", "load", "read", "step", "step"])
        fmt = rng.choice(["int", "fp8"])
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
        c = _case(kind, fmt, Hq, Hkv, d, rng.choice([32, 64, 128, 256]), _text(lens), _text(new), L, _text(first),
                  rng.choice(["halves", "halves", "pairs"]), rng.choice([32768, 131072]) if kind in ("append", "step") else 0,
                  rng.choice([8, 8, 6, 4]) if kind == "load" and fmt == "int" else 8)
        w = work(c)
        # no dearer than the largest listed case, and the plain form's padded scores and keys fit
        if (w["bytes"] <= 1.2e9 and w["flops"] <= 2.2e11 and len(lens) * max(lens) * Hkv * d <= 48 * 24576 * 8 * 128
                and len(lens) * max(lens) * max(new) * Hq <= 1.0e9):
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
    """The first token that a read takes: a case's own; for an append, that of the block of its first new token."""
    if c["kind"] == "append":
        return [(m - t) // 32 * 32 for m, t in zip(_ints(c["lens"]), _new(c))]
    n = _ints(c["first"])
    return n * len(_ints(c["lens"])) if len(n) == 1 else n


def _block_bytes(d):
    return 64 * d + 144


def _qmax(fmt, bits=8):
    return 448.0 if fmt == "fp8" else float((1 << (bits - 1)) - 1)


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
    L, Hq, Hkv, d, page, fmt = c["L"], c["Hq"], c["Hkv"], c["d"], c["page"], c["fmt"]
    lens, new, first = _ints(c["lens"]), _new(c), _first(c)
    B, per = len(lens), page // 32
    need = [-(-n // page) for n in lens]
    num_pages = sum(need) + 3
    order = torch.randperm(num_pages, device="cuda", generator=g)[:sum(need)].to(torch.int32)
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device="cuda")
    at = _offsets(need)
    for b in range(B):
        table[b, :need[b]] = order[at[b]:at[b + 1]]
    pages = torch.zeros((L, num_pages, Hkv, per, _block_bytes(d)), dtype=torch.uint8, device="cuda")

    def random_blocks(n, held=None):
        """n blocks, quantised as the operators do; slots behind the tokens held are zero keys."""
        k = _keys((n, 32, d), g)
        if held is not None:
            k.masked_fill_((torch.arange(32, device="cuda") >= held[:, None])[..., None], 0.0)
        ks = _fresh_scale(k.abs().amax((-1, -2)), fmt)
        vc, vs = _quantise_values(_values((n, 32, d), g), fmt)
        return _pack(_codes_of(k, ks[:, None, None], fmt), ks, vc, vs, fmt)

    flat = pages.view(-1, _block_bytes(d))
    for i in range(0, flat.shape[0], 32768):
        n = min(32768, flat.shape[0] - i)
        flat[i:i + n] = random_blocks(n)
    if c["kind"] in ("append", "step"):  # the blocks that the new tokens begin in hold those before them alone
        begin = torch.tensor([m - t for m, t in zip(lens, new)], device="cuda")
        page_of = table[torch.arange(B, device="cuda"), begin // page].long()
        n = B * Hkv
        tail = random_blocks(n, (begin % 32).repeat_interleave(Hkv)).view(B, Hkv, -1)
        pages[0, page_of, :, begin // 32 % per] = tail
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
        return (torch.cat(page_of), torch.cat(block_of)), (torch.cat(token_block), torch.cat(token_slot))

    if c["kind"] == "load":
        n = sum(lens)
        st["offsets"] = _offsets(lens)
        st["k"] = _keys((L, Hkv, n, d), g)
        codes, st["v_scales"] = _quantise_values(_values((L, Hkv, n, d), g), fmt, c["bits"])
        if fmt == "fp8":
            st["v_codes"] = codes.to(torch.float8_e4m3fn).view(torch.uint8)
        elif c["bits"] > 4:
            st["v_codes"] = codes.to(torch.int8).view(torch.uint8)
        else:  # two's complement, two to a byte, even element low
            codes = codes.to(torch.int8)
            st["v_codes"] = (codes[..., 0::2] & 15 | codes[..., 1::2] << 4).view(torch.uint8)
        st["blocks"], st["tokens"] = touched([0] * B, lens)
        st["read"] = st["tokens"]
        st["fresh"] = torch.ones(st["blocks"][0].numel(), dtype=torch.bool, device="cuda")
    elif c["kind"] == "read":
        st["offsets"] = _offsets(n - f for n, f in zip(lens, first))
        st["first"] = first
        st["blocks"], st["read"] = touched(first, lens)
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
            begin = [m - t for m, t in zip(lens, new)]
            st["blocks"], st["tokens"] = touched(begin, lens)
            st["fresh"] = torch.cat([torch.arange(f // 32, -(-m // 32), device="cuda") * 32 >= f for f, m in zip(begin, lens)])
            if c["kind"] == "append":
                st["first"] = first
                st["read_offsets"] = _offsets(m - f for m, f in zip(lens, first))
                st["read"] = touched(first, lens)[1]
        if c["kind"] != "append":
            back = torch.arange(max(new), device="cuda")
            start = torch.tensor(st["offsets"][:-1], device="cuda")
            st["rows"] = (start[:, None] + back).clamp_(max=n - 1)  # [B][max_new]: each padded row's query
            st["row_of"] = torch.cat([torch.arange(t, device="cuda") + b * max(new) for b, t in enumerate(new)])
    return st


# ------------------------------------------------------------------------------ the plain form
def _rounded(x, fmt):
    """fp32 numbers to the nearest code, within the format's range."""
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() if fmt == "fp8" else torch.round(x).clamp_(-127, 127)


def _fresh_scale(absmax, fmt):
    return (absmax.double() / _qmax(fmt)).float()


def _codes_of(x, scale, fmt):
    """bf16 rows -> codes as fp32 numbers."""
    return _rounded(torch.where(scale > 0, x.float() / scale, 0.0), fmt)


def _quantise_values(v, fmt, bits=8):
    """bf16 [..., d] -> codes [..., d] (fp32 numbers) and fp32 scales [...]."""
    scale = (v.float().abs().amax(-1).double() / _qmax(fmt, bits)).float()
    codes = _codes_of(v, scale[..., None], fmt)
    return (codes if fmt == "fp8" else codes.clamp_(-_qmax(fmt, bits), _qmax(fmt, bits))), scale


def _bytes_of(codes, fmt):
    return codes.to(torch.float8_e4m3fn).view(torch.uint8) if fmt == "fp8" else (codes + 128).to(torch.uint8)


def _codes(held, fmt):
    return held.contiguous().view(torch.float8_e4m3fn).float() if fmt == "fp8" else held.float() - 128


def _pack(kc, ks, vc, vs, fmt):
    """Codes [..., 32, d], the keys' scale [...], the values' [..., 32] -> blocks [..., bytes]."""
    d, lead, n = kc.shape[-1], kc.shape[:-2], kc.dim() - 2
    k = _bytes_of(kc, fmt).reshape(*lead, 2, 16, d // 64, 2, 4, 8)  # (t / 16, t % 16, x / 64, x / 32 % 2, x % 32 / 8, x % 8)
    k = k.permute(*range(n), n, n + 2, n + 4, n + 1, n + 3, n + 5).reshape(*lead, -1)
    v = _bytes_of(vc, fmt).reshape(*lead, 2, 4, 4, d // 32, 2, 16)  # (t / 16, t % 16 / 4, t % 4, x / 32, x / 16 % 2, x % 16)
    v = v.permute(*range(n), n + 3, n + 1, n + 5, n + 4, n, n + 2).reshape(*lead, -1)
    s = torch.cat([vs, ks[..., None], torch.zeros_like(vs[..., :3])], -1)
    return torch.cat([k, v, s.contiguous().view(torch.uint8)], -1)


def _unpack(blocks, d, fmt):
    """Blocks [..., bytes] -> codes [..., 32, d] (fp32 numbers), scale [...], codes, scales [..., 32]."""
    lead, n = blocks.shape[:-1], blocks.dim() - 1
    k, v, s = blocks.split([32 * d, 32 * d, 144], -1)
    k = k.reshape(*lead, 2, d // 64, 4, 16, 2, 8).permute(*range(n), n, n + 3, n + 1, n + 4, n + 2, n + 5)
    v = v.reshape(*lead, d // 32, 4, 16, 2, 2, 4).permute(*range(n), n + 4, n + 1, n + 5, n, n + 3, n + 2)
    s = s.contiguous().view(torch.float32)
    return _codes(k.reshape(*lead, 32, d), fmt), s[..., 32], _codes(v.reshape(*lead, 32, d), fmt), s[..., :32]


def _held(blocks, d, fmt):
    """Blocks -> the keys and values that they stand for, fp32 [..., 32, d]."""
    kc, ks, vc, vs = _unpack(blocks, d, fmt)
    return kc.mul_(ks[..., None, None]), vc.mul_(vs[..., None])


def _blocks_first(pages):
    return pages.permute(1, 3, 0, 2, 4)  # [pages][blocks of a page][L][Hkv][bytes]


def _plain_write(st, k, vc, vs):
    """Tokens' bf16 keys, value codes and scales [tokens][L][Hkv][..] into the pages; the rest of their blocks
    keeps what it holds, its keys in the block's new scale."""
    fmt, d = st["c"]["fmt"], st["c"]["d"]
    view = _blocks_first(st["pages"])
    kc, ks, held_vc, held_vs = _unpack(view[st["blocks"]], d, fmt)
    block, slot = st["tokens"]
    keys = torch.zeros(kc.shape, dtype=torch.bfloat16, device=k.device)
    keys[block, :, :, slot] = k
    want = _fresh_scale(keys.abs().amax((-1, -2)), fmt)
    held = torch.where(st["fresh"][:, None, None], 0.0, ks)
    (wm, we), (hm, he) = torch.frexp(want), torch.frexp(held)
    up = torch.where((want > held) & (held > 0), we - he + (wm > hm).int(), 0)  # the least power that holds them
    ks = torch.where(held > 0, torch.ldexp(held.double(), up).float(), want)
    kc = torch.where((up > 0)[..., None, None], _rounded(torch.ldexp(kc, -up[..., None, None]), fmt), kc)
    kc[block, :, :, slot] = _codes_of(keys, ks[..., None, None], fmt)[block, :, :, slot]
    held_vc[block, :, :, slot] = vc
    held_vs[block, :, :, slot] = vs
    view[st["blocks"]] = _pack(kc, ks, held_vc, held_vs, fmt)


def _plain_read(st):
    k, v = _held(_blocks_first(st["pages"])[st["blocks"]], st["c"]["d"], st["c"]["fmt"])
    block, slot = st["read"]
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
    vc, vs = _quantise_values(st["v"], st["c"]["fmt"])
    _plain_write(st, _plain_rotate(st, st["k"])[:, None], vc[:, None], vs[:, None])
    return _plain_rotate(st, st["q"])


def _plain_load(st):
    raw = st["v_codes"]
    if st["c"]["fmt"] == "fp8":
        vc = _codes(raw, "fp8")
    elif st["c"]["bits"] > 4:
        vc = raw.view(torch.int8).float()
    else:
        vc = torch.stack([(raw << 4).view(torch.int8) >> 4, raw.view(torch.int8) >> 4], -1).flatten(-2).float()
    _plain_write(st, *(x.movedim(2, 0) for x in (st["k"], vc, st["v_scales"])))


def _plain_attend(st, q):
    c = st["c"]
    B, d, Hkv, R, T = st["lens"].numel(), c["d"], c["Hkv"], c["Hq"] // c["Hkv"], st["rows"].shape[1]
    blocks = st["pages"][0][st["table"].long().clamp(min=0)]  # [B][pages][Hkv][blocks][bytes]
    k, v = (x.permute(0, 2, 1, 3, 4, 5).reshape(B, Hkv, -1, d) for x in _held(blocks, d, c["fmt"]))
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
    h["cache"] = B.Cache8(h["d"], st["pages"], st["table"], st["lens"], c["page"],
                          B.TP_QFMT_FP8_E4M3 if c["fmt"] == "fp8" else B.TP_QFMT_INT)
    n = st["offsets"][-1]
    if c["kind"] in ("load", "append", "read"):
        h["batch"] = B.Batch(st.get("read_offsets") or st["offsets"])
        h["first"] = st.get("first")
        h["k"] = torch.empty((c["L"], c["Hkv"], h["batch"].n_tot, c["d"]), dtype=torch.bfloat16, device="cuda")
        h["v"] = torch.empty_like(h["k"])
    if c["kind"] in ("append", "attend", "step"):
        h["step"] = B.Step(n, st["max_new"], st["new_offsets"])
    if c["kind"] in ("append", "step"):
        h["rope"] = B.Rope(st["cos_sin"], c["d"], B.TP_ROPE_HALVES if c["rope"] == "halves" else B.TP_ROPE_PAIRS)
        h["q"] = torch.empty((n, c["Hq"], c["d"]), dtype=torch.bfloat16, device="cuda")
    if c["kind"] in ("attend", "step"):
        h["o"] = torch.empty((n, c["Hq"], c["d"]), dtype=torch.bfloat16, device="cuda")
        h["lse"] = torch.empty((c["Hq"], n), device="cuda")
        h["ws"] = torch.empty(B.tp_cache8_workspace_size(h["d"], h["cache"], h["step"], st["max_len"]), dtype=torch.uint8,
                              device="cuda")
    return h


def _own_run(st):
    c = st["c"]
    h = st.get("handles") or st.setdefault("handles", _handles(st))
    B, d, cache = h["B"], h["d"], h["cache"]
    if c["kind"] == "load":
        B.tp_cache8_load(d, cache, st["offsets"], st["k"], st["v_codes"], st["v_scales"], c["bits"])
    if c["kind"] in ("append", "step"):
        B.tp_cache8_append(d, cache, h["step"], st["k"], st["v"], st["positions"], h["rope"], st["q"], h["q"])
    if c["kind"] in ("load", "append", "read"):
        B.tp_cache8_read(d, cache, h["batch"], h["k"], h["v"], h["first"])
        out = {"k": h["k"], "v": h["v"]}
        return {**out, "q": h["q"]} if c["kind"] == "append" else out
    q = h["q"] if c["kind"] == "step" else st["q"]
    B.tp_cache8_attention(d, cache, h["step"], q, st["scale"], st["max_len"], h["o"], h["lse"], h["ws"])
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
    held = 2 * d + 4.125  # bytes of a token of one head in the cache
    if c["kind"] == "load":  # keys, codes and scales in, the pages written and read, two bf16 rows out
        n, codes = segs * sum(lens), d if c["bits"] > 4 else d // 2
        return {"bytes": int(n * (2 * d + codes + 4 + 2 * held + 4 * d)), "flops": n * d * 4}
    if c["kind"] == "read":
        n = segs * sum(m - f for m, f in zip(lens, _first(c)))
        return {"bytes": int(n * (held + 4 * d)), "flops": n * d * 2}
    q = sum(new) * c["Hq"] * 2 * d
    if c["kind"] == "append":
        n = segs * sum(new)
        back = segs * sum(m - f for m, f in zip(lens, _first(c)))
        return {"bytes": int(n * (4 * d + held) + back * (held + 4 * d)) + 2 * q + sum(new) * (4 * d + 4),
                "flops": (n + sum(new) * c["Hq"]) * d * 4}
    seen = sum(t * m - t * (t - 1) // 2 for m, t in zip(lens, new))
    b = int(c["Hkv"] * sum(lens) * held) + 2 * q + sum(new) * c["Hq"] * 4
    if c["kind"] == "step":
        b += segs * sum(new) * 4 * d + q + sum(new) * (4 * d + 4)
    return {"bytes": b, "flops": 4 * c["Hq"] * d * seen}


# ------------------------------------------------------------------------------ in 64 bits
def _exact_round(x, fmt, most):
    """fp64 numbers to the nearest code of the format, ties to even."""
    if fmt == "int":
        return x.round().clamp(-most, most)
    unit = torch.exp2((torch.frexp(x)[1] - 4).clamp(min=-9).double())  # 4 significant bits, 2^-9 at least
    return ((x / unit).round() * unit).clamp(-448, 448)


def _exact_places(d):
    """The byte of every token and channel of a block: its key's code, and its value's."""
    t, x = torch.arange(32, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    k = t // 16 * 16 * d + x // 64 * 1024 + (x % 32 // 8 * 16 + t % 16) * 16 + x // 32 % 2 * 8 + x % 8
    v = 32 * d + x // 32 * 1024 + (t % 16 // 4 * 16 + x % 16) * 16 + x // 16 % 2 * 8 + t // 16 * 4 + t % 4
    return k.reshape(-1), v.reshape(-1)


def _exact_number(byte, fmt):
    """The number that a code's byte stands for, by the format's definition."""
    byte = byte.long()
    if fmt == "int":
        return byte.double() - 128
    e, m = byte >> 3 & 15, (byte & 7).double()
    size = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2((e - 7).double()))
    return torch.where(byte > 127, -size, size)


def _exact_tokens(st, b, start, stop):
    """Tokens start .. stop - 1 of sequence b, whole blocks: keys' codes fp64 [L][Hkv][blocks][32][d] and scale
    [L][Hkv][blocks], values [L][Hkv][blocks][32][d]."""
    c = st["c"]
    d, page = c["d"], c["page"]
    at_k, at_v = _exact_places(d)
    j = torch.arange(start // 32, (stop + 31) // 32, device="cuda")
    x = st["pages"][:, st["table"][b, j * 32 // page].long(), :, j % (page // 32)].permute(1, 2, 0, 3)
    s = x[..., 64 * d:].contiguous().view(torch.float32).double()
    k, v = (_exact_number(x[..., at], c["fmt"]).reshape(*x.shape[:-1], 32, d) for at in (at_k, at_v))
    return k, s[..., 32], v * s[..., :32, None]


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


def _exact_write(rows, begin, held, fmt):
    """fp64 keys rows [L][Hkv][tokens][d] written from token `begin` on; held: the first block's codes and scale
    before.  Returns the keys that the touched blocks then stand for, from the first block's start to the last token."""
    qmax = 448.0 if fmt == "fp8" else 127.0
    out, at = [], 0
    total = rows.shape[2]
    while at < total:
        slot = begin % 32 if at == 0 else 0
        x = rows[:, :, at:at + 32 - slot]
        s = (x.abs().amax((-1, -2)) / qmax).float().double()
        if slot:
            codes, old = held[0][..., :slot, :], held[1]
            up = torch.where((old > 0) & (s > old), torch.log2(s / old.clamp(min=1e-300)).ceil(), 0.0)
            up += ((old > 0) & (old * torch.exp2(up) < s)).double()  # (the logarithm is rounded)
            up -= ((up > 0) & (old * torch.exp2(up - 1) >= s)).double()
            s = torch.where(old > 0, old * torch.exp2(up), s)
            out.append(_exact_round(codes * torch.exp2(-up)[..., None, None], fmt, 127) * s[..., None, None])
        quotient = torch.where(s[..., None, None] > 0, x / s.clamp(min=1e-300)[..., None, None], 0.0)
        out.append(_exact_round(quotient.float().double(), fmt, 127) * s[..., None, None])  # an fp32 quotient, as defined
        at += 32 - slot
    return torch.cat(out, 2)


def _exact_values(v, fmt):
    v = v.double()
    g = (v.abs().max(-1, keepdim=True).values / _qmax(fmt)).float().double()
    return torch.where(g > 0, _exact_round((v / g.clamp(min=1e-300)).float().double(), fmt, 127) * g, 0.0)


def exact(c, seed):
    w = work(c)
    if w["flops"] > 2.5e11 or w["bytes"] > 6.0e9:
        return None
    st = prepare(c, seed)
    lens, new, d, R, fmt, L = _ints(c["lens"]), _new(c), c["d"], c["Hq"] // c["Hkv"], c["fmt"], c["L"]
    at = st["offsets"]
    if c["kind"] == "load":
        raw = st["v_codes"].long()
        if fmt == "fp8":
            codes = _exact_number(raw, fmt)
        elif c["bits"] > 4:
            codes = (raw - 256 * (raw > 127)).double()
        else:
            codes = torch.stack([raw & 15, raw >> 4], -1).flatten(-2)
            codes = (codes - 16 * (codes > 7)).double()
        k = [_exact_write(st["k"][:, :, at[b]:at[b + 1]].double(), 0, None, fmt) for b in range(len(lens))]
        return {"k": torch.cat(k, 2), "v": codes * st["v_scales"].double()[..., None]}
    if c["kind"] == "read":
        out = {"k": [], "v": []}
        for b, (f, n) in enumerate(zip(_first(c), lens)):
            codes, s, v = _exact_tokens(st, b, f, n)
            for name, x in (("k", codes * s[..., None, None]), ("v", v)):
                out[name].append(x.flatten(2, 3)[:, :, f % 32:n - f // 32 * 32])
        return {name: torch.cat(x, 2) for name, x in out.items()}
    out = {}
    q = st["q"].double()
    k_after, v_after = [], []
    if c["kind"] != "attend":
        out["q"] = _exact_rotate(st, st["q"])
        q = out["q"].float().bfloat16().double()  # the attention takes the rounded queries
        kn = _exact_rotate(st, st["k"]).float().bfloat16().double().permute(1, 0, 2)[None]
        vn = _exact_values(st["v"], fmt).permute(1, 0, 2)[None]
        for b, (n, t) in enumerate(zip(lens, new)):
            codes, s, v = _exact_tokens(st, b, n - t, n)
            slot = (n - t) % 32
            k_after.append(_exact_write(kn[:, :, at[b]:at[b + 1]], n - t, (codes[:, :, 0], s[:, :, 0]), fmt))
            v_after.append(torch.cat([v[:, :, 0, :slot], vn[:, :, at[b]:at[b + 1]]], 2))
        if c["kind"] == "append":
            return {**out, "k": torch.cat(k_after, 2), "v": torch.cat(v_after, 2)}
    o = torch.empty((sum(new), c["Hq"], d), dtype=torch.float64, device="cuda")
    lse = torch.empty((c["Hq"], sum(new)), dtype=torch.float64, device="cuda")
    for b, (n, t) in enumerate(zip(lens, new)):
        codes, s, v = _exact_tokens(st, b, 0, n)
        k, v = ((x[0].flatten(1, 2)[:, :n]) for x in (codes * s[..., None, None], v))
        del codes
        if c["kind"] == "step":
            f = (n - t) // 32 * 32
            k[:, f:], v[:, f:] = k_after[b][0], v_after[b][0]
        unseen = torch.arange(n, device="cuda") > torch.arange(n - t, n, device="cuda")[:, None]
        for h in range(c["Hq"]):
            x = (q[at[b]:at[b + 1], h] @ k[h // R].T / math.sqrt(d)).masked_fill(unseen, -math.inf)
            lse[h, at[b]:at[b + 1]] = torch.logsumexp(x, 1)
            o[at[b]:at[b + 1], h] = torch.softmax(x, 1) @ v[h // R]
    return {**out, "o": o, "lse": lse}
