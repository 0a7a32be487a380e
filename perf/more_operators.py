"""Latent attention on paged, packed caches: what is timed and how it is computed plainly.

A token leaves one row in the cache, shared by all heads: a latent of `Dc` numbers, from which every head's key (`Dk`) and value
(`Dv`) follow by one weight matrix w [Dc][H][Dk + Dv], and a position part of `Dr` numbers that is a key of every head as it is:

  k[h] = (c w[:, h, :Dk], r),   v[h] = c w[:, h, Dk:],   out[h] = softmax(q[h] k[h]^T / sqrt(Dk + Dr)) v[h]

Rows lie in pages of a pool, records of several layers each with a width of its own: 16 = fp16, 8 / 4 / 2 = codes of the latent with a
scale and a minimum per group of `G` numbers, the position part in fp16 always.  A record's sections, one layer after the other in
each: codes (fp16: the latents), scales, minima, position parts.  A table holds every page's offset and width.  Kinds of case:

  append   the latents and position parts of new tokens go to their places in the pages of one layer;
  read     rows come back from the pages as fp16, what a Load of them gives;
  round    append to packed pages, and what was appended read back;
  attend   the newest tokens' queries attend to one layer's pages in the absorbed form: queries are taken to the latents' space,
           so that the latents are keys and values of all heads at once;
  prompt   many new tokens attend in the expanded form: keys and values of every head are made from the latents first;
  step     append and attend as one decode step has them.

Latents are N(0,1), as a norm leaves them, with one number in a hundred four times larger; weights N(0,1) / sqrt(Dc), queries
N(0,2), which gives logits of spread 2.  Lengths and widths follow from the case, values from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
INF = float("inf")


# ------------------------------------------------------------------ the cases

def _case(name, kind, seqs, least, most, H, dims, T, G, widths, fmt=0, L=1, rows=1):
    """`least`, `most`: the shortest and the longest sequence (new tokens included); dims: Dc, Dr, Dk, Dv; `rows`: new tokens that
    a sequence has at most; `widths`: the widths of the pages (G: fp16), in turn over a shuffled order."""
    return {"name": name, "kind": kind, "seqs": seqs, "least": least, "most": most, "H": H, "Dc": dims[0], "Dr": dims[1],
            "Dk": dims[2], "Dv": dims[3], "T": T, "G": G, "widths": widths, "fmt": fmt, "L": L, "rows": rows}


_LARGE, _SMALL = (512, 64, 128, 128), (256, 32, 64, 64)


def listed():
    return [
        # one new token for each of 64 running sequences: a launch and little else
        _case("append-step-64", "append", 64, 30, 500, 128, _LARGE, 32, 128, "G", L=2),
        # prompts of up to 32768 tokens that arrive together
        _case("append-prompts-6", "append", 6, 300, 32768, 128, _LARGE, 16, 64, "G", rows=32768),
        # prompts that go straight to packed pages, and the same rows back for the expanded form
        _case("round-prompts-packed", "round", 8, 1000, 16384, 128, _LARGE, 16, 64, "842", L=2, rows=16384),
        # a few pages of a small model: latency
        _case("read-page", "read", 1, 48, 48, 40, _SMALL, 16, 64, "84", rows=48),
        # whole contexts come back for one layer, parameters in binary16
        _case("read-ragged-24", "read", 24, 1, 16384, 32, _LARGE, 32, 128, "G842", fmt=3, L=2, rows=16384),
        # one short context of a small model: latency
        _case("attend-short", "attend", 1, 333, 333, 40, _SMALL, 16, 64, "G"),
        # a ragged batch in packed records, parameters in binary16
        _case("attend-ragged-24", "attend", 24, 1, 8000, 32, _LARGE, 32, 128, "8842", fmt=3, L=2),
        # drafts of up to four tokens verified in one pass
        _case("attend-drafts", "attend", 16, 5, 3001, 40, _LARGE, 16, 64, "G84", rows=4),
        # the largest: 16 contexts of 32768 tokens in fp16, 128 heads on one latent
        _case("attend-16x32k", "attend", 16, 32768, 32768, 128, _LARGE, 32, 128, "G"),
        # a whole prompt
        _case("prompt-4k", "prompt", 1, 4096, 4096, 128, _LARGE, 16, 64, "G", rows=4096),
        # pieces of 512 tokens added to long contexts whose older pages are packed
        _case("prompt-pieces-4", "prompt", 4, 5003, 16384, 32, _LARGE, 32, 128, "8842", fmt=3, rows=512),
        # a decode step of 8 contexts whose older pages are packed: the new token is appended and attends
        _case("step-8", "step", 8, 700, 8192, 64, _LARGE, 16, 64, "842"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "read", "round", "attend", "attend", "attend", "prompt", "prompt", "step"])
    dims = rng.choice([512, 512, 256]), rng.choice([64, 64, 32]), rng.choice([128, 128, 64]), rng.choice([128, 128, 64])
    T = rng.choice([16, 32, 64, 48])
    G = rng.choice([g for g in (64, 128, 256, 512) if dims[0] % g == 0])
    H = rng.choice([1, 4, 5, 20, 40, 64, 128])
    most = _log_int(rng, 3, 32768)
    fmt, L = rng.choice([0, 0, 3]), rng.choice([1, 2])
    if kind == "prompt":
        # at most half of the work of a listed prompt for the scores, and half for keys and values
        rows, most_scores, most_keys = min(most, _log_int(rng, 2, 4096)), 2 ** 29, 3 * 2 ** 19
        while H * rows * most > most_scores or H * most > most_keys:
            H, rows, most = max(1, H // 2), max(1, rows // 2), max(rows, most * 2 // 3)
        seqs = max(1, min(_log_int(rng, 1, 8), most_scores // (H * rows * most), most_keys // (H * most)))
    else:
        # at most an eighth of the tokens of the largest listed attention, half of it for the moves
        budget = 2 ** 19 / (8 if kind in ("attend", "step") else 4)
        seqs = max(1, min(_log_int(rng, 1, 64), int(budget / most)))
        rows = {"attend": rng.choice([1, 1, rng.randint(2, 5)]), "step": 1, "append": rng.choice([1, rng.randint(1, 16), most])}.get(kind, most)
    least = rng.randint(1, most)
    widths = "G" if kind == "append" else rng.choice(["842", "8", "4", "2", "8842"] if kind == "round" else
                                                     ["G", "842", "8", "4", "2", "G84", "8842"])
    return _case("", kind, seqs, least, most, H, dims, T, G, widths, fmt, L, rows)


def _lengths(c):
    """Tokens of each sequence: spread over [least, most], both among them where there are two."""
    n, lo, hi = c["seqs"], c["least"], c["most"]
    if n == 1:
        return [hi]
    return [hi, lo] + [lo + int((hi - lo) * ((i * 0.6180339887) % 1.0)) for i in range(1, n - 1)]


def _new_rows(c):
    """New tokens of each sequence (no more than it has)."""
    if c["rows"] <= 16:
        return [min(n, 1 + (i * 7) % c["rows"]) for i, n in enumerate(_lengths(c))]
    return [min(n, c["rows"]) for n in _lengths(c)]


def _capacity(c):
    return -(-c["most"] // c["T"]) * c["T"]


_WIDTHS = {"G": 16, "8": 8, "4": 4, "2": 2}


def _page_widths(c):
    """[seqs][pages] widths; 0 behind a sequence's last page.  A step's newest page is fp16."""
    pages = _capacity(c) // c["T"]
    cycle = [_WIDTHS[w] for w in c["widths"]]
    order = np.random.RandomState(11).permutation(c["seqs"] * pages)
    bits = np.resize(np.array(cycle, dtype=np.uint8), c["seqs"] * pages)[order].reshape(c["seqs"], pages)
    for s, n in enumerate(_lengths(c)):
        last = -(-n // c["T"])
        bits[s, last:] = 0
        if c["kind"] == "step":
            bits[s, last - 1] = 16
    return bits


def _row_bytes(c, w):
    """One token's row."""
    return 2 * c["Dr"] + (2 * c["Dc"] if w == 16 else c["Dc"] * w // 8 + c["Dc"] // c["G"] * (4 if c["fmt"] == 3 else 8))


def _record_bytes(c, w):
    return c["L"] * c["T"] * _row_bytes(c, w)


def work(case):
    c = case
    new, length, bits = _new_rows(c), _lengths(c), _page_widths(c)
    H, Dc, Dr, Dk, Dv = (c[x] for x in ("H", "Dc", "Dr", "Dk", "Dv"))
    row = 2 * (Dc + Dr)
    held = 0                                                 # bytes of the tokens in the pages
    for s, n in enumerate(length):
        for w in (16, 8, 4, 2):
            held += int(np.minimum(c["T"], n - np.flatnonzero(bits[s] == w) * c["T"]).sum()) * _row_bytes(c, w)
    if c["kind"] == "append":
        return {"bytes": 2 * row * sum(new), "flops": 0}
    if c["kind"] == "read":
        return {"bytes": held + row * sum(new), "flops": 0}
    if c["kind"] == "round":                                 # rows read, records written and read, rows written
        return {"bytes": 2 * held + 2 * row * sum(new), "flops": 0}
    pairs = sum(r * n - r * (r - 1) // 2 for n, r in zip(length, new))
    total = held + Dc * H * (Dk + Dv) * 2 + sum(new) * H * (Dk + Dr + Dv) * 2
    if c["kind"] == "prompt":
        flops = 2 * sum(length) * Dc * H * (Dk + Dv) + 2 * H * (Dk + Dr + Dv) * pairs
    else:
        flops = 2 * sum(new) * H * Dc * (Dk + Dv) + 2 * H * (Dc + Dr + Dc) * pairs
        total += 2 * row * sum(new) if c["kind"] == "step" else 0
    return {"bytes": total, "flops": flops}


# ------------------------------------------------------------------ the inputs

def _sections(c, w):
    """Byte offsets of codes, scales, minima and position parts within a record of width w, and the bytes of each in one layer."""
    L, T = c["L"], c["T"]
    each = [T * c["Dc"] * w // 8] + ([0, 0] if w == 16 else [T * (c["Dc"] // c["G"]) * (2 if c["fmt"] == 3 else 4)] * 2) + [T * c["Dr"] * 2]
    return [L * sum(each[:i]) for i in range(4)], each


def _codes(c, x, w):
    """Codes, scales and minima [..][Dc / G][G | 1] of fp16 values, as the record format has them: binary32, the scale rounded to how
    it is held first, quotients to the nearest."""
    held = torch.float16 if c["fmt"] == 3 else torch.float32
    g = x.float().unflatten(-1, (c["Dc"] // c["G"], c["G"]))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    scale = ((hi - lo) / torch.full_like(hi, 2 ** w - 1)).to(held)          # (a tensor: a number would be divided by as a factor)
    wide = scale.double()
    code = torch.where(wide == 0, 0.0, ((g - lo).double() / torch.where(wide == 0, 1.0, wide)).float().round().clamp(0, 2 ** w - 1))
    return code, scale, lo.to(held)


def _packed(code, w):
    """Codes [.., n] as bytes, the lowest index in the lowest bits."""
    code = code.to(torch.uint8).unflatten(-1, (-1, 8 // w))
    shift = torch.arange(0, 8, w, device=DEV, dtype=torch.uint8)
    return (code << shift).sum(-1, dtype=torch.int32).to(torch.uint8)


def _fill(c, pool, off, bits, gen, mult):
    """Random records: values drawn, quantised and packed page by page (a batch of pages of one width at a time)."""
    L, T, Dc = c["L"], c["T"], c["Dc"]
    words = pool.view(torch.int64)
    for w in (16, 8, 4, 2):
        at = off[bits == w]
        step = max(1, (1 << 27) // (L * T * Dc))
        first, _ = _sections(c, w)
        for i in range(0, len(at), step):
            base = torch.from_numpy(at[i:i + step] // 8).to(DEV)
            x = torch.randn((len(base), L, T, Dc), generator=gen, device=DEV).mul_(mult).half()

            def put(section, data):
                data = data.reshape(len(base), -1).contiguous().view(torch.uint8).view(torch.int64)
                words[(base[:, None] + section // 8) + torch.arange(data.shape[1], device=DEV)] = data

            if w == 16:
                put(first[0], x)
            else:
                code, scale, low = _codes(c, x, w)
                put(first[0], _packed(code.flatten(-2), w))
                put(first[1], scale)
                put(first[2], low)
            put(first[3], torch.randn((len(base), L, T, c["Dr"]), generator=gen, device=DEV).half())


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV).manual_seed(seed * 7 + 5)
    bits = _page_widths(c)
    seqs, pages, H, Dc, Dr = c["seqs"], bits.shape[1], c["H"], c["Dc"], c["Dr"]
    size = np.array([_record_bytes(c, w) if w else 0 for w in range(17)], dtype=np.int64)[bits]
    order = np.random.RandomState(seed % 2 ** 31).permutation(seqs * pages)          # pages lie in the pool in any order
    off = np.zeros(seqs * pages, dtype=np.int64)
    off[order] = np.cumsum(size.reshape(-1)[order]) - size.reshape(-1)[order]
    off = off.reshape(seqs, pages)
    pool = torch.zeros(int(size.sum()), dtype=torch.uint8, device=DEV)
    mult = 1.0 + 3.0 * (torch.rand((Dc,), generator=gen, device=DEV) < 0.01)
    _fill(c, pool, off, bits, gen, mult)
    length, new = np.array(_lengths(c)), np.array(_new_rows(c))
    put = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(device=DEV, dtype=t)  # noqa: E731
    state = {"case": c, "layer": c["L"] - 1, "pool": pool, "off": put(off, torch.int64), "bits": put(bits, torch.uint8),
             "len": put(length, torch.int32), "row_start": put(np.concatenate([[0], np.cumsum(new)]), torch.int32)}
    n_rows = int(new.sum())
    if c["kind"] in ("append", "round", "step"):
        # the latents after their norm, the position parts where their rotation leaves them: beside each other
        new_kv = torch.randn((n_rows, Dc + Dr), generator=gen, device=DEV)
        new_kv[:, :Dc] *= mult
        new_kv = new_kv.half()
        state["c"], state["r"] = new_kv[:, :Dc], new_kv[:, Dc:]
    if c["kind"] in ("read", "round"):
        state["c_out"] = torch.empty((n_rows, Dc), dtype=torch.float16, device=DEV)
        state["r_out"] = torch.empty((n_rows, Dr), dtype=torch.float16, device=DEV)
    if c["kind"] in ("attend", "prompt", "step"):
        state["q"] = (2 * torch.randn((n_rows, H, c["Dk"] + Dr), generator=gen, device=DEV)).half()
        state["w"] = (torch.randn((Dc, H, c["Dk"] + c["Dv"]), generator=gen, device=DEV) / math.sqrt(Dc)).half()
        state["out"] = torch.empty((n_rows, H, c["Dv"]), dtype=torch.float16, device=DEV)
    # which row is which token: what the plain forms index with
    state["row_seq"] = put(np.repeat(np.arange(seqs), new), torch.int64)
    state["row_slot"] = put(np.concatenate([np.arange(n - r, n) for n, r in zip(length, new)]), torch.int64)
    state["row_nth"] = put(np.concatenate([np.arange(r) for r in new]), torch.int64)
    state["of_width"] = {w: put(np.flatnonzero(bits.reshape(-1) == w), torch.int64) for w in (16, 8, 4, 2) if (bits == w).any()}
    state["rows_of_width"] = {w: torch.nonzero(state["bits"][state["row_seq"], state["row_slot"] // c["T"]] == w)[:, 0] for w in state["of_width"]}
    if own:
        import paper_2403_11805_amd as kvs
        shape = kvs.LatentShape(c["L"], H, Dc, Dr, c["Dk"], c["Dv"], _capacity(c), c["T"], c["G"], c["fmt"])
        state["pages"] = kvs.LatentPages(shape, pool, state["off"], state["bits"], state["len"])
        state["tokens"] = int(length.sum())
        if c["kind"] in ("attend", "step"):
            need = kvs.kv_latent_attend_workspace_bytes(shape, seqs, c["rows"])
            state["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
        if c["kind"] == "prompt":
            need = kvs.kv_latent_prompts_workspace_bytes(shape, seqs, state["tokens"])
            state["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return state


# ------------------------------------------------------------------ the plain forms

def _at_width(c, st, w):
    """fp16 rows [pages of this width][T][Dc + Dr] of the state's layer: codes times scale, plus minimum, in binary32, rounded."""
    T, Dc, G, layer = c["T"], c["Dc"], c["G"], st["layer"]
    base = st["off"].view(-1)[st["of_width"][w]] // 8
    first, each = _sections(c, w)
    words = st["pool"].view(torch.int64)

    def part(i):
        return words[base[:, None] + (first[i] + layer * each[i]) // 8 + torch.arange(each[i] // 8, device=DEV)]

    r = part(3).view(torch.float16).view(-1, T, c["Dr"])
    if w == 16:
        return torch.cat([part(0).view(torch.float16).view(-1, T, Dc), r], -1)
    kind = torch.float16 if c["fmt"] == 3 else torch.float32
    scale, low = part(1).view(kind).view(-1, T, Dc // G, 1).float(), part(2).view(kind).view(-1, T, Dc // G, 1).float()
    raw = part(0).view(torch.uint8).view(-1, T, Dc * w // 8, 1)
    code = (raw >> torch.arange(0, 8, w, device=DEV, dtype=torch.uint8)) & (2 ** w - 1)
    x = code.view(-1, T, Dc // G, G).float() * scale
    return torch.cat([(x + low).half().view(-1, T, Dc), r], -1)


def _pages_rows(st):
    """fp16 [seqs][N][Dc + Dr]"""
    c = st["case"]
    seqs, N, T = c["seqs"], _capacity(c), c["T"]
    kv = torch.zeros((seqs * (N // T), T, c["Dc"] + c["Dr"]), dtype=torch.float16, device=DEV)
    held = {w: _at_width(c, st, w) for w in st["of_width"]}
    kv[torch.cat(list(st["of_width"].values()))] = torch.cat(list(held.values()))
    return kv.view(seqs, N, -1)


def _plain_read(st):
    rows = _pages_rows(st)[st["row_seq"], st["row_slot"]]
    st["c_out"].copy_(rows[:, :st["case"]["Dc"]])
    st["r_out"].copy_(rows[:, st["case"]["Dc"]:])


def _put_rows(st, w):
    """The new rows whose pages have width w, into them: every section's bytes of a token lie together."""
    c, pick = st["case"], st["rows_of_width"][w]
    T, layer = c["T"], st["layer"]
    seq, slot = st["row_seq"][pick], st["row_slot"][pick]
    page, in_page = st["off"][seq, slot // T], slot % T
    first, each = _sections(c, w)
    x = st["c"][pick]
    parts = (x, None, None) if w == 16 else _codes(c, x, w)
    parts = [parts[0] if w == 16 else _packed(parts[0].flatten(-2), w), parts[1], parts[2], st["r"][pick]]

    def put(i):
        data = parts[i].reshape(len(pick), -1).contiguous().view(torch.uint8)
        wide = {0: torch.int64, 2: torch.int16}.get(data.shape[1] % 8, torch.int32)
        n = data.shape[1] * data.element_size() // torch.empty((), dtype=wide).element_size()
        size = data.shape[1] // n
        at = (page + first[i] + layer * each[i] + in_page * data.shape[1]) // size
        st["pool"].view(wide)[at[:, None] + torch.arange(n, device=DEV)] = data.view(wide)

    return [put(i) for i in ((0, 3) if w == 16 else (0, 1, 2, 3))]


def _plain_append(st):
    return [_put_rows(st, w) for w in st["rows_of_width"] if len(st["rows_of_width"][w])]


def _plain_attend(st, absorbed):
    c = st["case"]
    seqs, N, R, H, Dc, Dr, Dk, Dv = c["seqs"], _capacity(c), max(_new_rows(c)), c["H"], c["Dc"], c["Dr"], c["Dk"], c["Dv"]
    kv = _pages_rows(st).float()
    w = st["w"].float().transpose(0, 1)                                                # [H][Dc][Dk + Dv]
    w_k, w_v = w[..., :Dk].contiguous(), w[..., Dk:].contiguous()
    q = torch.zeros((seqs, R, H, Dk + Dr), device=DEV)
    q[st["row_seq"], st["row_nth"]] = st["q"].float()
    q = q.transpose(1, 2).contiguous()                                                 # [seqs][H][R][Dk + Dr]
    if absorbed:
        q = torch.cat([torch.matmul(q[..., :Dk], w_k.transpose(1, 2).contiguous()), q[..., Dk:]], -1)
        s = torch.matmul(q.view(seqs, H * R, Dc + Dr), kv.transpose(1, 2).contiguous()).view(seqs, H, R, N)
    else:
        k = torch.cat([torch.matmul(kv[:, None, :, :Dc], w_k), kv[:, None, :, Dc:].expand(seqs, H, N, Dr)], -1)
        s = torch.matmul(q, k.transpose(2, 3).contiguous())
    s.mul_(1 / math.sqrt(Dk + Dr))
    # row r of a sequence's n new tokens is token len - n + r and sees the tokens up to itself; surplus rows see nothing
    n_new = (st["row_start"][1:] - st["row_start"][:-1])[:, None]
    nth = torch.arange(R, device=DEV)
    at = torch.where(nth < n_new, st["len"][:, None] - n_new + nth, -1)
    seen = torch.arange(N, device=DEV) <= at[:, :, None]
    s.masked_fill_(~seen[:, None], -INF)
    s.sub_(s.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    s.div_(s.sum(-1, keepdim=True).clamp(min=1e-30))
    if absorbed:
        o = torch.matmul(torch.matmul(s.view(seqs, H * R, N), kv[..., :Dc].contiguous()).view(seqs, H, R, Dc), w_v)
    else:
        o = torch.matmul(s, torch.matmul(kv[:, None, :, :Dc], w_v))
    st["out"].copy_(o.transpose(1, 2)[st["row_seq"], st["row_nth"]])


# ------------------------------------------------------------------ one pass

def run(state):
    st, c = state, state["case"]
    kind, layer = c["kind"], state["layer"]
    if own:
        import paper_2403_11805_amd as kvs
        starts = st["row_start"] if c["rows"] > 1 else None
        if kind in ("append", "round", "step"):
            kvs.kv_latent_append_tokens(st["pages"], layer, st["c"], st["r"], row_start=starts)
        if kind in ("read", "round"):
            kvs.kv_latent_read_tokens(st["pages"], layer, st["c_out"], st["r_out"], row_start=starts)
        if kind in ("attend", "step"):
            kvs.kv_latent_attend_tokens(st["pages"], layer, st["q"], st["w"], st["workspace"], st["out"], row_start=starts, max_rows=c["rows"])
        if kind == "prompt":
            kvs.kv_latent_attend_prompts(st["pages"], layer, st["q"], st["w"], st["workspace"], st["out"], st["tokens"], row_start=starts)
    else:
        if kind in ("append", "round", "step"):
            _plain_append(st)
        if kind in ("read", "round"):
            _plain_read(st)
        if kind in ("attend", "step", "prompt"):
            _plain_attend(st, kind != "prompt")
    if kind == "append":
        return {"pool": st["pool"].view(torch.float16)}
    if kind in ("read", "round"):
        return {"c": st["c_out"], "r": st["r_out"]}
    if kind == "step":          # the new token's row is fp16; the packed pages beside it are inputs, as bytes
        return {"out": st["out"], "pool": st["pool"]}
    return {"out": st["out"]}


# ------------------------------------------------------------------ in 64 bits

def _page_values(c, st, s, i):
    """Page i of sequence s in 64 bits: latents [T][Dc] as they are rounded to fp16 when read, position parts [T][Dr]."""
    L, T, Dc, w, layer = c["L"], c["T"], c["Dc"], int(st["widths"][s, i]), st["layer"]
    start = int(st["starts"][s, i])
    record = st["pool"][start:start + _record_bytes(c, w)]
    r = record[-L * T * c["Dr"] * 2:].view(torch.float16).view(L, T, -1)[layer].double()
    if w == 16:
        return record[:L * T * Dc * 2].view(torch.float16).view(L, T, Dc)[layer].double(), r
    n_codes = L * T * Dc * w // 8
    kind = torch.float16 if c["fmt"] == 3 else torch.float32
    d = torch.arange(Dc, device=DEV)
    code = record[:n_codes].view(L, T, -1)[layer].long()[..., d * w // 8]
    code = torch.bitwise_and(torch.bitwise_right_shift(code, d % (8 // w) * w), 2 ** w - 1)
    scale, low = (p[layer].double()[..., d // c["G"]] for p in record[n_codes:-L * T * c["Dr"] * 2].view(kind).view(2, L, T, Dc // c["G"]))
    return (code.double() * scale + low).half().double(), r


def exact(case, seed):
    """Attention a sequence and a head at a time, from keys and values.  What fp16 appends give are the inputs' own values in
    other places; nothing is computed that could be off."""
    c = dict(case)
    if c["kind"] == "append":
        return None
    st = prepare(case, seed)
    st["widths"], st["starts"] = st["bits"].cpu().numpy(), st["off"].cpu().numpy()
    T, Dc, Dr, Dk, H = c["T"], c["Dc"], c["Dr"], c["Dk"], c["H"]
    out, latents, positions, row = [], [], [], 0
    for s, (n, r) in enumerate(zip(_lengths(c), _new_rows(c))):
        if c["kind"] == "round":
            # what a row comes back as: its codes at its page's width, scales rounded as they are held
            for j, slot in enumerate(range(n - r, n)):
                if j == 0 or slot % T == 0:
                    k = min(r - j, T - slot % T)
                    x, w = st["c"][row + j:row + j + k].double().view(k, Dc // c["G"], c["G"]), int(st["widths"][s, slot // T])
                    low, span = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True) - x.amin(-1, keepdim=True)
                    step = (span / torch.full_like(span, 2 ** w - 1)).float()
                    step = (step.half() if c["fmt"] == 3 else step).double()
                    code = ((x - low) / step).float().round().clamp(max=2 ** w - 1).double()
                    latents.append(torch.where(step > 0, code * step + low, low).view(k, Dc))
            positions.append(st["r"][row:row + r].double())
            row += r
            continue
        pages = [_page_values(c, st, s, i) for i in range(-(-n // T))]
        lat, pos = (torch.cat([p[i] for p in pages])[:n] for i in (0, 1))
        if c["kind"] == "read":
            latents.append(lat[n - r:])
            positions.append(pos[n - r:])
            continue
        if c["kind"] == "step":
            lat[n - 1], pos[n - 1] = st["c"][s].double(), st["r"][s].double()
        found = torch.empty((r, H, c["Dv"]), dtype=torch.float64, device=DEV)
        unseen = torch.arange(n, device=DEV)[None, :] > torch.arange(n - r, n, device=DEV)[:, None]
        for h in range(H):
            kv = torch.mm(lat, st["w"][:, h].double())
            q = st["q"][row:row + r, h].double()
            logits = torch.mm(q[:, :Dk].contiguous(), kv[:, :Dk].t().contiguous()) + torch.mm(q[:, Dk:].contiguous(), pos.t().contiguous())
            a = torch.softmax((logits / (Dk + Dr) ** 0.5).masked_fill(unseen, -INF), -1)
            found[:, h] = torch.mm(a, kv[:, Dk:].contiguous())
        out.append(found)
        row += r
    if c["kind"] in ("read", "round"):
        return {"c": torch.cat(latents), "r": torch.cat(positions)}
    found = {"out": torch.cat(out)}
    return found | {"pool": None} if c["kind"] == "step" else found
