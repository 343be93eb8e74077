"""The paged key/value cache of chunked generation: what is timed, and what it has to return.

A clip is generated chunk by chunk: the tokens of a new chunk (one token, a latent
frame, a few frames) project their keys and values, which are written into pages of
a pool that many clips share, and their queries attend to everything that their clip
has in the cache.  Three operators: echo_kv_write (the pages hold bf16, or int8 codes
with one fp32 scale per token and head, quantised as they are written), echo_kv_read
(the cached rows of each sequence again, contiguous and in the compute precision) and
echo_kv_attention (a chunk of any number of new rows per sequence, single rows among
them, over the pages).

Layouts, the same for the plain forms and the kernels:
  pages  [n_pages, 2, H, page, d] int8 or bf16 (0: keys, 1: values)
  scale  f32 [n_pages, 2, H, page] for int8
  table  int32 [seqs, max_pages]: the pages of each sequence in order, -1 past the last
  lens   int32 [seqs]: tokens of each sequence, the new ones included
  row0   int32 [seqs + 1]: the new rows of sequence b are row0[b] .. row0[b + 1] - 1, and
         they stand at the last positions of the sequence
A row at position p sees the keys below min(len, (p // causal_block + 1) * causal_block),
or all of them where causal_block is 0.

Sizes come from synth/configs.py (2, 16 and 40 heads of 64 and 128; frames of 1560
tokens; 256 to 63960 tokens) or are generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
MOST_FLOPS = 1.5e12     # of the largest listed case; no drawn one takes more
MOST_SCORES = 3.2e9     # values of the plain form's score tensor


def listed():
    return [
        # one generated token of each of 64 sequences, quantised as it is stored
        dict(name="store_tokens_64_int8", op="store", form="int8", page=16, H=8, d=128, seqs=64,
             len=4096, rows=1, ragged=False, src="bf16"),
        # one new latent frame at the end of the long clip, quantised
        dict(name="store_frame_1560_int8", op="store", form="int8", page=64, H=40, d=128, seqs=1,
             len=32760, rows=1560, ragged=False, src="bf16"),
        # prompts of five sequences at once, kept in bf16, from fp32 projections
        dict(name="store_ragged_bf16", op="store", form="bf16", page=32, H=16, d=64, seqs=5,
             len=4681, rows=4681, ragged=True, src="f32"),
        # the whole cached clip read back in the compute precision
        dict(name="load_clip_32760_int8", op="load", form="int8", page=64, H=40, d=128, seqs=1,
             len=32760, rows=32760, ragged=False, dst="bf16"),
        # ragged sequences of the mid-size model, small pages, in fp32
        dict(name="load_ragged_int8_f32", op="load", form="int8", page=16, H=16, d=64, seqs=7,
             len=1999, rows=1999, ragged=True, dst="f32"),
        # a single new token of a short sequence: the latency of a call
        dict(name="token_257", op="attend", form="bf16", page=16, H=16, Hq=16, d=64, seqs=1,
             len=257, rows=1, ragged=False, cb=1),
        # a step of a serving batch: one token each, ragged lengths, shared heads, int8
        dict(name="tokens_48x8190_int8", op="attend", form="int8", page=64, H=8, Hq=32, d=128,
             seqs=48, len=8190, rows=1, ragged=False, cb=1),
        # one token of one very long sequence: few rows, a long axis
        dict(name="token_131071", op="attend", form="bf16", page=128, H=8, Hq=64, d=128, seqs=1,
             len=131071, rows=1, ragged=False, cb=1),
        # a few tokens of each sequence (drafts under verification), no shared heads
        dict(name="drafts_8x17_int8", op="attend", form="int8", page=32, H=16, Hq=16, d=64, seqs=8,
             len=7800, rows=17, ragged=False, cb=1),
        # prompts in pieces: ragged chunks over ragged caches, token by token causal
        dict(name="chunks_6x2001_bf16", op="attend", form="bf16", page=16, H=8, Hq=32, d=64,
             seqs=6, len=9001, rows=2001, ragged=True, cb=1),
        # one new latent frame over the long clip of the 40-head block
        dict(name="frame_1560x32760_bf16", op="attend", form="bf16", page=128, H=40, Hq=40, d=128,
             seqs=1, len=32760, rows=1560, ragged=False, cb=0),
        # two new frames, causal frame by frame, over the int8 cache
        dict(name="frames_3120x24960_int8", op="attend", form="int8", page=64, H=40, Hq=40, d=128,
             seqs=1, len=24960, rows=3120, ragged=False, cb=1560),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    form, page, d = rng.choice(("int8", "bf16")), rng.choice((16, 32, 64, 128)), rng.choice((64, 128))
    op = rng.choice(("store", "load", "attend", "attend", "attend", "attend"))
    if op != "attend":
        seqs = rng.choice((1, 1, _log(rng, 2, 64)))
        H = rng.randint(1, 40)
        most = max(2, int(6.4e8 / (H * d * seqs)))
        n = _log(rng, 1, min(32760, most))
        c = dict(op=op, form=form, page=page, H=H, d=d, seqs=seqs)
        if op == "load":
            return dict(c, len=n, rows=n, ragged=seqs > 1, dst=rng.choice(("bf16", "f32")))
        rows = rng.choice((1, _log(rng, 1, n), n))
        return dict(c, len=n, rows=rows, ragged=seqs > 1 and rows > 1, src=rng.choice(("bf16", "f32")))
    kind = rng.choice(("token", "drafts", "chunk", "chunk"))
    seqs = rng.choice((1, _log(rng, 2, 64))) if kind != "chunk" else rng.choice((1, 1, _log(rng, 2, 12)))
    group = rng.choice((1, 1, 2, 3, 4, 5, 8))
    H = rng.randint(1, max(1, 40 // group))
    rows = 1 if kind == "token" else _log(rng, 2, 40) if kind == "drafts" else _log(rng, 41, 4680)
    cb = rng.choice((1, 1, 0)) if kind != "chunk" else rng.choice((0, 1, rng.randint(64, 1560)))
    c = dict(op="attend", form=form, page=page, H=H, Hq=H * group, d=d, seqs=seqs,
             len=max(rows, _log(rng, 64, 131071 if kind == "token" else 63960)), rows=rows,
             ragged=kind == "chunk" and seqs > 1, cb=cb)
    while (work(c)["flops"] > MOST_FLOPS or work(c)["bytes"] > 1.2e9
           or float(c["seqs"]) * c["Hq"] * c["rows"] * c["len"] > MOST_SCORES):
        c["len"] = max(1, c["len"] * 3 // 4)
        c["rows"] = max(1, min(c["rows"], c["len"]) * 7 // 8) if c["rows"] > 1 else 1
    return c


def sizes(c):
    """(tokens, new rows) of each sequence: spread between a quarter and the whole of the
    case's where there are several (the rows only where they are ragged)."""
    def spread(most, b, on):
        if not on or c["seqs"] == 1:
            return most
        return max(1, round(most * (0.25 + 0.75 * ((b + 1) * 0.6180339887 % 1.0))))
    lens = [spread(c["len"], b, True) for b in range(c["seqs"])]
    if c["op"] == "load":
        return lens, list(lens)
    rows = [min(n, spread(c["rows"], b + 3, c["ragged"])) for b, n in enumerate(lens)]
    return lens, rows


def _seen(c, n, rows):
    """Keys that the rows of one sequence see, in all."""
    if c["cb"] == 0:
        return rows * n
    return sum(min(n, (p // c["cb"] + 1) * c["cb"]) for p in range(n - rows, n))


def work(c):
    lens, rows = sizes(c)
    H, d, n = c["H"], c["d"], sum(rows)
    cached = 2 * H * (d + 4 if c["form"] == "int8" else 2 * d)     # a token's keys and values
    size = {"bf16": 2, "f32": 4}
    if c["op"] == "store":
        values = 2 * n * H * d
        back = 2 * values if c["form"] == "int8" else 0             # read back in bf16
        return {"bytes": values * size[c["src"]] + n * cached + back, "flops": 0}
    if c["op"] == "load":
        return {"bytes": n * cached + 2 * n * H * d * size[c["dst"]], "flops": 0}
    return {"bytes": sum(lens) * cached + 2 * n * c["Hq"] * d * 2,
            "flops": 4.0 * c["Hq"] * d * sum(_seen(c, a, b) for a, b in zip(lens, rows))}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def prepare(c, seed):
    """The pool with every sequence's earlier tokens in it, the page table, and the new
    rows: their keys and values side by side as one projection leaves them, or their
    queries.  Keys have a part that all tokens share, as a trained model's do; pages
    stand in the pool in no order, and some belong to no sequence."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1))

    def randn(*shape, dtype=BF16):
        out = torch.empty(*shape, dtype=dtype, device=DEV)
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 26):
            n = min(1 << 26, flat.numel() - i)
            flat[i:i + n] = torch.randn(n, generator=g, device=DEV, dtype=F32)
        return out

    lens, rows = sizes(c)
    H, d, page, B = c["H"], c["d"], c["page"], c["seqs"]
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).to(I32).cpu()
    table = torch.full((B, max(need)), -1, dtype=I32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s = {"case": c, "n": sum(rows), "rows": max(rows), "table": table.to(DEV),
         "lens": torch.tensor(lens, dtype=I32, device=DEV),
         "row0": torch.tensor([sum(rows[:b]) for b in range(B + 1)], dtype=I32, device=DEV)}
    if c["form"] == "int8":
        s["pages"] = torch.randint(-127, 128, (n_pages, 2, H, page, d), generator=g, device=DEV,
                                   dtype=torch.int8)
        s["scale"] = (0.7 + 0.6 * torch.rand(n_pages, 2, H, page, generator=g, device=DEV)) / 64
    else:
        s["pages"], s["scale"] = randn(n_pages, 2, H, page, d), None
        s["pages"][:, 0] += randn(1, H, 1, d)
    if c["op"] == "store":
        kv = randn(s["n"], 2 * H * d, dtype=BF16 if c["src"] == "bf16" else F32)
        kv[:, :H * d] += randn(1, H * d, dtype=kv.dtype)
        s["k"], s["v"] = kv[:, :H * d], kv[:, H * d:]
    elif c["op"] == "attend":
        s["q"] = randn(s["n"], c["Hq"] * d)
    if own:
        # the handles that a program makes once (the pool of a layer, the batch of a step,
        # which all layers share) and the buffers that it keeps; they hold no data of their own
        from paper_2608_02474_gb300 import echocache as ec
        s["ec"], s["pool"] = ec, ec.KVPool(s["pages"], s["scale"])
        s["batch"] = ec.KVBatch(s["table"], s["lens"], s["row0"], s["n"], s["rows"])
        if c["op"] == "attend":
            s["out"] = torch.empty_like(s["q"])
            s["ws"] = torch.empty(ec.echo_kv_attention_workspace_size(s["pool"], s["batch"], c["Hq"]),
                                  dtype=torch.uint8, device=DEV)
        elif c["op"] == "load" or c["form"] == "int8":
            t = F32 if c.get("dst") == "f32" else BF16
            s["back"] = [torch.empty(s["n"], H * d, dtype=t, device=DEV) for _ in range(2)]
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if own:
        ec, pool, batch = s["ec"], s["pool"], s["batch"]
        if c["op"] == "attend":
            return ec.echo_kv_attention(pool, batch, s["q"], causal_block=c["cb"], out=s["out"],
                                        workspace=s["ws"])
        if c["op"] == "store":
            ec.echo_kv_write(pool, batch, s["k"], s["v"])
            if c["form"] == "bf16":
                return s["pages"]
        return ec.echo_kv_read(pool, batch, k=s["back"][0], v=s["back"][1])
    if c["op"] == "attend":
        return _attend(s)
    if c["op"] == "store":
        _store(s)
        if c["form"] == "bf16":
            return s["pages"]
    return _load(s, F32 if c.get("dst") == "f32" else BF16)


def _places(s):
    """Page and place in the page of every new row."""
    page = s["case"]["page"]
    r = torch.arange(s["n"], device=DEV)
    b = torch.bucketize(r, s["row0"][1:], right=True)
    p = s["lens"][b] - s["row0"][b + 1] + r
    return s["table"][b, p // page].long(), p % page


def _store(s):
    c = s["case"]
    pg, at = _places(s)
    for i, src in enumerate((s["k"], s["v"])):
        x = src.float().view(s["n"], c["H"], c["d"])
        if c["form"] == "bf16":
            s["pages"][pg, i, :, at] = x.to(BF16)
            continue
        a = x.abs().amax(dim=2, keepdim=True)
        inv = torch.where(a > 0, 127 / a, torch.zeros_like(a))
        s["pages"][pg, i, :, at] = torch.round(x * inv).clamp(-127, 127).to(torch.int8)
        s["scale"][pg, i, :, at] = (a / 127)[..., 0]


def _load(s, dtype):
    c = s["case"]
    pg, at = _places(s)
    out = []
    for i in range(2):
        x = s["pages"][pg, i, :, at].float()
        if c["form"] == "int8":
            x = x * s["scale"][pg, i, :, at][..., None]
        out.append(x.to(dtype).view(s["n"], c["H"] * c["d"]))
    return tuple(out)


def _attend(s):
    """All sequences at once, padded to the longest; a row's sum over no keys is 0."""
    c = s["case"]
    H, d, page, B = c["H"], c["d"], c["page"], c["seqs"]
    G, R, n = c["Hq"] // H, s["rows"], s["n"]
    pages = s["pages"][s["table"].clamp(min=0).long()].float()      # [B, pages, 2, H, page, d]
    if c["form"] == "int8":
        pages = pages * s["scale"][s["table"].clamp(min=0).long()][..., None]
    kv = pages.permute(2, 0, 3, 1, 4, 5).reshape(2, B, H, -1, d)    # keys and values in order
    L = kv.shape[3]
    r = torch.arange(n, device=DEV)
    b = torch.bucketize(r, s["row0"][1:], right=True)
    i = r - s["row0"][b]
    q = torch.zeros(B, R, H, G, d, device=DEV)
    q[b, i] = s["q"].float().view(n, H, G, d)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, H, R * G, d)
    x = (q @ kv[0].transpose(2, 3)) / math.sqrt(d)
    lens = s["lens"].long()[:, None]
    pos = lens - (s["row0"][1:] - s["row0"][:-1])[:, None] + torch.arange(R, device=DEV)
    cb = c["cb"]
    seen = torch.minimum(lens, (pos // cb + 1) * cb) if cb else lens.expand(B, R)
    hide = torch.arange(L, device=DEV) >= seen.repeat_interleave(G, dim=1)[:, :, None]
    x.masked_fill_(hide[:, None], -math.inf)
    m = x.amax(dim=3, keepdim=True)
    x.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    total = x.sum(dim=3, keepdim=True)
    o = (x @ kv[1]) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.view(B, H, R, G, d).permute(0, 2, 1, 3, 4)[b, i]
    return o.reshape(n, H * G * d).to(BF16)


# ---------------------------------------------------------------------------
# the definition in 64 bits, sequence by sequence
# ---------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    lens, rows = sizes(c)
    H, d, page = c["H"], c["d"], c["page"]
    table = s["table"].tolist()

    def slots(b, lo, hi):
        p = torch.arange(lo, hi, device=DEV)
        ids = torch.tensor(table[b], device=DEV)
        return ids[torch.div(p, page, rounding_mode="floor")], p.remainder(page)

    def cached(b, lo, hi, i):
        pg, at = slots(b, lo, hi)
        x = s["pages"][pg, i, :, at].to(F64)
        return x * s["scale"][pg, i, :, at].to(F64).unsqueeze(2) if c["form"] == "int8" else x

    first = [sum(rows[:b]) for b in range(len(rows))]
    if c["op"] == "load":
        return tuple(torch.cat([cached(b, 0, n, i).flatten(1) for b, n in enumerate(lens)])
                     for i in range(2))
    if c["op"] == "store":
        if c["form"] == "bf16":
            pages = s["pages"].to(F64)
            for b, n in enumerate(lens):
                pg, at = slots(b, n - rows[b], n)
                for i, src in enumerate((s["k"], s["v"])):
                    pages[pg, i, :, at] = src[first[b]:first[b] + rows[b]].to(F64).view(-1, H, d)
            return pages
        back = []
        for src in (s["k"], s["v"]):
            x = src.to(F64).view(-1, H, d)
            step = x.abs().amax(2, True) / 127
            back.append((torch.where(step > 0, (x / step.clamp(min=1e-300)).round(), 0 * x) * step)
                        .view(-1, H * d))
        return tuple(back)
    G = c["Hq"] // H
    out = torch.zeros(s["n"], c["Hq"], d, dtype=F64, device=DEV)
    for b, n in enumerate(lens):
        k, v = cached(b, 0, n, 0), cached(b, 0, n, 1)
        at = slice(first[b], first[b] + rows[b])
        q = s["q"][at].to(F64).view(rows[b], c["Hq"], d)
        p = torch.arange(n - rows[b], n, device=DEV)
        top = (torch.div(p, c["cb"], rounding_mode="floor") + 1) * c["cb"] if c["cb"] else p * 0 + n
        hidden = torch.arange(n, device=DEV)[None, :] >= top[:, None]
        for h in range(c["Hq"]):
            w = torch.softmax((q[:, h] @ k[:, h // G].T * d ** -0.5).masked_fill(hidden, -math.inf), 1)
            out[at, h] = w @ v[:, h // G]
    return out.view(s["n"], -1)
