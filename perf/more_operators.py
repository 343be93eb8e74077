"""A step of chunked generation around its cache: what is timed, and what it has to return.

Four operators, in the order in which a step uses them:

tables  the page tables and slot maps of a step, built on the GPU from how many new rows each
        clip has (echo_kv_extend), and clips shortened again (echo_kv_shorten).  Clips have
        slots; slot i's pages are table[i], in order, len[i] tokens of them in use; the free
        pages are free[0 .. n_free), taken from the end.  With have = ceil(len / page) and
        want = ceil((len + rows) / page), page j of sequence b (have_b <= j < want_b) is
        free[n_free - 1 - (before_b + j - have_b)], before_b the pages that the sequences
        before it take.  A step's row row0[b] + i stands at position pos = len_b + i, its
        place in the pool is table[b, pos / page] page + pos mod page, and its sequence is b;
        rows behind the last sequence have -1 for all three.  Shortening puts pages back in
        the order that undoes this.
norm    h = alpha x + beta gate N_after(y), n = N_before(h) (1 + scale) + shift over rows of D
        values: N is the layer norm, the norm by the root of the mean square, each with
        or without weights, or nothing; gate, scale and shift are rows of a modulation table
        that a row's index picks.
rotary  the first 2 pairs columns of each head turned by the angle pos f: columns 2 i and
        2 i + 1 (pairs) or i and i + pairs (halves), f = theta^(-i / pairs of the axis), slowed
        down for long contexts; a row's position is one number, or its token index split into
        frame, row and column with some of the pairs each.
int4    keys and values held in 4 bits in the pages (echo_kv_write_at, echo_kv_read,
        echo_kv_attention): 32 neighbouring values u of a head, in bf16, share a scale s, the
        least number of 5 significant bits at or above max |u| / 7 (at least 2^-112); a value's
        code is the nearest whole number to u / s, halves away from zero, stored as code + 8.
        Four bytes, a little-endian word, hold 8 columns: column 2 i in bits 4 i and up, column
        2 i + 1 in bits 16 + 4 i and up.  code s is exact in bf16.
          pages uint8 [n_pages, 2, H, page, d / 2], scale bf16 [n_pages, 2, H, page, d / 32]
        A row at position p sees the keys below min(len, (p // cb + 1) cb), all where cb is 0.

Sizes come from synth/configs.py (16 and 40 heads of 64 and 128; rows of 1024 and 5120
values; frames of 30 rows of 52 tokens; 7800 to 63960 tokens) or are generic.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64
TYPE = {"bf16": BF16, "f32": F32}
SIZE = {"bf16": 2, "f32": 4}
MOST_FLOPS = 1.0e12     # of the largest listed case; no drawn one takes more
MOST_BYTES = 1.3e9
MOST_SCORES = 3.2e9     # values of the plain form's score tensor
FRAME, ROW = 1560, 52   # tokens of a latent frame and of one of its rows


def listed():
    return [
        # four draft tokens of each clip of a serving batch, all rejected afterwards
        dict(name="tables_drafts_200x4", op="tables", seqs=200, slots=256, page=64, len=8190, rows=4, pad=24,
             ragged=False),
        # five clips opened whole, of up to 63960 tokens, and closed again
        dict(name="tables_clips_5x63960", op="tables", seqs=5, slots=8, page=16, len=0, rows=63960, pad=0,
             ragged=True),
        # the middle of a block for the tokens of a serving batch: a call's latency counts
        dict(name="norm_tokens_48x5120", op="norm", rows=48, D=5120, xt="f32", yt="bf16", nt="bf16", after="none",
             before="layer", affine=False, mods=48, mod_t="f32", alpha=1.0, beta=1.0),
        # a whole clip with one modulation per latent frame
        dict(name="norm_clip_32760x5120", op="norm", rows=32760, D=5120, xt="bf16", yt="bf16", nt="bf16",
             after="none", before="layer", affine=False, mods=21, mod_t="f32", alpha=1.0, beta=1.0),
        # the same tokens' queries and shared keys, halves, a context scaled to four times its length
        dict(name="rotary_tokens_48", op="rotary", rows=48, Hq=32, H=8, d=128, t="bf16", layout="halves", pairs=64,
             grid=False, scaling="yarn", factor=4.0, theta=10000.0, far=131072, inverse=False),
        # queries and keys of a whole clip by frame, row and column
        dict(name="rotary_clip_32760", op="rotary", rows=32760, Hq=40, H=40, d=128, t="bf16", layout="pairs",
             pairs=64, grid=True, scaling="none", factor=1.0, theta=10000.0, far=32760, inverse=False),
        # one new latent frame's keys and values into the pages, and back
        dict(name="int4_store_frame_1560", op="store", page=64, H=40, d=128, seqs=1, len=32760, rows=1560,
             ragged=False, t="bf16"),
        # prompts of five sequences at once, from fp32 projections
        dict(name="int4_store_ragged", op="store", page=16, H=16, d=64, seqs=5, len=4681, rows=4681, ragged=True,
             t="f32"),
        # a single new token of a short sequence
        dict(name="int4_token_301", op="attend", page=16, H=16, Hq=16, d=64, seqs=1, len=301, rows=1, ragged=False,
             cb=1),
        # a step of a serving batch: one token each, ragged lengths, shared heads
        dict(name="int4_tokens_48x8190", op="attend", page=64, H=8, Hq=32, d=128, seqs=48, len=8190, rows=1,
             ragged=False, cb=1),
        # drafts under verification, no shared heads
        dict(name="int4_drafts_8x17", op="attend", page=32, H=16, Hq=16, d=64, seqs=8, len=7800, rows=17,
             ragged=False, cb=1),
        # a new latent frame over the whole clip
        dict(name="int4_frame_1560x31200", op="attend", page=64, H=40, Hq=40, d=128, seqs=1, len=31200, rows=1560,
             ragged=False, cb=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "norm", "rotary", "store", "attend", "attend"))
    if op == "tables":
        seqs = _log(rng, 1, 512)
        most = max(1, min(63960, 300000 // seqs))
        return dict(op=op, seqs=seqs, slots=seqs + rng.randint(0, 64), page=rng.choice((16, 32, 64, 128)),
                    len=rng.choice((0, _log(rng, 1, 32760))), rows=_log(rng, 1, most),
                    pad=rng.choice((0, rng.randint(1, 100))), ragged=rng.random() < 0.5)
    if op == "norm":
        rows, D = _log(rng, 1, 32760), 8 * _log(rng, 16, 1024)
        while rows * D > 32760 * 5120:
            rows = rows * 3 // 4
        most = rows * D * 8 < 0.6 * MOST_BYTES            # fp32 takes twice the bytes
        t = ("bf16", "f32") if most else ("bf16",)
        return dict(op=op, rows=rows, D=D, xt=rng.choice(t), yt=rng.choice(t), nt="bf16",
                    after=rng.choice(("none", "layer", "rms")), before=rng.choice(("layer", "rms")),
                    affine=rng.random() < 0.5, mods=rng.choice((1, rows, _log(rng, 1, min(rows, 64)))) if D * rows < 4e7
                    else rng.randint(1, 41), mod_t=rng.choice(("f32", "bf16")),
                    alpha=rng.choice((1.0, rng.uniform(0.5, 2))), beta=rng.choice((1.0, rng.uniform(0.1, 1))))
    if op == "rotary":
        d, grid = rng.choice((64, 128)), rng.random() < 0.4
        H = rng.randint(1, 40)
        Hq = H * rng.choice((1, 1, 2, 4, 5)) if H <= 8 else H
        t = rng.choice(("bf16", "bf16", "f32"))
        most = int(MOST_BYTES / (2 * (H + Hq) * d * SIZE[t]))
        return dict(op=op, rows=_log(rng, 1, min(32760, most)), Hq=Hq, H=H, d=d, t=t,
                    layout=rng.choice(("pairs", "halves")),
                    pairs=rng.choice((d // 2, d // 4, rng.randint(3, d // 2))), grid=grid,
                    scaling="none" if grid else rng.choice(("none", "linear", "ntk", "yarn")),
                    factor=rng.uniform(1, 32), theta=rng.choice((10000.0, 500000.0, 1000000.0)),
                    far=_log(rng, 32768, 1048576), inverse=rng.random() < 0.25)
    page, d = rng.choice((16, 32, 64, 128)), rng.choice((64, 128))
    if op == "store":
        seqs, H = rng.choice((1, 1, _log(rng, 2, 64))), rng.randint(1, 40)
        n = _log(rng, 1, min(32760, max(2, int(6.4e8 / (H * d * seqs)))))
        rows = min(rng.choice((1, _log(rng, 1, n), n)), max(1, int(8e7 / (H * d * seqs))))
        return dict(op=op, page=page, H=H, d=d, seqs=seqs, len=n, rows=rows, ragged=seqs > 1 and rows > 1,
                    t=rng.choice(("bf16", "f32")))
    kind = rng.choice(("token", "drafts", "chunk", "chunk"))
    seqs = rng.choice((1, _log(rng, 2, 64))) if kind != "chunk" else rng.choice((1, 1, _log(rng, 2, 12)))
    group = rng.choice((1, 1, 2, 3, 4, 5, 8))
    H = rng.randint(1, max(1, 40 // group))
    rows = 1 if kind == "token" else _log(rng, 2, 40) if kind == "drafts" else _log(rng, 41, 4680)
    cb = rng.choice((1, 1, 0)) if kind != "chunk" else rng.choice((0, 1, rng.randint(64, 1560)))
    c = dict(op="attend", page=page, H=H, Hq=H * group, d=d, seqs=seqs,
             len=max(rows, _log(rng, 64, 131071 if kind == "token" else 63960)), rows=rows,
             ragged=kind == "chunk" and seqs > 1, cb=cb)
    while (work(c)["flops"] > MOST_FLOPS or work(c)["bytes"] > 0.6e9
           or float(c["seqs"]) * c["Hq"] * c["rows"] * c["len"] > MOST_SCORES):
        c["len"] = max(1, c["len"] * 3 // 4)
        c["rows"] = max(1, min(c["rows"], c["len"]) * 7 // 8) if c["rows"] > 1 else 1
    return c


def sizes(c):
    """(tokens, new rows) of each sequence: spread between a quarter and the whole of the
    case's where there are several (the rows only where they are ragged).  The tables'
    tokens are those before the new rows, the others' with them."""
    def spread(most, b, on):
        if not on or c["seqs"] == 1:
            return most
        return max(1, round(most * (0.25 + 0.75 * ((b + 1) * 0.6180339887 % 1.0))))
    if c["op"] == "tables":
        return ([spread(c["len"], b, True) if c["len"] else 0 for b in range(c["seqs"])],
                [spread(c["rows"], b + 3, c["ragged"]) for b in range(c["seqs"])])
    lens = [spread(c["len"], b, True) for b in range(c["seqs"])]
    return lens, [min(n, spread(c["rows"], b + 3, c["ragged"])) for b, n in enumerate(lens)]


def _seen(c, n, rows):
    """Keys that the rows of one sequence see, in all."""
    if c["cb"] == 0:
        return rows * n
    return sum(min(n, (p // c["cb"] + 1) * c["cb"]) for p in range(n - rows, n))


def axis_pairs(c):
    """Pairs of each axis: an even third for rows and columns each, the rest for frames."""
    if not c["grid"]:
        return [c["pairs"]]
    third = c["pairs"] // 3
    return [c["pairs"] - 2 * third, third, third]


def work(c):
    if c["op"] == "tables":
        lens, rows = sizes(c)
        n, page = sum(rows), c["page"]
        new = sum(-(-(a + r) // page) - -(-a // page) for a, r in zip(lens, rows))
        old = sum(-(-a // page) for a in lens)
        # in: slots, rows, lengths, the earlier pages, the pages taken; out: the batch's table, lengths, first
        # rows and row maps, the slots' new pages and lengths.  Shortening: slots, rows, lengths, pages, back
        extend = 4 * (3 * c["seqs"] + old + new) + 4 * (2 * new + old + 3 * c["seqs"] + 2) + 16 * (n + c["pad"])
        return {"bytes": extend + 4 * (3 * c["seqs"] + new) + 4 * (c["seqs"] + new), "flops": 0}
    if c["op"] == "norm":
        n = c["rows"] * c["D"]
        side = 3 * c["mods"] * c["D"] * SIZE[c["mod_t"]] + 4 * c["rows"]
        if c["affine"]:
            side += 4 * (2 if c["before"] == "layer" else 1) * c["D"]
        return {"bytes": n * (2 * SIZE[c["xt"]] + SIZE[c["yt"]] + SIZE[c["nt"]]) + side, "flops": 14 * n}
    if c["op"] == "rotary":
        n = c["rows"] * (c["Hq"] + c["H"])
        return {"bytes": 2 * n * c["d"] * SIZE[c["t"]] + 4 * c["rows"], "flops": 6 * n * c["pairs"]}
    lens, rows = sizes(c)
    H, d, n = c["H"], c["d"], sum(rows)
    cached = 2 * H * (d // 2 + d // 16)                            # a token's keys and values
    if c["op"] == "store":
        return {"bytes": 2 * n * H * d * (SIZE[c["t"]] + 2) + 2 * n * cached + 16 * n, "flops": 0}
    return {"bytes": sum(lens) * cached + 2 * n * c["Hq"] * d * 2,
            "flops": 4.0 * c["Hq"] * d * sum(_seen(c, a, b) for a, b in zip(lens, rows))}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def prepare(c, seed):
    """A program's state before the call: tables in use with their pages in no order; the
    residual stream, a branch's output and the modulations; queries and keys with their
    positions; a pool with every sequence's earlier tokens in it and the new rows."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1))

    def randn(*shape, dtype=BF16):
        out = torch.empty(*shape, dtype=dtype, device=DEV)
        flat = out.view(-1)
        for i in range(0, flat.numel(), 1 << 26):
            n = min(1 << 26, flat.numel() - i)
            flat[i:i + n] = torch.randn(n, generator=g, device=DEV, dtype=F32)
        return out

    s = {"case": c}
    if own:
        from paper_2608_02474_gb300 import echocache as ec
        s["ec"] = ec
    make = {"tables": _tables_state, "norm": _norm_state, "rotary": _rotary_state}.get(c["op"], _int4_state)
    make(c, s, g, randn)
    return s


def _tables_state(c, s, g, randn):
    lens, rows = sizes(c)
    page, B = c["page"], c["seqs"]
    pages = [-(-a // page) for a in lens]
    want = [-(-(a + r) // page) for a, r in zip(lens, rows)]
    n_pages, width = sum(want) + 7, max(want) + 1
    order = torch.randperm(n_pages, generator=g, device=DEV).to(I32)
    ids = order.cpu()
    slot = torch.randperm(c["slots"], generator=g, device=DEV)[:B].to(I32)
    at, host = 0, torch.full((B, width), -1, dtype=I32)
    for b, n in enumerate(pages):
        host[b, :n] = ids[at:at + n]
        at += n
    s["table"] = torch.full((c["slots"], width), -1, dtype=I32, device=DEV)
    s["table"][slot.long()] = host.to(DEV)
    s["len"] = torch.zeros(c["slots"], dtype=I32, device=DEV)
    s["len"][slot.long()] = torch.tensor(lens, dtype=I32, device=DEV)
    s["free"] = torch.full((n_pages,), -1, dtype=I32, device=DEV)
    s["free"][:n_pages - at] = order[at:]
    s["n_free"] = torch.tensor([n_pages - at], dtype=I32, device=DEV)
    s["slots"], s["rows"] = slot, torch.tensor(rows, dtype=I32, device=DEV)
    n = sum(rows) + c["pad"]
    # what a step keeps from call to call
    s["out"] = dict(table=torch.full((B, width), -1, dtype=I32, device=DEV), len=torch.zeros(B, dtype=I32, device=DEV),
                    row0=torch.zeros(B + 1, dtype=I32, device=DEV), place=torch.zeros(n, dtype=I64, device=DEV),
                    pos=torch.zeros(n, dtype=I32, device=DEV), seq=torch.zeros(n, dtype=I32, device=DEV))
    if own:
        ec, o = s["ec"], s["out"]
        s["tables"] = ec.KVTables(s["table"], s["len"], s["free"], s["n_free"], page)
        s["step"] = ec.KVStep(o["table"], o["len"], o["row0"], o["place"], o["pos"], o["seq"], max(rows))


def _norm_state(c, s, g, randn):
    rows, D = c["rows"], c["D"]
    # a residual stream with a few large columns, and a branch's output next to it
    s["x"] = randn(rows, D, dtype=TYPE[c["xt"]])
    s["x"][:, ::97] *= 8
    s["x"] += 0.5
    s["y"] = randn(rows, D, dtype=TYPE[c["yt"]])
    mod = TYPE[c["mod_t"]]
    table = (0.3 * randn(c["mods"], 3 * D, dtype=F32)).to(mod)     # as one projection leaves them
    s["gate"], s["scale"], s["shift"] = table[:, :D], table[:, D:2 * D], table[:, 2 * D:]
    s["mod_rows"] = torch.div(torch.arange(rows, device=DEV) * c["mods"], rows, rounding_mode="floor").to(I32)
    s["weight"] = s["bias"] = None
    if c["affine"]:
        s["weight"] = 1 + 0.2 * randn(D, dtype=F32)
        s["bias"] = 0.2 * randn(D, dtype=F32) if c["before"] == "layer" else None
    if own:
        ec = s["ec"]
        s["norm"] = ec.GatedNorm(D, c["before"], s["weight"], s["bias"], after=c["after"], alpha=c["alpha"],
                                 beta=c["beta"])
        s["h"] = torch.empty_like(s["x"])
        s["n"] = torch.empty(rows, D, dtype=TYPE[c["nt"]], device=DEV)


def _rotary_state(c, s, g, randn):
    rows, t = c["rows"], TYPE[c["t"]]
    s["q"], s["k"] = randn(rows, c["Hq"] * c["d"], dtype=t), randn(rows, c["H"] * c["d"], dtype=t)
    if c["grid"]:
        first = int(torch.randint(0, 32760, (1,), generator=g, device=DEV))
        s["pos"] = (first + torch.arange(rows, device=DEV)).to(I32)
    elif rows <= 64:
        s["pos"] = torch.randint(0, c["far"], (rows,), generator=g, device=DEV, dtype=I32)
    else:
        first = int(torch.randint(0, max(1, c["far"] - rows), (1,), generator=g, device=DEV))
        s["pos"] = (first + torch.arange(rows, device=DEV)).to(I32)
    turn, s["size"] = _frequencies(c)
    s["freq"] = torch.tensor([f for axis in turn for f in axis], dtype=F64, device=DEV)
    if own:
        ec = s["ec"]
        s["rotary"] = ec.Rotary(c["d"], axis_pairs(c), layout=c["layout"], theta=c["theta"], scaling=c["scaling"],
                                factor=c["factor"], original=4096, frame=(FRAME, ROW) if c["grid"] else None)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])


def _frequencies(c):
    """Angles per position of each axis's pairs, and the factor of the turned columns."""
    out, size = [], 1.0
    for n in axis_pairs(c):
        theta, f = c["theta"], c["factor"]
        if c["scaling"] == "ntk" and n > 1:
            theta *= f ** (n / (n - 1))
        freq = [theta ** (-i / n) for i in range(n)]
        if c["scaling"] == "linear":
            freq = [a / f for a in freq]
        if c["scaling"] == "yarn":
            # by how often a pair turns within the original context: whole above 32, slowed below 1
            keep = [min(1.0, max(0.0, (4096 * a / (2 * math.pi) - 1) / 31)) for a in freq]
            freq = [a * k + a / f * (1 - k) for a, k in zip(freq, keep)]
            size = 0.1 * math.log(f) + 1
        out.append(freq)
    return out, size


def _int4_state(c, s, g, randn):
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
    s.update(n=sum(rows), rows=max(rows), table=table.to(DEV), lens=torch.tensor(lens, dtype=I32, device=DEV),
             row0=torch.tensor([sum(rows[:b]) for b in range(B + 1)], dtype=I32, device=DEV))
    # codes -7 .. 7 in both halves of a byte; scales of 5 significant bits around 1 / 4
    codes = [torch.randint(1, 16, (n_pages, 2, H, page, d // 2), generator=g, device=DEV, dtype=torch.uint8)
             for _ in range(2)]
    s["pages"] = codes[0] | codes[1] << 4
    del codes
    s["scale"] = (torch.randint(16, 32, (n_pages, 2, H, page, d // 32), generator=g, device=DEV) / 96).to(BF16)
    bits = s["scale"].view(torch.int16)
    bits &= -8
    if c["op"] == "store":
        kv = randn(s["n"], 2 * H * d, dtype=TYPE[c["t"]])
        kv[:, :H * d] += randn(1, H * d, dtype=kv.dtype)           # a part that all keys share
        s["k"], s["v"] = kv[:, :H * d], kv[:, H * d:]
        pg, slot = _places(s)
        s["place"] = pg * page + slot                              # the step's slot map
    else:
        s["q"] = randn(s["n"], c["Hq"] * d)
    if own:
        # the handles that a program makes once and the buffers that it keeps
        ec = s["ec"]
        s["pool"] = ec.KVPool(s["pages"], s["scale"])
        s["batch"] = ec.KVBatch(s["table"], s["lens"], s["row0"], s["n"], s["rows"])
        if c["op"] == "attend":
            s["out"] = torch.empty_like(s["q"])
            s["ws"] = torch.empty(ec.echo_kv_attention_workspace_size(s["pool"], s["batch"], c["Hq"]),
                                  dtype=torch.uint8, device=DEV)
        else:
            s["back"] = [torch.empty(s["n"], H * d, dtype=BF16, device=DEV) for _ in range(2)]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    c = s["case"]
    if own:
        ec = s["ec"]
        if c["op"] == "tables":
            ec.echo_kv_extend(s["tables"], s["rows"], s["step"], s["slots"])
            ec.echo_kv_shorten(s["tables"], s["rows"], s["slots"])
            return _tables_out(s)
        if c["op"] == "norm":
            return ec.echo_gated_norm(s["norm"], s["x"], s["y"], s["gate"], s["scale"], s["shift"],
                                      mod_rows=s["mod_rows"], h=s["h"], n=s["n"])
        if c["op"] == "rotary":
            return ec.echo_rotary(s["rotary"], s["pos"], s["q"], s["k"], inverse=c["inverse"], q_out=s["q_out"],
                                  k_out=s["k_out"])
        if c["op"] == "store":
            ec.echo_kv_write_at(s["pool"], s["place"], s["k"], s["v"])
            return ec.echo_kv_read(s["pool"], s["batch"], k=s["back"][0], v=s["back"][1])
        return ec.echo_kv_attention(s["pool"], s["batch"], s["q"], causal_block=c["cb"], out=s["out"],
                                    workspace=s["ws"])
    if c["op"] == "tables":
        return _tables(s)
    if c["op"] == "norm":
        return _norm(s)
    if c["op"] == "rotary":
        return _rotary(s)
    if c["op"] == "store":
        _store(s)
        return tuple(x.view(s["n"], -1).to(BF16) for x in _values(s, *_places(s)))
    return _attend(s)


def _tables_out(s):
    return dict(s["out"], slots_table=s["table"], slots_len=s["len"], free=s["free"], n_free=s["n_free"])


def _tables(s):
    page, o, slot = s["case"]["page"], s["out"], s["slots"].long()
    n = s["len"][slot].long()
    rows = s["rows"].long()
    j = torch.arange(s["table"].shape[1], device=DEV)
    # longer
    have, want = (n + page - 1) // page, (n + rows + page - 1) // page
    need = want - have
    before = need.cumsum(0) - need
    at = s["n_free"] - 1 - (before[:, None] + j - have[:, None])
    t = s["table"][slot]
    t = torch.where((j >= have[:, None]) & (j < want[:, None]), s["free"][at.clamp(0, len(s["free"]) - 1)], t)
    s["table"][slot] = t
    o["table"].copy_(torch.where(j < want[:, None], t, o["table"]))
    s["n_free"] -= need.sum().to(I32)
    s["len"][slot] = (n + rows).to(I32)
    o["len"].copy_((n + rows).to(I32))
    o["row0"][0] = 0
    o["row0"][1:] = rows.cumsum(0).to(I32)
    r = torch.arange(len(o["pos"]), device=DEV)
    b = torch.bucketize(r, o["row0"][1:], right=True)
    live = b < len(rows)
    b = b.clamp(max=len(rows) - 1)
    pos = n[b] + r - o["row0"][b]
    place = t[b, (pos // page).clamp(max=t.shape[1] - 1)].long() * page + pos % page
    for name, v in (("place", place), ("pos", pos), ("seq", b)):
        o[name].copy_(torch.where(live, v, torch.full_like(v, -1)).to(o[name].dtype))
    # and back
    n = s["len"][slot].long()
    cut = torch.minimum(rows, n)
    keep, have = (n - cut + page - 1) // page, (n + page - 1) // page
    drop = have - keep
    before = drop.cumsum(0) - drop
    gone = (j >= keep[:, None]) & (j < have[:, None])
    at = s["n_free"] + drop.sum() - 1 - (before[:, None] + j - keep[:, None])
    spare = torch.full((1,), -1, dtype=I32, device=DEV)
    free = torch.cat((s["free"], spare))                           # what no page goes to: the last entry
    free[torch.where(gone, at, torch.full_like(at, len(s["free"])))] = torch.where(gone, t, spare)
    s["free"].copy_(free[:-1])
    s["n_free"] += drop.sum().to(I32)
    s["len"][slot] = (n - cut).to(I32)
    return _tables_out(s)


def _normed(v, kind, weight=None, bias=None, eps=1e-6):
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(1, keepdim=True) + eps)
    if weight is not None:
        v = v * weight.float()
    return v if bias is None else v + bias.float()


def _norm(s):
    c, m = s["case"], s["mod_rows"].long()
    h = c["alpha"] * s["x"].float() + c["beta"] * s["gate"][m].float() * _normed(s["y"].float(), c["after"])
    n = _normed(h, c["before"], s["weight"], s["bias"]) * (1 + s["scale"][m].float()) + s["shift"][m].float()
    return h.to(s["x"].dtype), n.to(TYPE[c["nt"]])


def _axes(c, pos, dtype):
    """A row's position on the axis of each pair."""
    pos = pos.to(I64)
    if not c["grid"]:
        return pos.to(dtype)[:, None].expand(-1, c["pairs"])
    at = (pos // FRAME, pos % FRAME // ROW, pos % ROW)
    return torch.cat([a.to(dtype)[:, None].expand(-1, n) for a, n in zip(at, axis_pairs(c))], 1)


def _rotary(s):
    c = s["case"]
    angle = _axes(c, s["pos"], F64) * s["freq"]
    cos, sin = (s["size"] * angle.cos()).float()[:, None], (s["size"] * angle.sin()).float()[:, None]
    if c["inverse"]:
        sin = -sin
    out = []
    for x in (s["q"], s["k"]):
        y = x.float().view(c["rows"], -1, c["d"]).clone()
        n = c["pairs"]
        a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["layout"] == "pairs" else (slice(0, n), slice(n, 2 * n))
        x1, x2 = y[:, :, a].clone(), y[:, :, b].clone()
        y[:, :, a] = x1 * cos - x2 * sin
        y[:, :, b] = x2 * cos + x1 * sin
        out.append(y.view(c["rows"], -1).to(x.dtype))
    return tuple(out)


def _places(s):
    """Page and place in the page of every new row."""
    page = s["case"]["page"]
    r = torch.arange(s["n"], device=DEV)
    b = torch.bucketize(r, s["row0"][1:], right=True)
    p = s["lens"][b] - s["row0"][b + 1] + r
    return s["table"][b, p // page].long(), p % page


def _store(s):
    c, page = s["case"], s["case"]["page"]
    pg, at = s["place"] // page, s["place"] % page
    for i, src in enumerate((s["k"], s["v"])):
        u = src.to(BF16).float().view(s["n"], c["H"], c["d"] // 32, 32)
        # the least number of 5 significant bits at or above max / 7: the fp32 quotient's last 19 bits, up
        # (a quotient of two tensors: one by a number is a product with its rounded inverse)
        step = (u.abs().amax(3) / torch.full((1,), 7.0, device=DEV)).clamp(min=2.0 ** -112)
        step = ((step.view(I32) + 0x7FFFF) & ~0x7FFFF).view(F32)
        x = u / step[..., None]
        code = (torch.sign(x) * torch.floor(x.abs() + 0.5) + 8).to(torch.uint8)
        code = code.view(s["n"], c["H"], -1, 4, 2).transpose(3, 4).reshape(s["n"], c["H"], c["d"] // 2, 2)
        s["pages"][pg, i, :, at] = code[..., 0] | code[..., 1] << 4
        s["scale"][pg, i, :, at] = step.to(BF16)


def _value(w, scale):
    """What bytes and scales stand for, in 32 bits."""
    code = torch.stack((w & 15, w >> 4), -1).view(*w.shape[:-1], -1, 2, 4).transpose(-1, -2).float() - 8
    return (code.reshape(*w.shape[:-1], -1, 32) * scale.float()[..., None]).flatten(-2)


def _values(s, pg, at):
    return [_value(s["pages"][pg, i, :, at], s["scale"][pg, i, :, at]) for i in range(2)]


def _attend(s):
    """All sequences at once, padded to the longest; a row's sum over no keys is 0."""
    c = s["case"]
    H, d, B = c["H"], c["d"], c["seqs"]
    G, R, n = c["Hq"] // H, s["rows"], s["n"]
    ids = s["table"].clamp(min=0).long()
    kv = _value(s["pages"][ids], s["scale"][ids])                  # [B, pages, 2, H, page, d]
    kv = kv.permute(2, 0, 3, 1, 4, 5).reshape(2, B, H, -1, d)
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
# the definitions in 64 bits, written apart from the plain forms
# ---------------------------------------------------------------------------
def exact(c, seed):
    if c["op"] == "tables":
        return None                                                # whole numbers only
    s = prepare(c, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "store": _exact_store, "attend": _exact_attend}[c["op"]](c, s)


def _exact_norm(c, s):
    def norm(v, kind):
        if kind == "none":
            return v
        d = v - v.mean(1, True) if kind == "layer" else v
        return d / (d.square().mean(1, True) + 1e-6).sqrt()
    hs, ns = [], []
    for lo in range(0, c["rows"], 4096):
        at = slice(lo, min(c["rows"], lo + 4096))
        m = s["mod_rows"][at].long()
        h = s["x"][at].to(F64) * c["alpha"] + s["gate"][m].to(F64) * norm(s["y"][at].to(F64), c["after"]) * c["beta"]
        n = norm(h, c["before"])
        if s["weight"] is not None:
            n = n * s["weight"].to(F64)
        if s["bias"] is not None:
            n = n + s["bias"].to(F64)
        hs.append(h)
        ns.append(n + n * s["scale"][m].to(F64) + s["shift"][m].to(F64))
    return torch.cat(hs), torch.cat(ns)


def _exact_rotary(c, s):
    at = s["pos"].to(F64)
    if c["grid"]:
        frame = torch.floor(at / FRAME)
        row = torch.floor((at - FRAME * frame) / ROW)
        at = [frame, row, at - FRAME * frame - ROW * row]
    else:
        at = [at]
    freqs, size = _frequencies(c)
    angles = torch.cat([torch.outer(p, torch.tensor(f, dtype=F64, device=DEV)) for p, f in zip(at, freqs)], 1)
    turn = torch.polar(torch.full_like(angles, size), -angles if c["inverse"] else angles)[:, None]
    n, out = c["pairs"], []
    for x in (s["q"], s["k"]):
        x = x.to(F64).view(c["rows"], -1, c["d"])
        part = x[..., :2 * n]
        part = part.unflatten(2, (n, 2)) if c["layout"] == "pairs" else part.unflatten(2, (2, n)).transpose(2, 3)
        part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
        part = part if c["layout"] == "pairs" else part.transpose(2, 3)
        out.append(torch.cat((part.flatten(2), x[..., 2 * n:]), 2).flatten(1))
    return tuple(out)


def _exact_store(c, s):
    out = []
    for src in (s["k"], s["v"]):
        u = src.to(BF16).to(F64).reshape(-1, 32)
        least = (u.abs().amax(1, True) / 7).clamp(min=2.0 ** -112)
        one = torch.exp2(torch.floor(torch.log2(least)) - 4)       # a unit of the fifth bit
        one = torch.where(least / one >= 32, 2 * one, torch.where(least / one < 16, one / 2, one))
        step = torch.ceil(least / one) * one
        out.append((torch.sign(u) * torch.floor((u / step).abs() + 0.5) * step).view(s["n"], -1))
    return tuple(out)


def _exact_attend(c, s):
    lens, rows = sizes(c)
    H, d, page = c["H"], c["d"], c["page"]
    G, out, first = c["Hq"] // H, torch.zeros(s["n"], c["Hq"], d, dtype=F64, device=DEV), 0
    for b, n in enumerate(lens):
        ids = s["table"][b, :-(-n // page)].long()
        kv = []
        for i in range(2):
            w = s["pages"][ids, i].transpose(1, 2).flatten(0, 1)[:n].to(I64)    # [n, H, d / 2]
            word = w[..., 0::4] + 256 * w[..., 1::4] + 65536 * w[..., 2::4] + 16777216 * w[..., 3::4]
            x = torch.empty(n, H, d, dtype=F64, device=DEV)
            for col in range(8):
                x[..., col::8] = ((word >> (4 * (col // 2) + 16 * (col % 2))) % 16 - 8).to(F64)
            sc = s["scale"][ids, i].transpose(1, 2).flatten(0, 1)[:n].to(F64)
            kv.append(x * sc.repeat_interleave(32, dim=2))
        at = slice(first, first + rows[b])
        first += rows[b]
        q = s["q"][at].to(F64).view(rows[b], c["Hq"], d)
        p = torch.arange(n - rows[b], n, device=DEV)
        top = (torch.div(p, c["cb"], rounding_mode="floor") + 1) * c["cb"] if c["cb"] else p * 0 + n
        hidden = torch.arange(n, device=DEV)[None, :] >= top[:, None]
        for h in range(c["Hq"]):
            w = torch.softmax((q[:, h] @ kv[0][:, h // G].T * d ** -0.5).masked_fill(hidden, -math.inf), 1)
            out[at, h] = w @ kv[1][:, h // G]
    return out.view(s["n"], -1)
