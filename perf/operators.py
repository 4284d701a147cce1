"""The paged cache's operators as timed and compared cases: appending keys and values with the position rotation applied
on the way, attention that reads the pages (whole contexts, or a sliding window and a few first tokens that stay visible;
prompts, chunks of prompts and single tokens), and attention for a batch that shares a long prefix.

A case is a dict of plain values:
  op        append | attend | shared
  batch     sequences
  lo, hi    tokens of a sequence in the call (new rows for append, queries for attend and shared): spread over lo..hi
  past      (lowest, highest) rows a sequence's cache holds ahead of them
  hq, hkv, d, dtype, page     heads, storage type, rows of a page
  window, sinks               attend: 0 = whole contexts
  prefix                      shared: rows of the prefix
  rot, pairs                  append: rotated elements of a head, and how they pair up
"""
import math
import random

import torch

own = False

MODEL = dict(hq=32, hkv=8, d=128, dtype="bf16")
SMALL = dict(hq=8, hkv=2, d=64, dtype="fp32")


def listed():
    return [
        # a decode step of a few short sequences of a small model: what counts is the latency of the call
        dict(name="append_4x1_fp32", op="append", batch=4, lo=1, hi=1, past_lo=60, past_hi=500, page=16, rot=64, pairs="halves", **SMALL),
        # a decode step of a large serving batch, one layer
        dict(name="append_256x1", op="append", batch=256, lo=1, hi=1, past_lo=0, past_hi=300, page=16, rot=128, pairs="halves", **MODEL),
        # a prefill step over prompts of very different lengths, half of each head rotated, neighbours paired
        dict(name="append_prompts", op="append", batch=12, lo=200, hi=4096, past_lo=0, past_hi=100, page=64, rot=64,
             pairs="neighbours", **MODEL),
        # a functional check's prompts in fp32, none a multiple of anything
        dict(name="attend_prompts_fp32", op="attend", batch=3, lo=65, hi=512, past_lo=0, past_hi=0, page=16, window=0, sinks=0, **SMALL),
        # one token of one long context: few heads, many rows
        dict(name="attend_1x32k", op="attend", batch=1, lo=1, hi=1, past_lo=32767, past_hi=32767, page=64, window=0, sinks=0, **MODEL),
        # a serving batch's decode step, lengths from short to long, small pages
        dict(name="attend_64_ragged", op="attend", batch=64, lo=1, hi=1, past_lo=1000, past_hi=16000, page=16, window=0, sinks=0, **MODEL),
        # decode over the most recent rows and the attention sinks, whatever the text's length
        dict(name="attend_32_window", op="attend", batch=32, lo=1, hi=1, past_lo=3000, past_hi=32000, page=32, window=2048, sinks=32, **MODEL),
        # a long prompt, every query against all before it
        dict(name="attend_prompt_16k", op="attend", batch=1, lo=16384, hi=16384, past_lo=0, past_hi=0, page=64, window=0, sinks=0, **MODEL),
        # ragged prompts under a sliding window with sinks, three query heads to a KV head, pages that end inside every tile
        dict(name="attend_prompts_window", op="attend", batch=8, lo=500, hi=8192, past_lo=0, past_hi=0, page=48, window=1024, sinks=32,
             hq=24, hkv=8, d=128, dtype="bf16"),
        # the next chunk of prompts that are worked through piece by piece, behind a long cache
        dict(name="attend_chunk", op="attend", batch=4, lo=300, hi=512, past_lo=8000, past_hi=32000, page=64, window=0, sinks=0, **MODEL),
        # a few short questions to one small document in fp32
        dict(name="shared_8_fp32", op="shared", batch=8, lo=1, hi=1, past_lo=0, past_hi=64, page=16, prefix=1000, **SMALL),
        # a decode step of many continuations of one 32k document
        dict(name="shared_64_32k", op="shared", batch=64, lo=1, hi=1, past_lo=0, past_hi=512, page=64, prefix=32768, **MODEL),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every operator, from one token to long prompts, odd sizes, both types, all head layouts."""
    op = rng.choice(["append", "attend", "attend", "attend", "shared"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (8, 2), (16, 2), (8, 8), (40, 8), (24, 8), (16, 1), (9, 3)])
    c = dict(op=op, hq=hq, hkv=hkv, d=rng.choice([128, 128, 64]), dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]),
             page=rng.choice([16, 16, 32, 64, 64, 128, 48, rng.randint(5, 200)]))
    row = hkv * c["d"] * (2 if c["dtype"] == "bf16" else 4)
    if op == "append":
        c["batch"] = _log(rng, 1, 256)
        c["hi"] = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, 24000 // c["batch"]))
        c["past_hi"] = rng.randint(0, 300)
        c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 2, 16, 0])
        c["pairs"] = rng.choice(["halves", "neighbours"])
    elif op == "shared":
        c["batch"], c["hi"] = _log(rng, 2, 96), rng.choice([1, 1, 1, rng.randint(2, 5)])
        c["prefix"], c["past_hi"] = _log(rng, 100, 32768 if c["dtype"] == "bf16" else 8192), _log(rng, 2, 512)
    else:
        kind = rng.choice(["token", "token", "prompt", "chunk"])
        if kind == "token":
            n = _log(rng, 20, 40000)
            c["batch"], c["hi"], c["past_hi"] = _log(rng, 1, max(1, min(64, (1 << 29) // (row * n)))), rng.choice([1, 1, 1, rng.randint(2, 6)]), n
        elif kind == "prompt":
            n = _log(rng, 20, 12000 if c["dtype"] == "bf16" else 3000)
            c["batch"], c["hi"], c["past_hi"] = _log(rng, 1, max(1, min(16, 16000 // n))), n, 0
        else:
            c["batch"], c["hi"], c["past_hi"] = rng.randint(1, 4), _log(rng, 8, 512), _log(rng, 100, 30000 if c["dtype"] == "bf16" else 8000)
        c["window"] = rng.choice([0, 0, _log(rng, 1, 4096)])
        c["sinks"] = rng.choice([0, 4, 32, rng.randint(1, 100)]) if c["window"] else 0
    c["lo"] = c["hi"] if rng.random() < 0.4 else rng.randint((c["hi"] + 1) // 2, c["hi"])
    c["past_lo"] = c["past_hi"] if rng.random() < 0.3 else c["past_hi"] // rng.randint(1, 6)
    return c


# ---- what the program holds before the call -----------------------------------------------------------------

def _spread(lo, hi, n, salt):
    """n whole numbers of lo..hi, both ends among them, in an irregular order that the case alone decides."""
    if n == 1 or lo == hi:
        return [hi] * n
    out = [hi, lo] + [lo + (7919 * b * b + (104729 + salt) * b) % (hi - lo + 1) for b in range(2, n)]
    random.Random(n + salt).shuffle(out)
    return out


def _tokens(case):
    return _spread(case["lo"], case["hi"], case["batch"], 1)


def _past(case):
    return _spread(case["past_lo"], case["past_hi"], case["batch"], 2)


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    """Tensors of the call.  Page tables name pages in random order; entries that no row needs are -1."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    nb, hq, hkv, d, page = case["batch"], case["hq"], case["hkv"], case["d"], case["page"]
    nq, past = _tokens(case), _past(case)
    lens = [a + b for a, b in zip(past, nq)]
    need = [-(-n // page) for n in lens]
    first = -(-case.get("prefix", 0) // page)
    n_pages = first + sum(need)
    order = torch.randperm(n_pages, generator=g, device="cuda").int().tolist()
    table, at = [], first
    for m in need:
        table.append(order[at:at + m] + [-1] * (max(need) - m))
        at += m
    T = sum(nq)
    s = dict(case=case, nq=nq, past=past, lens=lens, offs=_offsets(nq), order=order, rows_of=table, n_pages=n_pages, max_pages=max(need),
             table=_ints(table), q_offsets=_ints(_offsets(nq)), first=first)
    s["k_pages"] = torch.randn((n_pages, hkv, page, d), generator=g, device="cuda", dtype=dt)
    s["v_pages"] = torch.randn((n_pages, hkv, page, d), generator=g, device="cuda", dtype=dt)
    if case["op"] == "append":
        s["cache_lens"] = _ints(past)
        # a projection's output: query, key and value heads of a token side by side
        s["qkv"] = torch.randn((T, (hq + 2 * hkv) * d), generator=g, device="cuda", dtype=dt)
        s["q"], s["k"], s["v"] = (x.unflatten(1, (-1, d)) for x in s["qkv"].split([hq * d, hkv * d, hkv * d], 1))
        # texts that began somewhere behind their caches' first rows: rotation by the place in the text
        shift = torch.randint(0, 4000, (nb,), generator=g, device="cuda").tolist()
        s["positions"] = _ints([shift[b] + past[b] + t for b in range(nb) for t in range(nq[b])])
        if case["rot"]:
            n_pos, half = 4000 + max(lens), case["rot"] // 2
            angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * 500000.0 ** (
                -torch.arange(half, dtype=torch.float64, device="cuda") / half)
            s["rot_table"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        else:
            s["rot_table"] = None
        s["new_lens"] = torch.zeros_like(s["cache_lens"])
        s["q_out"] = torch.empty((T, hq, d), dtype=dt, device="cuda")
        return s
    s["cache_lens"] = _ints(lens)
    # heavy hitters and an attention sink among the keys, queries as far from normal as those of a trained model
    k = s["k_pages"].view(-1, d)
    heavy = torch.randint(0, k.shape[0], (max(1, k.shape[0] // 1000),), generator=g, device="cuda").unique()
    k[heavy] = k[heavy] * 4
    s["k_pages"][order[0], :, 0] *= 1.5
    s["q"] = (torch.randn((T, hq, d), generator=g, device="cuda") * 2.3).to(dt)
    s["out"] = torch.empty((T, hq, d), dtype=dt, device="cuda")
    s["lse"] = torch.empty((T, hq), dtype=torch.float32, device="cuda")
    if first:
        s["shared_table"] = _ints(order[:first])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2507_19906_amd import binding as cd
        p = cd.make_paged_params(dtype=case["dtype"], batch=case["batch"], n_q_heads=case["hq"], n_kv_heads=case["hkv"],
                                 head_dim=case["d"], page_size=case["page"], n_pages=s["n_pages"], max_pages=s["max_pages"],
                                 window=case.get("window", 0), sinks=case.get("sinks", 0), rot_dim=case.get("rot", 0),
                                 rot_pairs=case.get("pairs", "halves"))
        s["cache"] = cd.PagedCache(p, s["k_pages"], s["v_pages"], s["table"], s["cache_lens"])
        s["most"] = dict(max_q_len=max(s["nq"]), max_cache_len=max(s["lens"]))
        if case["op"] == "attend":
            s["cache"].reserve(sum(s["nq"]), max(s["nq"]), max(s["lens"]))
        elif case["op"] == "shared":
            s["cache"].reserve(sum(s["nq"]), max(s["nq"]), max(s["lens"]), case["prefix"])
    return s


# ---- the call ---------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    one = case["lo"] == case["hi"] == 1
    if case["op"] == "append":
        if own:
            s["cache"].append(s["k"], s["v"], q=s["q"], q_out=s["q_out"], new_offsets=None if one else s["q_offsets"],
                              max_new=max(s["nq"]), positions=s["positions"], rot_table=s["rot_table"], new_lens=s["new_lens"])
        else:
            _append_plain(s)
        return dict(k_pages=s["k_pages"], v_pages=s["v_pages"], q=s["q_out"], new_lens=s["new_lens"])
    if not own:
        return _attend_plain(s)
    offs = None if one else s["q_offsets"]
    if case["op"] == "attend":
        s["cache"].attend(s["q"], s["out"], s["lse"], q_offsets=offs, **s["most"])
    else:
        s["cache"].attend_shared(s["q"], s["out"], s["lse"], s["shared_table"], case["prefix"], q_offsets=offs, **s["most"])
    return dict(out=s["out"], lse=s["lse"])


def _turned(x, table, positions, rot, pairs):
    """x [T][heads][d] in 32 bits, the first `rot` elements of every head turned by the angles of their positions."""
    x = x.float()
    if not rot:
        return x
    cs = table[positions.long()][:, None, :]
    c, s = cs[..., :rot // 2], cs[..., rot // 2:]
    if pairs == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([r, x[..., rot:]], -1)


def _append_plain(s):
    case = s["case"]
    dt, page = s["k_pages"].dtype, case["page"]
    n = s["q_offsets"].diff()
    seq = torch.repeat_interleave(torch.arange(case["batch"], device="cuda"), n.long(), output_size=s["qkv"].shape[0])
    row = s["cache_lens"][seq] + torch.arange(s["qkv"].shape[0], device="cuda") - s["q_offsets"][seq]
    at, inside = s["table"][seq, row // page].long(), (row % page).long()
    turn = (s["rot_table"], s["positions"], case["rot"], case["pairs"])
    s["k_pages"][at, :, inside] = _turned(s["k"], *turn).to(dt)
    s["v_pages"][at, :, inside] = s["v"]
    s["q_out"].copy_(_turned(s["q"], *turn).to(dt))
    s["new_lens"].copy_(s["cache_lens"] + n)


def _partial(q, k, v, scale, seen):
    """Attention of q [n][hq][d] over k, v [hkv][rows][d] in 32 bits, a block of queries at a time: unnormalised outputs,
    largest logits and sums of exponentials.  `seen(lo, hi)`: which rows the queries lo..hi-1 see, or None for all."""
    n, hq, d = q.shape
    hkv, rows = k.shape[:2]
    o = torch.zeros((n, hq, d), device="cuda")
    m = torch.full((n, hq), -math.inf, device="cuda")
    l = torch.zeros((n, hq), device="cuda")
    if rows == 0:
        return o, m, l
    kt = k.transpose(1, 2).contiguous()
    step = max(1, min(n, (1 << 28) // (hq * rows)))
    for lo in range(0, n, step):
        hi = min(n, lo + step)
        z = q[lo:hi].float().view(hi - lo, hkv, hq // hkv, d).permute(1, 2, 0, 3).reshape(hkv, -1, d) @ kt
        z = z.view(hkv, hq // hkv, hi - lo, rows) * scale
        see = seen(lo, hi)
        if see is not None:
            z = z.masked_fill(~see, -math.inf)
        top = z.amax(-1, keepdim=True)
        e = (z - top.clamp(min=-1e30)).exp()
        l[lo:hi] = e.sum(-1).permute(2, 0, 1).reshape(hi - lo, hq)
        m[lo:hi] = top[..., 0].permute(2, 0, 1).reshape(hi - lo, hq)
        w = e.view(hkv, -1, rows) @ v
        o[lo:hi] = w.view(hkv, hq // hkv, hi - lo, d).permute(2, 0, 1, 3).reshape(hi - lo, hq, d)
    return o, m, l


def _rows(pages, entries, n):
    """The first n rows of the pages that `entries` names, [hkv][n][d] in 32 bits."""
    page = pages.shape[2]
    x = pages[entries[:-(-n // page)].long()].transpose(0, 1).flatten(1, 2)
    return x[:, :n].float()


def _attend_plain(s):
    case = s["case"]
    scale = 1.0 / math.sqrt(case["d"])
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    if s["first"]:
        before = _partial(s["q"], _rows(s["k_pages"], s["shared_table"], case["prefix"]),
                          _rows(s["v_pages"], s["shared_table"], case["prefix"]), scale, lambda lo, hi: None)
    for b in range(case["batch"]):
        lo_q, hi_q, n, past = s["offs"][b], s["offs"][b + 1], s["lens"][b], s["past"][b]
        j = torch.arange(n, device="cuda")[None]

        def seen(lo, hi):
            i = past + torch.arange(lo, hi, device="cuda")[:, None]
            see = j <= i
            return see & ((j > i - window) | (j < sinks)) if window else see
        o, m, l = _partial(s["q"][lo_q:hi_q], _rows(s["k_pages"], s["table"][b], n), _rows(s["v_pages"], s["table"][b], n), scale, seen)
        if s["first"]:
            o2, m2, l2 = (x[lo_q:hi_q] for x in before)
            top = torch.maximum(m, m2)
            f, f2 = (m - top).exp(), (m2 - top).exp()
            o, l, m = o * f[..., None] + o2 * f2[..., None], l * f + l2 * f2, top
        s["out"][lo_q:hi_q] = torch.where(l[..., None] > 0, o / l[..., None], 0.0).to(s["out"].dtype)
        s["lse"][lo_q:hi_q] = m + l.log()
    return dict(out=s["out"], lse=s["lse"])


# ---- what a pass cannot do without -----------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    nq, past = _tokens(case), _past(case)
    T = sum(nq)
    if case["op"] == "append":
        # every head read and written once, the angles of each position, lengths and offsets
        b = 2 * T * (hq + 2 * hkv) * d * e + T * (case["rot"] * 4 + 4) + 12 * case["batch"]
        return dict(bytes=b, flops=3 * T * (hq + hkv) * case["rot"])
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    rows = pairs = 0
    for n, p in zip(nq, past):
        if not window:
            rows += p + n
            pairs += n * p + n * (n + 1) // 2
            continue
        lo = max(0, p + 1 - window)                                     # first row the first query's window holds
        rows += min(sinks, lo) + p + n - lo
        for i in range(p, p + n):
            pairs += min(i + 1, window) + min(sinks, max(0, i + 1 - window))
    rows += case.get("prefix", 0)
    pairs += T * case.get("prefix", 0)
    return dict(bytes=2 * rows * hkv * d * e + 2 * T * hq * d * e + 4 * T * hq, flops=4 * pairs * hq * d)


# ---- the same in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    """The definitions, head by head and row by row of the page tables, in 64 bits."""
    s = _inputs(case, seed)
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    G = hq // hkv
    if case["op"] == "append":
        out = dict(k_pages=s["k_pages"].double(), v_pages=s["v_pages"].double(), q=torch.empty((len(s["positions"]), hq, d),
                   dtype=torch.float64, device="cuda"), new_lens=s["cache_lens"].clone())
        for b in range(case["batch"]):
            t0, t1 = s["offs"][b], s["offs"][b + 1]
            out["new_lens"][b] += t1 - t0
            rows = torch.arange(s["past"][b], s["lens"][b], device="cuda")
            where = (s["table"][b].long()[torch.div(rows, page, rounding_mode="floor")], rows.remainder(page))
            for name in ("q", "k"):
                x = s[name][t0:t1].double().clone()
                half = case["rot"] // 2
                for i in range(half):
                    a, c = (i, i + half) if case["pairs"] == "halves" else (2 * i, 2 * i + 1)
                    w = torch.complex(*(s["rot_table"][s["positions"][t0:t1].long(), i + off].double() for off in (0, half)))
                    z = torch.complex(x[:, :, a].clone(), x[:, :, c].clone()) * w[:, None]
                    x[:, :, a], x[:, :, c] = z.real, z.imag
                if name == "q":
                    out["q"][t0:t1] = x
                else:
                    out["k_pages"].permute(0, 2, 1, 3)[where] = x
            out["v_pages"].permute(0, 2, 1, 3)[where] = s["v"][t0:t1].double()
        return out
    window, sinks, prefix = case.get("window", 0), case.get("sinks", 0), case.get("prefix", 0)
    out = torch.empty((s["offs"][-1], hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((s["offs"][-1], hq), dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        t0, t1, n, past = s["offs"][b], s["offs"][b + 1], s["lens"][b], s["past"][b]
        for g in range(hkv):
            def column(pages):
                ahead = [pages[x, g] for x in s["order"][:s["first"]]]
                ahead = torch.cat(ahead)[:prefix] if ahead else pages[0, g, :0]
                return torch.cat([ahead, torch.cat([pages[x, g] for x in s["rows_of"][b] if x >= 0])[:n]]).double()
            k, v = column(s["k_pages"]), column(s["v_pages"])
            place = torch.arange(-prefix, n, device="cuda")
            for lo in range(t0, t1, 4096):
                hi = min(t1, lo + 4096)
                at = past + torch.arange(lo - t0, hi - t0, device="cuda")
                hidden = place[None, :] > at[:, None]
                if window:
                    hidden |= (place[None, :] <= at[:, None] - window) & (place[None, :] >= sinks)
                for h in range(g * G, (g + 1) * G):
                    z = (s["q"][lo:hi, h].double() @ k.t()) / math.sqrt(d)
                    z.masked_fill_(hidden, -math.inf)
                    lse[lo:hi, h] = torch.logsumexp(z, 1)
                    out[lo:hi, h] = torch.exp(z - lse[lo:hi, h, None]) @ v
    return dict(out=out, lse=lse)
