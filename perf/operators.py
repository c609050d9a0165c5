"""What the operators on a paged cache are timed and checked on, as cases.

Three operators share one cache of 16-key pages that many sequences live in:

* `rope`: the newest rows of several sequences get their query and key heads normalised (where gains are given) and
  rotated, and their keys and values are rounded into the cache's pages;
* `attention`: those rows attend to their sequences' pages, with a cap on the scores, a bias by distance, a window, a
  prefix that every row sees, documents that do not see each other;
* `copy`: pages move within a cache or from one to another, keys and values of all layers (a sequence is forked, a
  cache compacted).

With `own` false, `run` computes them from elementary torch operations in 32 bits; with `own` true it makes the calls
that a program makes of the library.  A cache is bfloat16, [layer][keys, values][page][kv head][16 x head_dim], the
values of a page transposed ([head_dim][16]).
"""
import math
import random

import torch

own = False

DEV = "cuda"
PAGE = 16


def listed():
    return [
        # one new token of one sequence at the grouped-query 8B shape: the launch is what counts
        dict(name="rope_8b_row1", kind="rope", q=32, kv=8, hd=128, fp32=False, norm=True, inter=False, rot=128, seqs=1,
             lo=1, hi=1, past=700, mix=1),
        # verification rows of 48 sequences at the 7B shape, float32 rows as the library's own passes have them, half of
        # each head rotated in neighbouring pairs
        dict(name="rope_7b_verify48", kind="rope", q=32, kv=32, hd=128, fp32=True, norm=False, inter=True, rot=64, seqs=48,
             lo=1, hi=8, past=1500, mix=2),
        # three prompts side by side, 8192 rows or so, heads normalised
        dict(name="rope_8b_prompts", kind="rope", q=32, kv=8, hd=128, fp32=False, norm=True, inter=False, rot=128, seqs=3,
             lo=1800, hi=3600, past=37, mix=3),
        # one new token behind a 7B prompt, float32 rows: the smallest attention
        dict(name="attention_7b_row1", kind="attention", q=32, kv=32, hd=128, fp32=True, seqs=1, lo=1, hi=1, past=520,
             spread=False, cap=0.0, bias=False, window=0, prefix=False, docs=0, mix=4),
        # a serving step: 64 sequences of very different lengths, one token each, scores capped
        dict(name="attention_8b_decode64", kind="attention", q=32, kv=8, hd=128, fp32=False, seqs=64, lo=1, hi=1, past=8000,
             spread=True, cap=50.0, bias=False, window=0, prefix=False, docs=0, mix=5),
        # a round's six rows behind a book, bias by distance: the cache is what is read
        dict(name="attention_8b_verify_131k", kind="attention", q=32, kv=8, hd=128, fp32=True, seqs=1, lo=6, hi=6, past=131000,
             spread=False, cap=0.0, bias=True, window=0, prefix=False, docs=0, mix=6),
        # the second half of a 4096-token prompt at the 7B shape, plain causal: the matrix products are what counts
        dict(name="attention_7b_prompt_4096", kind="attention", q=32, kv=32, hd=128, fp32=False, seqs=1, lo=2048, hi=2048,
             past=2048, spread=False, cap=0.0, bias=False, window=0, prefix=False, docs=0, mix=7),
        # documents packed into one row of 8000 tokens, each seeing 1024 keys of its own at most
        dict(name="attention_8b_packed_8000", kind="attention", q=32, kv=8, hd=128, fp32=False, seqs=1, lo=8000, hi=8000,
             past=0, spread=False, cap=0.0, bias=False, window=1024, prefix=False, docs=900, mix=8),
        # five prompts with a prefix that is seen from both sides, capped scores, float32 rows, small heads
        dict(name="attention_prefix5", kind="attention", q=16, kv=4, hd=64, fp32=True, seqs=5, lo=150, hi=1300, past=90,
             spread=False, cap=30.0, bias=False, window=0, prefix=True, docs=0, mix=9),
        # a chat turn is forked: five pages of four layers at the 7B shape
        dict(name="copy_7b_fork", kind="copy", kv=32, hd=128, fp32=False, layers=4, pages=5, inside=False, mix=10),
        # a long context is forked into another cache at the 8B shape
        dict(name="copy_8b_fork_11k", kind="copy", kv=8, hd=128, fp32=False, layers=8, pages=700, inside=False, mix=11),
        # a cache is compacted at the 13B shape: pages above the live count move into holes below it
        dict(name="copy_13b_compact", kind="copy", kv=40, hd=128, fp32=False, layers=4, pages=333, inside=True, mix=12),
    ]


def draw(rng):
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rope", "attention", "attention", "attention", "copy"])
    mix = rng.randrange(1 << 30)
    hd = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8, 16, 32, 40])
    if kind == "copy":
        layers = rng.randint(1, 8)
        kv = rng.choice([4, 8, 32, 40])
        fp32 = rng.random() < 0.25
        top = max(2, int(400e6 / (layers * 2 * kv * PAGE * hd * (4 if fp32 else 2))))
        return dict(kind=kind, kv=kv, hd=hd, fp32=fp32, layers=layers, pages=logu(1, min(top, 1500)), inside=rng.random() < 0.5,
                    mix=mix)
    q = kv * (rng.choice([1, 2, 4, 5, 8, 16]) if kv <= 4 else rng.choice([1, 2, 4]) if kv <= 16 else 1)
    fp32 = rng.random() < 0.4
    c = dict(kind=kind, q=q, kv=kv, hd=hd, fp32=fp32)
    if kind == "rope":
        seqs = logu(1, 96)
        if rng.random() < 0.5:
            lo, hi = 1, rng.randint(1, 8)
        else:
            hi = logu(9, max(10, 8192 // seqs))
            lo = rng.randint(1, hi)
        c.update(norm=rng.random() < 0.5, inter=rng.random() < 0.4, rot=rng.choice([hd, hd, hd // 2, hd // 4, 24]), seqs=seqs,
                 lo=lo, hi=hi, past=rng.choice([0, logu(1, 4000)]), mix=mix)
        return c
    if rng.random() < 0.5:   # few rows a sequence
        seqs = logu(1, 64)
        hi = rng.choice([1, 1, rng.randint(1, 8)])
        lo = rng.randint(1, hi)
        top = int(min(131000, 1.0e9 / (seqs * kv * hd * 4)))
        past = logu(3, max(8, top))
    else:                    # prompts
        seqs = rng.randint(1, 6)
        hi = logu(16, 6000 // seqs)
        lo = rng.randint(1, hi)
        past = rng.choice([0, 0, logu(1, 3000)])
    c.update(seqs=seqs, lo=lo, hi=hi, past=past, spread=rng.random() < 0.5, cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
             bias=rng.random() < 0.25, window=rng.choice([0, 0, 0, logu(1, 4000)]), prefix=rng.random() < 0.25,
             docs=rng.choice([0, 0, 0, logu(4, 1500)]), mix=mix)
    return c


# ---------------------------------------------------------------- what a case fixes
def _batch(case):
    """New rows, cached keys in all and prefix of each sequence, and the first position of each document of it."""
    r = random.Random(case["mix"])
    rows, lens, prefix, docs = [], [], [], []
    for _ in range(case["seqs"]):
        n = r.randint(case["lo"], case["hi"])
        past = case["past"]
        if case.get("spread"):
            past = int(past * r.random())
        rows.append(n)
        lens.append(past + n)
        prefix.append(r.randint(0, max(1, lens[-1] // 2)) if case.get("prefix") else 0)
        starts = [0]
        while case.get("docs") and starts[-1] < lens[-1]:
            starts.append(starts[-1] + r.randint(1, 2 * case["docs"]))
        docs.append(starts)
    return rows, lens, prefix, docs


def _doc_start(starts, pos):
    """Start of the document that holds each of the ascending positions."""
    t = torch.tensor(starts, dtype=torch.int64)
    return t[torch.searchsorted(t, pos, right=True) - 1]


def _row_ranges(case):
    """Per sequence: position and visible key ranges [a0, a1) and [b0, b1) of its rows (int64, on the CPU)."""
    rows, lens, prefix, docs = _batch(case)
    for n, ln, pre, st in zip(rows, lens, prefix, docs):
        pos = torch.arange(ln - n, ln)
        d = _doc_start(st, pos)
        a1 = torch.full_like(pos, min(pre, ln))
        b0 = torch.maximum(d, pos + 1 - case["window"]) if case["window"] else d
        yield pos, d, a1, b0, pos + 1


def work(case):
    es = 4 if case["fp32"] else 2
    if case["kind"] == "copy":
        n = case["pages"] * case["layers"] * 2 * case["kv"] * PAGE * case["hd"] * es
        return {"bytes": 2 * n, "flops": 0}
    hd, hq, hkv = case["hd"], case["q"], case["kv"]
    rows = sum(_batch(case)[0])
    if case["kind"] == "rope":
        return {"bytes": rows * ((2 * hq + 2 * hkv) * hd * es + 2 * hkv * hd * 2 + case["rot"] * 4),
                "flops": rows * (hq + hkv) * (3 * case["rot"] + (4 * hd if case["norm"] else 0))}
    pairs = keys = 0
    for pos, a0, a1, b0, b1 in _row_ranges(case):
        seen = (a1 - a0).clamp(min=0) + (b1 - torch.maximum(b0, a1)).clamp(min=0)
        pairs += int(seen.sum())
        hit = torch.zeros(int(b1[-1]) + 1, dtype=torch.int32)   # keys that some row sees
        for lo, hi in ((a0, a1), (b0, b1)):
            ok = hi > lo
            hit.index_add_(0, lo[ok], torch.ones(int(ok.sum()), dtype=torch.int32))
            hit.index_add_(0, hi[ok], -torch.ones(int(ok.sum()), dtype=torch.int32))
        keys += int((hit.cumsum(0) > 0).sum())
    return {"bytes": 2 * rows * hq * hd * es + keys * 2 * hkv * hd * 2, "flops": 4 * pairs * hq * hd}


# ---------------------------------------------------------------- seeded inputs
def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + what * 7919 + 12345) % (1 << 62))
    return g


def _normal(seed, what, shape, std=1.0, fp32=True):
    x = torch.randn(shape, generator=_gen(seed, what), device=DEV, dtype=torch.float32)
    x *= std
    return x if fp32 else x.to(torch.bfloat16)


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32).to(DEV)


def _rope_tables(rot, n_pos, base=500000.0):
    """Angles pos base^(-2 i / rot), every frequency an eighth of it past 8192 positions a turn (a stretched context)."""
    f = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    f = torch.where(2 * math.pi / f > 8192, f / 8, f).to(DEV)
    a = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * f[None, :]
    return torch.cos(a).float(), torch.sin(a).float()


def _inputs(case, seed):
    s = {}
    hd, hkv = case["hd"], case["kv"]
    r = random.Random(case["mix"] + 1)
    if case["kind"] == "copy":
        n = case["pages"]
        total = 2 * n + 3
        dt = torch.float32 if case["fp32"] else torch.bfloat16
        shape = (case["layers"], 2, total, hkv, PAGE, hd)
        s["src"] = _normal(seed, 1, shape, fp32=False).to(dt)
        if case["inside"]:
            s["dst"] = s["src"]
            s["src_pages"] = sorted(r.sample(range(n + 3, total), n), reverse=True)
            s["dst_pages"] = sorted(r.sample(range(0, n + 3), n))
        else:
            s["dst"] = _normal(seed, 2, shape, fp32=False).to(dt)
            s["src_pages"] = r.sample(range(total), n)
            s["dst_pages"] = r.sample(range(total), n)
        return s
    rows, lens, prefix, docs = _batch(case)
    n_rows = sum(rows)
    per = [(ln + PAGE - 1) // PAGE for ln in lens]
    n_pages = sum(per) + 3
    order = torch.randperm(n_pages, generator=_gen(seed, 3), device=DEV).to(torch.int32)
    table = torch.zeros((len(rows), max(per)), dtype=torch.int32, device=DEV)
    at = 0
    for b, p in enumerate(per):
        table[b, :p] = order[at:at + p]
        at += p
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    s.update(rows=rows, lens=lens, n_rows=n_rows, n_pages=n_pages, table=table, row_start=_i32(starts), kv_len=_i32(lens))
    s["pool"] = _normal(seed, 4, (1, 2, n_pages, hkv, PAGE, hd), fp32=False)
    if case["kind"] == "rope":
        s["qkv"] = _normal(seed, 5, (n_rows, (case["q"] + 2 * hkv) * hd), 1.3, case["fp32"])
        s["cos"], s["sin"] = _rope_tables(case["rot"], max(lens))
        s["q_gain"] = 1.0 + _normal(seed, 6, (hd,), 0.1) if case["norm"] else None
        s["k_gain"] = 1.0 + _normal(seed, 7, (hd,), 0.1) if case["norm"] else None
        return s
    # queries a little larger than keys: some rows look at few keys, most at many
    s["q"] = _normal(seed, 8, (n_rows, case["q"] * hd), 1.7, case["fp32"])
    s["slopes"] = None
    if case["bias"]:
        s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, case["q"] + 1, dtype=torch.float64) / case["q"])).float().to(DEV)
    s["prefix_len"] = _i32(prefix) if case["prefix"] else None
    s["doc_start"] = None
    if case["docs"]:
        s["doc_start"] = _i32(torch.cat([_doc_start(st, torch.arange(ln - n, ln)) for n, ln, st in zip(rows, lens, docs)]))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own and case["kind"] != "copy":
        import paper_2604_12247_amd as sb
        s["kv"] = sb.Paged(s["pool"], s["table"], s["row_start"], s["kv_len"], n_rows=s["n_rows"], max_len=max(s["lens"]))
        if case["kind"] == "attention":
            s["scratch"] = sb.paged_attention_scratch(s["kv"], case["q"])
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    f = {"rope": (_rope_plain, _rope_own), "attention": (_attention_plain, _attention_own), "copy": (_copy_plain, _copy_own)}
    return f[case["kind"]][1 if own else 0](case, state)


def _rope_own(case, s):
    import paper_2604_12247_amd as sb
    q = sb.op_rope_append(s["kv"], s["qkv"], case["q"], s["cos"], s["sin"], interleaved=case["inter"], q_gain=s["q_gain"],
                          k_gain=s["k_gain"], eps=1e-6)
    return q, s["pool"]


def _attention_own(case, s):
    import paper_2604_12247_amd as sb
    return sb.op_paged_attention(s["kv"], s["q"], case["q"], softcap=case["cap"], slopes=s["slopes"], window=case["window"],
                                 prefix_len=s["prefix_len"], doc_start=s["doc_start"], scratch=s["scratch"])


def _copy_own(case, s):
    import paper_2604_12247_amd as sb
    sb.op_copy_pages(s["dst"], s["src"], s["dst_pages"], s["src_pages"])
    return s["dst"]


def _rotate(x, c, n, rot, inter):
    """x [rows, heads, hd] float32 rotated by c, n [rows, rot / 2]."""
    c, n = c[:, None, :], n[:, None, :]
    y = x.clone()
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * n, b * c + a * n
    else:
        h = rot // 2
        a, b = x[..., :h], x[..., h:rot]
        y[..., :h], y[..., h:rot] = a * c - b * n, b * c + a * n
    return y


def _rope_plain(case, s):
    hq, hkv, hd, rot = case["q"], case["kv"], case["hd"], case["rot"]
    M = s["n_rows"]
    row = torch.arange(M, device=DEV)
    seq = torch.searchsorted(s["row_start"][1:].contiguous(), row.to(torch.int32), right=True)
    pos = (s["kv_len"][seq] - s["row_start"][seq + 1] + row).long()
    x = s["qkv"].float().view(M, hq + 2 * hkv, hd)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    if case["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + 1e-6) * s["q_gain"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + 1e-6) * s["k_gain"]
    c, n = s["cos"][pos], s["sin"][pos]
    q, k = _rotate(q, c, n, rot, case["inter"]), _rotate(k, c, n, rot, case["inter"])
    page = s["table"][seq, pos // PAGE].long()
    slot = pos % PAGE
    s["pool"][0, 0][page, :, slot] = k.to(torch.bfloat16)
    s["pool"][0, 1].view(s["n_pages"], hkv, hd, PAGE)[page, :, :, slot] = v.to(torch.bfloat16)
    return q.reshape(M, hq * hd).to(s["qkv"].dtype), s["pool"]


def _attention_plain(case, s):
    hq, hkv, hd = case["q"], case["kv"], case["hd"]
    g = hq // hkv
    out = torch.empty_like(s["q"])
    at = 0
    for b, (n, ln) in enumerate(zip(s["rows"], s["lens"])):
        pages = s["table"][b, :(ln + PAGE - 1) // PAGE].long()
        k = s["pool"][0, 0, pages].float().permute(1, 0, 2, 3).reshape(hkv, -1, hd)[:, :ln]
        v = s["pool"][0, 1].view(s["n_pages"], hkv, hd, PAGE)[pages].float().permute(1, 0, 3, 2).reshape(hkv, -1, hd)[:, :ln]
        kt = k.transpose(1, 2).contiguous()
        key = torch.arange(ln, device=DEV)
        step = max(1, int(2.0e8 / (hq * ln)))
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            q = s["q"][at + r0:at + r1].float().view(r1 - r0, hkv, g, hd).permute(1, 2, 0, 3).reshape(hkv, g * (r1 - r0), hd)
            w = torch.matmul(q, kt).view(hkv, g, r1 - r0, ln) * (1.0 / math.sqrt(hd))
            if case["cap"]:
                w = case["cap"] * torch.tanh(w / case["cap"])
            p = torch.arange(ln - n + r0, ln - n + r1, device=DEV)[:, None]
            if s["slopes"] is not None:
                w = w - s["slopes"].view(hkv, g, 1, 1) * (p - key).abs().float()
            see = key <= p
            if case["window"]:
                see = see & (key > p - case["window"])
            if s["prefix_len"] is not None:
                see = see | (key < s["prefix_len"][b])
            if s["doc_start"] is not None:
                see = see & (key >= s["doc_start"][at + r0:at + r1, None])
            w = torch.where(see, w, -math.inf)
            m = w.amax(-1, keepdim=True)
            w = torch.exp(w - torch.where(m == -math.inf, 0.0, m))
            t = w.sum(-1, keepdim=True)
            o = torch.matmul(w.view(hkv, -1, ln), v).view(hkv, g, r1 - r0, hd) / torch.where(t == 0, 1.0, t)
            out[at + r0:at + r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, hq * hd).to(out.dtype)
        at += n
    return out


def _copy_plain(case, s):
    i, j = torch.tensor(s["dst_pages"], device=DEV), torch.tensor(s["src_pages"], device=DEV)
    s["dst"][:, :, i] = s["src"][:, :, j]
    return s["dst"]


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    if case["kind"] == "copy":   # nothing is computed
        return None
    s = _inputs(case, seed)
    hq, hkv, hd = case["q"], case["kv"], case["hd"]
    return _exact_rope(case, s, hq, hkv, hd) if case["kind"] == "rope" else _exact_attention(case, s, hq, hkv, hd)


def _exact_rope(case, s, hq, hkv, hd):
    rot, half = case["rot"], case["rot"] // 2
    x = s["qkv"].double()
    q = torch.empty((s["n_rows"], hq, hd), dtype=torch.float64, device=DEV)
    pool = s["pool"].double()
    if case["inter"]:
        first, second = torch.arange(0, rot, 2, device=DEV), torch.arange(1, rot, 2, device=DEV)
    else:
        first, second = torch.arange(0, half, device=DEV), torch.arange(half, rot, device=DEV)
    at = 0
    for b, (n, ln) in enumerate(zip(s["rows"], s["lens"])):
        pos = torch.arange(ln - n, ln, device=DEV)
        turn = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())
        heads = x[at:at + n].view(n, hq + 2 * hkv, hd)
        for h in range(hq + hkv):   # a head at a time: norm, then the pairs as complex numbers
            u = heads[:, h]
            gain = s["q_gain"] if h < hq else s["k_gain"]
            if gain is not None:
                u = u / torch.sqrt(torch.sum(u ** 2, 1, keepdim=True) / hd + 1e-6) * gain.double()
            z = torch.complex(u[:, first].contiguous(), u[:, second].contiguous()) * turn
            u = u.clone()
            u[:, first], u[:, second] = z.real, z.imag
            if h < hq:
                q[at:at + n, h] = u
            else:
                pool[0, 0, s["table"][b, pos // PAGE].long(), h - hq, pos % PAGE] = u
        tail = pool[0, 1].view(-1, hkv, hd, PAGE)
        tail[s["table"][b, pos // PAGE].long(), :, :, pos % PAGE] = heads[:, hq + hkv:]
        at += n
    return q.view(s["n_rows"], hq * hd), pool


def _exact_attention(case, s, hq, hkv, hd):
    if work(case)["flops"] > 1.5e12:
        return None
    g = hq // hkv
    out = torch.zeros((s["n_rows"], hq, hd), dtype=torch.float64, device=DEV)
    at = 0
    for b, (pos, a0, a1, b0, b1) in enumerate(_row_ranges(case)):
        n, ln = len(pos), s["lens"][b]
        pages = s["table"][b].long()[torch.arange(ln, device=DEV) // PAGE]
        slot = torch.arange(ln, device=DEV) % PAGE
        a0, a1, b0, b1, pos = (t.to(DEV)[:, None] for t in (a0, a1, b0, b1, pos))
        key = torch.arange(ln, device=DEV)[None, :]
        for h in range(hkv):
            k = s["pool"][0, 0, :, h][pages, slot].double()
            v = s["pool"][0, 1].view(-1, hkv, hd, PAGE)[:, h][pages, :, slot].double()
            for r in range(0, n, 1024):
                e = slice(r, min(n, r + 1024))
                hidden = ~(((key >= a0[e]) & (key < a1[e])) | ((key >= b0[e]) & (key < b1[e])))
                for i in range(h * g, (h + 1) * g):
                    z = (s["q"][at:at + n].view(n, hq, hd)[e, i].double() @ k.t()) / math.sqrt(hd)
                    if case["cap"]:
                        z = torch.tanh(z / case["cap"]) * case["cap"]
                    if case["bias"]:
                        z = z - (key - pos[e]).abs() * s["slopes"][i].double()
                    z = z.masked_fill(hidden, -math.inf)
                    z = torch.softmax(z, 1).masked_fill(hidden.all(1, keepdim=True), 0.0)
                    out[at + r:at + r + z.shape[0], i] = z @ v
        at += n
    return out.view(s["n_rows"], hq * hd)
