"""Operators on a paged cache against their definitions in 64 bits: rotary append, attention by a rule, page copies,
forked sessions, and all of them together as a serving loop uses them."""
import math

import numpy as np
import pytest
import torch

import paper_2604_12247_amd as sb
import sb_inputs as si
from helpers import gpu_model, gpu_params

pytestmark = pytest.mark.gpu

DEV = "cuda"
PAGE = sb.SB_KV_BLOCK
U = 2.0 ** -24        # a rounding to float is off by at most this, relatively
UB = 2.0 ** -8        # to bfloat16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(seed, *shape):
    return torch.randn(shape, generator=gen(seed), device=DEV)


class Case:
    """A ragged batch on a shuffled pool: rows and cached keys of each sequence."""

    def __init__(self, rows, lens, hq, hkv, hd, dtype, seed=0, layers=1, spare=3, table_ld=None, lead=0, tail=0, layer=0, junk=None):
        self.rows, self.lens, self.hq, self.hkv, self.hd, self.dtype, self.layer = rows, lens, hq, hkv, hd, dtype, layer
        per = [(n + PAGE - 1) // PAGE for n in lens]
        self.n_pages = sum(per) + spare
        order = torch.randperm(self.n_pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        ld = max(per + [1]) if table_ld is None else table_ld
        table = torch.full((len(rows), ld), 0x7fff0000, dtype=torch.int32)   # (what lies behind a sequence's pages is not read)
        at = 0
        for b, p in enumerate(per):
            table[b, :p] = order[at:at + p]
            at += p
        self.table_cpu = table
        self.table = table.to(DEV)
        starts = [lead]
        for n in rows:
            starts.append(starts[-1] + n)
        self.starts, self.n_rows = starts, starts[-1] + tail
        self.row_start = torch.tensor(starts, dtype=torch.int32, device=DEV)
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.pool = randn(seed + 1, layers, 2, self.n_pages, hkv, PAGE, hd).to(torch.bfloat16)
        if junk is not None:   # everywhere but in the sequences' own keys
            keep = self.used_mask()
            self.pool[:, 0][:, ~keep[0]] = junk
            self.pool[:, 1][:, ~keep[1]] = junk
        self.kv = sb.Paged(self.pool, self.table, self.row_start, self.kv_len, n_rows=self.n_rows)

    def used_mask(self):
        """[2][n_pages, hkv, PAGE, hd] truth values: elements of the pool that are keys / values of a sequence."""
        k = torch.zeros((self.n_pages, self.hkv, PAGE, self.hd), dtype=torch.bool, device=DEV)
        v = torch.zeros((self.n_pages, self.hkv, self.hd, PAGE), dtype=torch.bool, device=DEV)
        for b, n in enumerate(self.lens):
            pos = torch.arange(n)
            pg, sl = self.table_cpu[b, pos // PAGE].long().to(DEV), (pos % PAGE).to(DEV)
            k[pg, :, sl] = True
            v[pg, :, :, sl] = True
        return k, v.view(self.n_pages, self.hkv, PAGE, self.hd)

    def cached(self, b, pool=None):
        """Keys and values of sequence b in 64 bits, [len, hkv, hd]."""
        pool = self.pool if pool is None else pool
        pos = torch.arange(self.lens[b])
        pg, sl = self.table_cpu[b, pos // PAGE].long().to(DEV), (pos % PAGE).to(DEV)
        k = pool[self.layer, 0][pg, :, sl]
        v = pool[self.layer, 1].view(self.n_pages, self.hkv, self.hd, PAGE)[pg, :, :, sl]
        return k.double(), v.double()

    def rows_of(self, b):
        return slice(self.starts[b], self.starts[b + 1])

    def positions(self, b):
        return torch.arange(self.lens[b] - self.rows[b], self.lens[b], device=DEV)


# ---------------------------------------------------------------- rotary append
def rope_reference(c, qkv, cos, sin, inter, q_gain, k_gain, eps):
    """Per sequence: q, k, v of its rows in 64 bits and bounds of their errors in float."""
    rot = 2 * cos.shape[1]
    half = rot // 2
    i = torch.arange(half, device=DEV)
    first, second = (2 * i, 2 * i + 1) if inter else (i, i + half)
    for b in range(len(c.rows)):
        x = qkv[c.rows_of(b)].double().view(-1, c.hq + 2 * c.hkv, c.hd)
        pos = c.positions(b)
        out, tol = x.clone(), torch.zeros_like(x)
        for lo, hi, gain in ((0, c.hq, q_gain), (c.hq, c.hq + c.hkv, k_gain)):
            y = x[:, lo:hi]
            e = torch.zeros_like(y)
            if gain is not None:
                y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain.double()
                # hd products and sums (half of that after the root), root, division, two products
                e = (c.hd / 2 + 6) * U * y.abs()
            if half:
                cs, sn = cos[pos].double()[:, None], sin[pos].double()[:, None]
                a, z = y[..., first].clone(), y[..., second].clone()
                ea, ez = e[..., first].clone(), e[..., second].clone()
                y = y.clone()
                y[..., first], y[..., second] = a * cs - z * sn, z * cs + a * sn
                mag = a.abs() + z.abs()   # (|c|, |s| <= 1: two products and a sum)
                e = e.clone()
                e[..., first] = ea + ez + 3 * U * mag
                e[..., second] = ea + ez + 3 * U * mag
            out[:, lo:hi], tol[:, lo:hi] = y, e
        yield b, out, tol


ROPE_CASES = [
    # rows, lens, hq, hkv, hd, rot
    ([1], [1], 1, 1, 64, 64),
    ([1], [701], 32, 8, 128, 128),
    ([3, 0, 1, 8], [3, 5, 700, 23], 4, 2, 64, 32),
    ([17, 1, 40], [33, 16, 40], 8, 8, 128, 64),
    ([5, 2], [21, 18], 40, 40, 128, 24),
    ([33], [33], 6, 2, 64, 16),
    ([130, 70, 16, 15], [200, 71, 48, 31], 12, 4, 128, 128),
    ([1] * 70, list(range(1, 71)), 4, 1, 128, 8),
    ([2, 20], [900, 21], 3, 1, 64, 0),
    ([600, 1], [1500, 2], 16, 2, 64, 56),
]


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("inter", [False, True], ids=["half", "inter"])
@pytest.mark.parametrize("norm", [False, True], ids=["raw", "norm"])
@pytest.mark.parametrize("n", range(len(ROPE_CASES)))
def test_rope_append(n, norm, inter, fp32):
    rows, lens, hq, hkv, hd, rot = ROPE_CASES[n]
    dt = torch.float32 if fp32 else torch.bfloat16
    c = Case(rows, lens, hq, hkv, hd, dt, seed=n, lead=n % 3, tail=(n * 5) % 4, layers=2, layer=1)
    width = (hq + 2 * hkv) * hd
    wide = randn(n + 50, c.n_rows, width + 16 * (n % 3)).to(dt)   # (rows further apart than they are long)
    qkv = wide[:, :width]
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(max(rot, 2), 10000.0, max(lens)))
    if rot == 0:
        cos, sin = cos[:, :0].contiguous(), sin[:, :0].contiguous()
    qg = 1 + 0.2 * randn(n + 60, hd) if norm else None
    kg = 1 + 0.2 * randn(n + 61, hd) if norm else None
    before = c.pool.clone()
    out = torch.full((c.n_rows, hq * hd + 8), 7.0, dtype=dt, device=DEV)[:, :hq * hd]
    got = sb.op_rope_append(c.kv, qkv, hq, cos, sin, interleaved=inter, q_gain=qg, k_gain=kg, eps=1e-5, out=out, layer=1)
    assert got is out
    want_pool = before.clone()
    touched = torch.zeros(c.n_rows, dtype=torch.bool, device=DEV)
    for b, ref, tol in rope_reference(c, qkv, cos, sin, inter, qg, kg, 1e-5):
        touched[c.rows_of(b)] = True
        q = ref[:, :hq]
        tq = tol[:, :hq] + (0 if fp32 else UB) * (q.abs() + tol[:, :hq])
        assert ((got[c.rows_of(b)].double().view(-1, hq, hd) - q).abs() <= tq).all()
        pos = c.positions(b)
        pg, sl = c.table[b].long()[pos // PAGE], pos % PAGE
        k = c.pool[1, 0][pg, :, sl].double()
        tk = tol[:, hq:hq + hkv] * (1 + UB) + UB * ref[:, hq:hq + hkv].abs()
        assert ((k - ref[:, hq:hq + hkv]).abs() <= tk).all()
        want_pool[1, 0][pg, :, sl] = c.pool[1, 0][pg, :, sl]   # (checked)
        want_pool[1, 1].view(c.n_pages, hkv, hd, PAGE)[pg, :, :, sl] = ref[:, hq + hkv:].to(dt).to(torch.bfloat16)
    assert torch.equal(c.pool.view(torch.int16), want_pool.view(torch.int16))   # v's bits, and nothing else written
    assert (out[~touched] == 7).all()
    # in place
    again = qkv.clone() if wide.shape[1] == width else wide.clone()[:, :width]
    pool2 = c.pool.clone()
    c.pool.copy_(before)
    sb.op_rope_append(c.kv, again, hq, cos, sin, interleaved=inter, q_gain=qg, k_gain=kg, eps=1e-5, out=again[:, :hq * hd], layer=1)
    assert torch.equal(again[touched][:, :hq * hd], got[touched]) and torch.equal(again[~touched], qkv[~touched])
    assert torch.equal(again[:, hq * hd:], qkv[:, hq * hd:])
    assert torch.equal(c.pool.view(torch.int16), pool2.view(torch.int16))


def test_rope_append_leaves_out_rows_without_a_place():
    """Positions before the sequence's start or past the table's end, pages outside the pool: nothing is read or written
    for them, the other rows are as they are alone."""
    c = Case([4, 6, 20], [40, 6, 36], 4, 2, 64, torch.float32, seed=3)
    c.kv_len[1] = 3                       # its first three rows would be at -3 .. -1
    c.table[0, 2] = -1                    # keys 32 .. 39 of sequence 0 have no page
    c.table[2, 1] = c.n_pages             # nor have keys 16 .. 31 of sequence 2
    qkv = randn(9, c.n_rows, 8 * 64)
    qkv[4:7] = math.nan
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(64, 10000.0, 34))   # positions 34, 35 of sequence 2 and 36 .. 39 of 0 have no angle
    before = c.pool.clone()
    out = torch.full((c.n_rows, 4 * 64), 7.0, device=DEV)
    sb.op_rope_append(c.kv, qkv, 4, cos, sin, out=out)
    away = list(range(0, 4)) + [4, 5, 6, 28, 29]
    there = [i for i in range(c.n_rows) if i not in away]
    assert (out[away] == 7).all() and (out[there] != 7).any(1).all() and torch.isfinite(out[there]).all()
    changed = (c.pool.view(torch.int16) != before.view(torch.int16)).view(2, c.n_pages, 2, PAGE, 64)
    k_pages = sorted(set(changed[0].any(-1).any(-1).any(-1).nonzero().flatten().tolist()))
    # sequence 1: keys 0 .. 2; sequence 2: keys 32 and 33 (its keys 16 .. 31 have no page)
    assert k_pages == sorted([int(c.table[1, 0]), int(c.table[2, 2])])
    assert changed[0, int(c.table[1, 0])].any(-1).any(0).nonzero().flatten().tolist() == [0, 1, 2]
    assert changed[0, int(c.table[2, 2])].any(-1).any(0).nonzero().flatten().tolist() == [0, 1]


# ---------------------------------------------------------------- attention
def visible(c, b, window=0, prefix=None, doc=None):
    p = c.positions(b)[:, None]
    k = torch.arange(c.lens[b], device=DEV)[None, :]
    see = k <= p
    if window:
        see = see & (k > p - window)
    if prefix is not None:
        see = see | (k < prefix[b])
    if doc is not None:
        see = see & (k >= doc[c.rows_of(b)][:, None])
    return see


def attention_reference(c, q, scale=None, cap=0.0, slopes=None, **rule):
    """Outputs of all rows in 64 bits (zeros for rows of no sequence) and a bound of the error of each."""
    fp32 = q.dtype == torch.float32
    out = torch.zeros(c.n_rows, c.hq, c.hd, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    scale = 1 / math.sqrt(c.hd) if scale is None else scale
    g = c.hq // c.hkv
    for b in range(len(c.rows)):
        if not c.rows[b]:
            continue
        see = visible(c, b, **rule)
        k, v = c.cached(b)
        x = q[c.rows_of(b)].double().view(-1, c.hq, c.hd)
        for h in range(c.hq):
            kh, vh = k[:, h // g], v[:, h // g]
            kh = torch.where(see.any(0)[:, None], kh, 0.0)
            vh = torch.where(see.any(0)[:, None], vh, 0.0)
            z = (x[:, h] @ kh.t()) * scale
            # products and sums in float over hd terms (in any order), the scale; then what follows, each a few roundings
            dz = (c.hd + 4) * U * scale * (x[:, h].abs() @ kh.abs().t())
            if cap:
                z = cap * torch.tanh(z / cap)
                dz = dz + 6 * U * cap    # quotient, exponential, sum, reciprocal, sum, product: about 2 each on values up to 1
            if slopes is not None:
                d = (c.positions(b)[:, None] - torch.arange(c.lens[b], device=DEV)).abs() * slopes[h].double()
                z = z - d
                dz = dz + 2 * U * d
            dz = dz + 4 * U * z.abs()    # to powers of two and from the reference point
            z = torch.where(see, z, -math.inf)
            m = z.amax(1, keepdim=True)
            p = torch.exp(z - torch.where(m == -math.inf, 0.0, m))
            t = p.sum(1, keepdim=True)
            p = p / torch.where(t == 0, 1.0, t)
            o = p @ vh
            # a score off by d moves p by p (d + the mean of d): twice the largest d among the keys that count, plus the
            # exponential's own 2, the sums over the keys (three at a time, then a tree or tiles: at most len)
            far = (p * torch.where(see, dz, 0.0)).sum(1, keepdim=True)
            w = p * (torch.where(see, dz, 0.0) + far + (4 + min(c.lens[b], 4096)) * U)
            e = w @ vh.abs()
            if not fp32:
                e = e + UB * (p @ vh.abs())          # probabilities as bfloat16
                e = e + UB * (o.abs() + e)           # the output
            else:
                e = e + 2 * U * (p @ vh.abs())
            out[c.rows_of(b), h], tol[c.rows_of(b), h] = o, e * 1.01 + 1e-30
    return out.view(c.n_rows, -1), tol.view(c.n_rows, -1)


def check_attention(c, q, out=None, slopes=None, scale=None, cap=0.0, **rule):
    kw = {}
    if "window" in rule:
        kw["window"] = rule["window"]
    if rule.get("prefix") is not None:
        kw["prefix_len"] = torch.tensor(rule["prefix"], dtype=torch.int32, device=DEV)
    if rule.get("doc") is not None:
        kw["doc_start"] = rule["doc"].to(torch.int32)
    if out is None:
        out = torch.full((c.n_rows, c.hq * c.hd), 7.0, dtype=q.dtype, device=DEV)
    want, tol = attention_reference(c, q, scale=scale, cap=cap, slopes=slopes, **rule)
    got = sb.op_paged_attention(c.kv, q, c.hq, scale=scale or 0.0, softcap=cap, slopes=slopes, out=out, layer=c.layer, **kw)
    mine = torch.zeros(c.n_rows, dtype=torch.bool, device=DEV)
    for b in range(len(c.rows)):
        mine[c.rows_of(b)] = True
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad[mine].any(), (int(bad[mine].sum()), float((got.double() - want).abs()[mine].max()), float(((got.double() - want).abs() / tol)[mine].max()))
    assert (got[~mine] == 7).all()
    return got


ATT_SHAPES = [
    # rows, lens, hq, hkv, hd
    ([1], [1], 1, 1, 64),
    ([1], [17], 4, 4, 128),
    ([1], [521], 32, 32, 128),
    ([2, 1, 0, 5], [2, 300, 9, 5], 8, 2, 64),
    ([6], [1300], 32, 8, 128),
    ([1] * 9, [1, 15, 16, 17, 31, 32, 33, 129, 2000], 8, 1, 128),
    ([1, 3, 8], [4097, 100, 9], 64, 2, 64),
    ([1, 1], [6000, 40], 16, 16, 64),
    ([40, 7], [40, 60], 5, 1, 128),
    ([100, 33, 64], [100, 500, 65], 8, 8, 64),
    ([300], [1111], 16, 4, 128),
    ([700, 257], [700, 400], 40, 40, 64),
    # enough rows that blocks of 128 queries fill the card
    ([1500, 1200, 70], [1500, 1333, 900], 24, 4, 64),
    ([1000, 40, 300], [1601, 41, 777], 64, 16, 128),
]


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n", range(len(ATT_SHAPES)))
def test_attention_causal(n, fp32):
    rows, lens, hq, hkv, hd = ATT_SHAPES[n]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=n, lead=n % 2, tail=n % 3, layers=1 + n % 2, layer=n % 2, junk=math.nan)
    wide = (1.5 * randn(n + 20, c.n_rows, hq * hd + 8 * (n % 3))).to(c.dtype)
    check_attention(c, wide[:, :hq * hd])


RULES = [
    dict(cap=20.0), dict(slopes=True), dict(window=1), dict(window=37), dict(window=700), dict(prefix=True), dict(doc=True),
    dict(window=50, prefix=True), dict(doc=True, window=64, cap=5.0), dict(doc=True, prefix=True, slopes=True), dict(scale=0.03, cap=1.0),
    dict(cap=30.0, slopes=True, window=200, prefix=True, doc=True),
]


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [3, 4, 6, 8, 9, 10, 11, 12, 13])
@pytest.mark.parametrize("r", range(len(RULES)), ids=lambda i: "-".join(RULES[i]))
def test_attention_rules(r, shape, fp32):
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=r)
    rule = dict(RULES[r])
    rng = np.random.default_rng(r + 100 * shape)
    if rule.get("slopes"):
        rule["slopes"] = torch.tensor(2.0 ** (-8 * np.arange(1, hq + 1) / hq), dtype=torch.float32, device=DEV)
    if rule.get("prefix"):
        rule["prefix"] = [int(rng.integers(0, n + 2)) for n in lens]     # (0: none; more than there are: all)
    if rule.get("doc"):
        doc = torch.zeros(c.n_rows, dtype=torch.int64, device=DEV)
        for b, n in enumerate(lens):
            starts = np.unique(np.concatenate([[0], rng.integers(0, n, size=1 + n // 60)]))
            pos = np.arange(n - rows[b], n)
            doc[c.rows_of(b)] = torch.tensor(starts[np.searchsorted(starts, pos, side="right") - 1], device=DEV)
        rule["doc"] = doc
    check_attention(c, (2 * randn(r + 20, c.n_rows, hq * hd)).to(c.dtype), **rule)


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("cap", [1e6, 1e30])
@pytest.mark.parametrize("shape", [4, 8, 10, 12, 13])
def test_a_cap_far_above_the_scores_changes_nothing(shape, cap, fp32):
    """cap tanh(z / cap) is z but for z^3 / (3 cap^2), below 1e-9 here."""
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=shape)
    q = (2 * randn(shape + 40, c.n_rows, hq * hd)).to(c.dtype)
    want, tol = attention_reference(c, q)
    got = sb.op_paged_attention(c.kv, q, hq, softcap=cap, layer=c.layer)
    # quotient, square, three steps of the series that count, product: 8 roundings of z more, beside the hd + 4 of its bound
    bad = ~((got.double() - want).abs() <= tol * (1 + 8 / (hd + 4)))
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / tol).max()))


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [4, 12, 13])
def test_a_cap_above_scores_whose_squares_floats_cannot_hold(shape, fp32):
    """Scores of 1e20 far below a cap of 1e30: one key has all the weight, as without a cap."""
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=shape + 3)
    q = (1e20 * randn(shape + 80, c.n_rows, hq * hd)).to(c.dtype)
    want = sb.op_paged_attention(c.kv, q, hq, scale=1.0, layer=c.layer)
    got = sb.op_paged_attention(c.kv, q, hq, scale=1.0, softcap=1e30, layer=c.layer)
    assert torch.isfinite(want.float()).all() and torch.equal(got, want)


@pytest.mark.parametrize("cap", [512.0, 513.0])
@pytest.mark.parametrize("shape", [4, 12, 13])
def test_both_ways_to_cap_the_scores(shape, cap):
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.bfloat16, seed=shape)
    check_attention(c, (2 * randn(shape + 60, c.n_rows, hq * hd)).to(c.dtype), cap=cap, scale=4.0)


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [3, 5, 10, 11, 12, 13])
def test_rows_that_see_nothing_get_zeros(shape, fp32):
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=5, junk=math.inf)
    doc = torch.zeros(c.n_rows, dtype=torch.int64, device=DEV)
    blind = torch.arange(c.n_rows, device=DEV) % 3 == 1
    doc[blind] = 1 << 20     # a document that starts behind every key
    got = check_attention(c, randn(6, c.n_rows, hq * hd).to(c.dtype), doc=doc)
    assert (got[blind] == 0).all() and (got[~blind] != 0).any(1).all()
    # all of them, and sequences without keys
    doc[:] = 1 << 20
    assert (check_attention(c, randn(6, c.n_rows, hq * hd).to(c.dtype), doc=doc) == 0).all()
    c.kv_len[:] = 0
    assert (sb.op_paged_attention(c.kv, randn(6, c.n_rows, hq * hd).to(c.dtype), hq) == 0).all()


@pytest.mark.parametrize("bits", [math.nan, math.inf, -math.inf, torch.finfo(torch.bfloat16).min], ids=str)
@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [0, 3, 4, 8, 10, 11, 12, 13])
def test_what_a_row_does_not_see_does_not_reach_it(shape, fp32, bits):
    """Keys and values of another document of the same sequence, of later positions and of slots past the end hold `bits`:
    rows that do not see them are, bit for bit, what they are without."""
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    dt = torch.float32 if fp32 else torch.bfloat16
    c = Case(rows, lens, hq, hkv, hd, dt, seed=8)
    q = randn(9, c.n_rows, hq * hd).to(dt)
    doc = torch.zeros(c.n_rows, dtype=torch.int32, device=DEV)
    sick = torch.zeros(c.n_rows, dtype=torch.bool, device=DEV)
    for b, n in enumerate(lens):
        cut = n - (rows[b] + 1) // 2      # the later half of the rows is a second document ...
        pos = c.positions(b)
        doc[c.rows_of(b)] = torch.where(pos >= cut, cut, 0).to(torch.int32)
    clean = sb.op_paged_attention(c.kv, q, hq, doc_start=doc)
    for b, n in enumerate(lens):
        cut = n - (rows[b] + 1) // 2
        hit = [x for x in (cut - 1, cut - 2, (n + cut) // 2) if 0 <= x < n and rows[b] > 0]   # ... bits at the end of the first, in the middle of the second
        for x in hit:
            pg = int(c.table_cpu[b, x // PAGE])
            c.pool[0, 0, pg, :, x % PAGE, 3] = bits
            c.pool[0, 1].view(c.n_pages, hkv, hd, PAGE)[pg, :, 5, x % PAGE] = bits
            pos = c.positions(b)
            sick[c.rows_of(b)] |= (pos >= x) & (doc[c.rows_of(b)] <= x)
        for x in range(n, (n + PAGE - 1) // PAGE * PAGE):   # slots past the end
            pg = int(c.table_cpu[b, x // PAGE])
            c.pool[0, 0, pg, :, x % PAGE] = bits
            c.pool[0, 1].view(c.n_pages, hkv, hd, PAGE)[pg, :, :, x % PAGE] = bits
    got = sb.op_paged_attention(c.kv, q, hq, doc_start=doc)
    assert torch.equal(got[~sick], clean[~sick])
    if math.isnan(bits) and sick.any():
        assert not torch.isfinite(got[sick].view(-1, hq, hd)[:, :, 5]).any()


@pytest.mark.parametrize("shape", [4, 10, 12])
def test_large_and_equal_scores(shape):
    """Scores near the top of the float range, and rows whose scores are all alike."""
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32, seed=2)
    c.pool[:, 0] = 0
    check_attention(c, randn(3, c.n_rows, hq * hd))
    c.pool[:, 0] = randn(4, *c.pool[:, 0].shape).to(torch.bfloat16)
    q = 1e30 * randn(3, c.n_rows, hq * hd)
    got = sb.op_paged_attention(c.kv, q, hq)
    for b in range(len(rows)):   # the largest score takes all
        k, v = c.cached(b)
        see = visible(c, b)
        for h in range(hq):
            z = q[c.rows_of(b)].double().view(-1, hq, hd)[:, h] @ k[:, h // (hq // hkv)].t()
            z = torch.where(see, z, -math.inf)
            want = v[:, h // (hq // hkv)][z.argmax(1)]
            assert torch.equal(got[c.rows_of(b)].view(-1, hq, hd)[:, h].double(), want)


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows,lens,hq,hkv,hd", [
    ([i % 3 for i in range(300)], [i % 3 + i // 2 for i in range(300)], 4, 2, 64),
    ([1] * 4200, [1 + i % 40 for i in range(4200)], 2, 1, 64),
    ([40] * 80, [40 + 3 * i for i in range(80)], 16, 4, 64),
    ([0] * 130 + [2], [9] * 130 + [700], 40, 1, 64),
    ([8] * 130, [8 + 2 * i for i in range(130)], 32, 8, 128),
    ([i % 17 for i in range(120)], [20 + i for i in range(120)], 32, 8, 64),
    ([(13 * i) % 60 for i in range(40)], [(13 * i) % 60 + 100 * (i % 3) for i in range(40)], 64, 8, 64),
    ([300, 0, 300, 1, 299], [300, 0, 300, 4000, 600], 64, 8, 128),
    ([i % 3 for i in range(200)], [i % 3 + (37 * i) % 900 for i in range(200)], 8, 2, 64),
    ([1 + i % 16 for i in range(256)], [16 + 3 * i for i in range(256)], 16, 4, 128),
    ([1] * 40, [1 + 50 * (i % 20) for i in range(40)], 8, 2, 128),
    ([3] * 65, [50] * 65, 6, 2, 128)], ids=lambda x: str(len(x)) if isinstance(x, list) else str(x))
def test_many_sequences(rows, lens, hq, hkv, hd, fp32):
    """Sequences without rows or equally long ones, more of them than a wave looks at at once; the same through the append."""
    dt = torch.float32 if fp32 else torch.bfloat16
    c = Case(rows, lens, hq, hkv, hd, dt, seed=len(rows), lead=1, tail=2, junk=math.nan)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(hd, 10000.0, max(lens)))
    qkv = randn(5, c.n_rows, (hq + 2 * hkv) * hd).to(dt)
    out = torch.full((c.n_rows, hq * hd), 7.0, dtype=dt, device=DEV)
    q = sb.op_rope_append(c.kv, qkv, hq, cos, sin, out=out)
    for b, ref, tol in rope_reference(c, qkv, cos, sin, False, None, None, 0.0):
        x = q[c.rows_of(b)].double().view(-1, hq, hd)
        assert ((x - ref[:, :hq]).abs() <= tol[:, :hq] + (0 if fp32 else UB) * (ref[:, :hq].abs() + tol[:, :hq])).all()
    assert (q[0] == 7).all() and (q[-2:] == 7).all()
    got = sb.op_paged_attention(c.kv, q, hq, out=torch.full_like(q, 7.0))
    assert (got[0] == 7).all() and (got[-2:] == 7).all() and torch.isfinite(got.float()).all()
    some = [b for b in range(len(rows)) if rows[b]][:: max(1, len(rows) // 24)]   # (the oracle on a few of them)
    for b in some:
        one = Case([rows[b]], [lens[b]], hq, hkv, hd, dt, seed=0)
        k, v = c.cached(b)
        pos = torch.arange(lens[b], device=DEV)
        pg = one.table[0].long()[pos // PAGE]
        one.pool[0, 0][pg, :, pos % PAGE] = k.to(torch.bfloat16)
        one.pool[0, 1].view(one.n_pages, hkv, hd, PAGE)[pg, :, :, pos % PAGE] = v.to(torch.bfloat16)
        want, tol = attention_reference(one, q[c.rows_of(b)])
        assert ((got[c.rows_of(b)].double() - want).abs() <= tol).all(), b


def test_table_rows_apart_and_lengths_above_max_len():
    c = Case([3, 5], [100, 61], 8, 2, 128, torch.bfloat16, seed=2, table_ld=9)
    wide = torch.full((2, 25), -1, dtype=torch.int32, device=DEV)
    wide[:, :9] = c.table
    kv = sb.Paged(c.pool, wide[:, :9], c.row_start, c.kv_len, n_rows=8)
    assert kv.c.table_ld == 25
    q = randn(3, 8, 1024).to(torch.bfloat16)
    assert torch.equal(sb.op_paged_attention(kv, q, 8), sb.op_paged_attention(c.kv, q, 8))
    # max_len cuts a longer sequence: its rows are the last max_len's
    short = sb.Paged(c.pool, c.table, c.row_start, c.kv_len, n_rows=8, max_len=64)
    c.kv_len[0] = 64
    assert torch.equal(sb.op_paged_attention(short, q, 8), sb.op_paged_attention(c.kv, q, 8))


@pytest.mark.parametrize("shape", [2, 5, 6])
def test_scratch_needs_no_clearing(shape):
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32, seed=1)
    q = randn(2, c.n_rows, hq * hd)
    scratch = sb.paged_attention_scratch(c.kv, hq)
    want = sb.op_paged_attention(c.kv, q, hq, scratch=scratch)
    for fill in (0xff, 0x7f):
        scratch.fill_(fill)
        assert torch.equal(sb.op_paged_attention(c.kv, q, hq, scratch=scratch), want)


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [3, 10, 12])
def test_a_row_without_numbers_stays_alone(shape, fp32):
    """NaN and infinite queries make their own outputs so, the others keep their bits."""
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=3)
    q = randn(4, c.n_rows, hq * hd).to(c.dtype)
    want = sb.op_paged_attention(c.kv, q, hq)
    bad = torch.arange(c.n_rows, device=DEV) % 5 == 2
    q[bad] = math.nan
    q[bad, 1] = math.inf
    got = sb.op_paged_attention(c.kv, q, hq)
    assert torch.equal(got[~bad], want[~bad]) and torch.isnan(got[bad]).all()


def test_attention_pages_outside_the_pool_read_as_zeros():
    c = Case([2, 90], [70, 200], 8, 2, 64, torch.float32, seed=4, spare=0)
    zero = c.pool.clone()
    q = randn(5, c.n_rows, 8 * 64)
    for b, i, bad in ((0, 1, -1), (0, 4, c.n_pages), (1, 3, -7), (1, 12, 0x7fffffff)):
        pg = int(c.table_cpu[b, i])
        zero[:, :, pg] = 0
    c2 = sb.Paged(zero, c.table.clone(), c.row_start, c.kv_len, n_rows=c.n_rows)
    want = sb.op_paged_attention(c2, q, 8)
    for b, i, bad in ((0, 1, -1), (0, 4, c.n_pages), (1, 3, -7), (1, 12, 0x7fffffff)):
        c.table[b, i] = bad
    assert torch.equal(sb.op_paged_attention(c.kv, q, 8), want)


@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", [2, 4, 10, 12, 13])
def test_attention_in_place(shape, fp32):
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.float32 if fp32 else torch.bfloat16, seed=6)
    q = randn(7, c.n_rows, hq * hd).to(c.dtype)
    want = sb.op_paged_attention(c.kv, q, hq)
    assert torch.equal(sb.op_paged_attention(c.kv, q, hq, out=q), want) and torch.equal(q, want)


def test_row_starts_and_lengths_out_of_range_are_cut():
    c = Case([4, 4], [40, 20], 4, 2, 64, torch.float32, seed=1)
    q = randn(2, c.n_rows, 256)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(64, 10000.0, 64))
    want = sb.op_paged_attention(c.kv, q, 4)
    c.row_start[2] = 99     # more rows than there are: the rows that are there, counted from the sequence's end
    assert torch.equal(sb.op_paged_attention(c.kv, q, 4), want)
    c.kv_len[0] = 1 << 30   # longer than the table: max_len
    c.table[0] = int(c.table_cpu[0, 0])
    assert torch.isfinite(sb.op_paged_attention(c.kv, q, 4)).all()
    before = c.pool.clone()
    sb.op_rope_append(c.kv, randn(3, c.n_rows, 8 * 64), 4, cos, sin)
    diff = (c.pool != before).any(-1).any(-1).any(-1)[0].any(0).nonzero().flatten().tolist()
    assert set(diff) <= {int(c.table_cpu[0, 0])} | set(c.table_cpu[1, :2].tolist())
    c.row_start[:] = torch.tensor([5, 2, -3], dtype=torch.int32)   # descending: no rows
    out = torch.full((c.n_rows, 256), 7.0, device=DEV)
    assert (sb.op_paged_attention(c.kv, q, 4, out=out) == 7).all()


@pytest.mark.parametrize("starts", [[100, 150, 0, 64], [200, 0, 210, 40], [7, 6, 300, 5]])
def test_row_starts_that_do_not_ascend_stay_within_the_operands(starts):
    """Which rows are worked on is open then; nothing else is touched, and the next call is as ever."""
    c = Case([70, 60, 200], [5000, 3000, 4000], 6, 2, 64, torch.float32, seed=4)
    q = randn(2, c.n_rows, 384)
    want = sb.op_paged_attention(c.kv, q, 6)
    scratch = sb.paged_attention_scratch(c.kv, 6)
    assert scratch.numel() > 256          # (the keys are split)
    scratch.fill_(0x7f)
    good, pool, keep = c.row_start.clone(), c.pool.clone(), torch.full((3 * c.n_rows, 384), 7.0, device=DEV)
    c.row_start.copy_(torch.tensor(starts, dtype=torch.int32))
    sb.op_paged_attention(c.kv, q, 6, out=keep[c.n_rows:2 * c.n_rows], scratch=scratch)
    assert (keep[:c.n_rows] == 7).all() and (keep[2 * c.n_rows:] == 7).all() and torch.equal(c.pool, pool)
    c.row_start.copy_(good)
    assert torch.equal(sb.op_paged_attention(c.kv, q, 6, scratch=scratch), want)


def test_empty_batches():
    c = Case([0, 0], [10, 0], 4, 2, 64, torch.bfloat16)
    q = torch.empty((0, 256), dtype=torch.bfloat16, device=DEV)
    assert sb.op_paged_attention(c.kv, q, 4).shape == (0, 256)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(64, 10000.0, 8))
    assert sb.op_rope_append(c.kv, torch.empty((0, 512), dtype=torch.bfloat16, device=DEV), 4, cos, sin).shape == (0, 256)
    kv = sb.Paged(c.pool, c.table[:0], torch.zeros(1, dtype=torch.int32, device=DEV), c.kv_len[:0], n_rows=2)
    out = torch.full((2, 256), 7.0, device=DEV)
    assert (sb.op_paged_attention(kv, torch.zeros((2, 256), device=DEV), 4, out=out) == 7).all()


def test_offsets_past_32_bits():
    """A pool whose layer has more than 2^32 bytes of keys: the last pages are written and read."""
    hq, hkv, hd, n_pages = 8, 8, 128, 140000
    pool = torch.empty((1, 2, n_pages, hkv, PAGE, hd), dtype=torch.bfloat16, device=DEV)
    lens, rows = [100, 48], [20, 1]
    pages = [n_pages - 1 - 2 * i for i in range(7)], [0, 70000, n_pages - 2]
    table = torch.zeros((2, 7), dtype=torch.int32)
    table[0], table[1, :3] = torch.tensor(pages[0], dtype=torch.int32), torch.tensor(pages[1], dtype=torch.int32)
    c = Case(rows, lens, hq, hkv, hd, torch.bfloat16, seed=3)
    for b in range(2):
        for i, p in enumerate(pages[b]):
            pool[:, :, p] = c.pool[:, :, int(c.table_cpu[b, i])]
    kv = sb.Paged(pool, table.to(DEV), c.row_start, c.kv_len, n_rows=c.n_rows)
    qkv = randn(4, c.n_rows, (hq + 2 * hkv) * hd).to(torch.bfloat16)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(hd, 10000.0, 100))
    qa, qb = (sb.op_rope_append(k, qkv, hq, cos, sin) for k in (c.kv, kv))
    assert torch.equal(qa, qb)
    for b in range(2):
        for i, p in enumerate(pages[b]):
            assert torch.equal(pool[:, :, p], c.pool[:, :, int(c.table_cpu[b, i])])
    assert torch.equal(sb.op_paged_attention(c.kv, qa, hq), sb.op_paged_attention(kv, qb, hq))
    src = pool[:, :, n_pages - 1].clone()
    sb.op_copy_pages(pool, pool, [n_pages - 4], [n_pages - 1])
    assert torch.equal(pool[:, :, n_pages - 4], src)


@pytest.mark.parametrize("shape", [2, 5, 6, 10, 13])
def test_attention_captured_and_replayed(shape):
    """Captured with one batch, replayed while lengths and keys change in place; eager calls in between."""
    rows, lens, hq, hkv, hd = ATT_SHAPES[shape]
    c = Case(rows, lens, hq, hkv, hd, torch.bfloat16, seed=11)
    q = randn(1, c.n_rows, hq * hd).to(c.dtype)
    out, scratch = torch.zeros_like(q), sb.paged_attention_scratch(c.kv, hq)
    sb.op_paged_attention(c.kv, q, hq, out=out, scratch=scratch)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sb.op_paged_attention(c.kv, q, hq, out=out, scratch=scratch)
    for i in range(4):
        if i:
            short = [max(r, n - 3 * i) for r, n in zip(rows, lens)]
            c.kv_len.copy_(torch.tensor(short, dtype=torch.int32))
            q.copy_(randn(30 + i, c.n_rows, hq * hd).to(c.dtype))
        want = sb.op_paged_attention(c.kv, q, hq)
        torch.cuda.synchronize()
        out.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_calls_on_another_stream_and_side_by_side():
    cs = [Case([1, 2], [3000, 500], 16, 4, 128, torch.bfloat16, seed=s) for s in (1, 2)]
    qs = [randn(s, 3, 16 * 128).to(torch.bfloat16) for s in (3, 4)]
    want = [sb.op_paged_attention(c.kv, q, 16) for c, q in zip(cs, qs)]
    scratch = [sb.paged_attention_scratch(c.kv, 16) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    outs = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, q, o, sc, st in zip(cs, qs, outs, scratch, streams):
            with torch.cuda.stream(st):
                sb.op_paged_attention(c.kv, q, 16, out=o, scratch=sc)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_binding_refusals():
    c = Case([2], [20], 4, 2, 64, torch.float32)
    q = randn(1, 2, 256)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(64, 10000.0, 32))
    qkv = randn(2, 2, 512)
    att, rope = (lambda **k: sb.op_paged_attention(**{**dict(kv=c.kv, q=q, n_heads=4), **k})), (lambda **k: sb.op_rope_append(**{**dict(kv=c.kv, qkv=qkv, n_heads=4, rope_cos=cos, rope_sin=sin), **k}))
    for bad in (dict(q=q[:1]), dict(q=q[:, :128]), dict(q=q.cpu()), dict(layer=1), dict(layer=-1), dict(slopes=torch.zeros(3, device=DEV)),
                dict(prefix_len=torch.zeros(2, dtype=torch.int32, device=DEV)), dict(doc_start=torch.zeros(3, dtype=torch.int32, device=DEV)),
                dict(q=q.t().contiguous().t()), dict(out=torch.empty((2, 128), device=DEV)), dict(scratch=torch.empty(512, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            att(**bad)
    for bad in (dict(q=q.half()), dict(slopes=torch.zeros(4, dtype=torch.float64, device=DEV)), dict(doc_start=torch.zeros(2, dtype=torch.int64, device=DEV)),
                dict(out=torch.empty((2, 256), dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(TypeError):
            att(**bad)
    for bad in (dict(qkv=qkv[:, :500]), dict(qkv=qkv.cpu()), dict(rope_cos=cos[:4]), dict(rope_sin=sin.cpu()), dict(q_gain=torch.ones(63, device=DEV)), dict(layer=2)):
        with pytest.raises(ValueError):
            rope(**bad)
    for bad in (dict(qkv=qkv.double()), dict(k_gain=torch.ones(64, device=DEV).half()), dict(out=torch.empty((2, 256), dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(TypeError):
            rope(**bad)
    with pytest.raises(sb.SbError):
        rope(rope_cos=cos[:, :6].contiguous(), rope_sin=sin[:, :6].contiguous())
    with pytest.raises(sb.SbError):
        att(softcap=-1.0)
    for bad in (dict(window=-1), dict(window=-(1 << 32) + 5)):
        with pytest.raises(sb.SbError):
            att(**bad)
    for bad in (dict(scale=1e-50), dict(softcap=1e-60)):   # (0 in 32 bits: another rule)
        with pytest.raises(ValueError):
            att(**bad)
    assert torch.equal(att(window=(1 << 32) + 1), att())
    with pytest.raises(sb.SbError):
        rope(out=qkv[:, 8:264])
    mk = lambda **k: sb.Paged(**{**dict(pool=c.pool, table=c.table, row_start=c.row_start, kv_len=c.kv_len, n_rows=2), **k})
    for bad in (dict(pool=c.pool[0]), dict(pool=c.pool.cpu()), dict(pool=c.pool.transpose(3, 4)), dict(table=c.table[0]), dict(table=c.table.cpu()),
                dict(row_start=c.row_start[:1]), dict(kv_len=c.kv_len.cpu()), dict(max_len=0), dict(max_len=33)):
        with pytest.raises(ValueError):
            mk(**bad)
    for bad in (dict(pool=c.pool.float()), dict(table=c.table.long()), dict(kv_len=c.kv_len.long())):
        with pytest.raises(TypeError):
            mk(**bad)


def test_agrees_with_the_single_sequence_operators():
    """Append and plain causal attention of one sequence: what sb_op_attention / sb_op_prompt_attention give (their own
    precision is 16 bits of queries and probabilities)."""
    for rows, past in ((6, 900), (400, 130)):
        hq, hkv, hd = 8, 2, 128
        c = Case([rows], [past + rows], hq, hkv, hd, torch.float32, seed=past, spare=0)   # (they take a pool of as many pages as the table)
        qkv = randn(3, rows, (hq + 2 * hkv) * hd)
        cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table(hd, 10000.0, past + rows))
        pool = c.pool.clone()
        if rows <= sb.SB_MAX_W:
            want = sb.op_attention(qkv, hq, hkv, hd, sb.BF16, pool, c.table[0], 0, cos, sin, past)
        else:
            want = sb.op_prompt_attention(qkv, hq, hkv, hd, pool, c.table[0], 0, cos, sin, past)
        q = sb.op_rope_append(c.kv, qkv, hq, cos, sin)
        got = sb.op_paged_attention(c.kv, q, hq)
        own = torch.stack(c.used_mask())   # (sb_op_attention stores pieces of eight values, zeros behind the last key)
        k = (pool[0].view(torch.int16) != c.pool[0].view(torch.int16)) & own
        assert not k[1].any() and k[0].float().mean() < 1e-3   # (a rotated key next to a rounding border)
        # such a key is a step of 2^-7 off in one of its dims, which moves a score by 2^-7 |q| |k| / sqrt(hd) at most
        assert (got - want).abs().max() < 0.05
        assert (got - want).abs().mean() < 1e-4


# ---------------------------------------------------------------- page copies
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("layers,n,hkv,hd", [(1, 1, 1, 64), (3, 7, 2, 64), (2, 900, 1, 64), (4, 33, 8, 128), (1, 5, 40, 128)])
def test_copy_pages_between_pools(layers, n, hkv, hd, dt):
    g = np.random.default_rng(n)
    src = randn(1, layers, 2, n + 4, hkv, PAGE, hd).to(dt)
    dst = randn(2, layers, 2, n + 9, hkv, PAGE, hd).to(dt)
    frm, to = g.integers(0, n + 4, n), g.permutation(n + 9)[:n]   # (a page may be read twice)
    want = dst.clone()
    want[:, :, torch.tensor(to, device=DEV)] = src[:, :, torch.tensor(frm, device=DEV)]
    keep = src.clone()
    sb.op_copy_pages(dst, src, to, frm)
    assert torch.equal(dst, want) and torch.equal(src, keep)
    sb.op_copy_pages(dst, src, [], [])
    assert torch.equal(dst, want)


def test_copy_pages_refusals_from_python():
    a, b = torch.zeros((1, 2, 4, 2, PAGE, 64), device=DEV), torch.zeros((1, 2, 6, 2, PAGE, 64), device=DEV)
    for bad in ((a, b.to(torch.bfloat16)), (a, b[:, :1]), (a, torch.zeros((1, 2, 4, 3, PAGE, 64), device=DEV)), (a.cpu(), b), (a[0], b[0])):
        with pytest.raises(ValueError):
            sb.op_copy_pages(*bad, [0], [0])
    with pytest.raises(ValueError):
        sb.op_copy_pages(a, b, [0, 1], [0])
    for to, frm in (([4], [0]), ([0], [6]), ([1, 1], [2, 3]), ([-1], [0])):
        with pytest.raises(sb.SbError):
            sb.op_copy_pages(a, b, to, frm)
    with pytest.raises(sb.SbError):
        sb.op_copy_pages(a, a, [0, 1], [1, 2])


# ---------------------------------------------------------------- forked sessions
@pytest.mark.parametrize("bf16", [False, True], ids=["fp32", "bf16"])
def test_forked_session_continues_as_the_source_does(bf16):
    kw = dict(weight_dtype=sb.BF16, kv_dtype=sb.BF16, d_ffn=768) if bf16 else {}
    shape = si.tiny_shape(**kw)
    m = gpu_model(shape, si.make_weights(shape, 77), 160)
    p = gpu_params(2, 4, threshold=0.0)
    prompt = si.make_prompt(shape.vocab, 37, 5)
    src = m.session()
    src.prefill(prompt)
    head, _ = src.decode(9, p)
    rng = np.random.default_rng(0)
    forks = [src.fork(), src.fork(rng.permutation(10))]
    base, _ = src.decode(40, p)
    for f in forks:
        out, st = f.decode(40, p)
        assert out.tolist() == base.tolist() and st["emitted"] > 0
    # independent caches: a fork of a fork from an earlier point, with another token
    f = forks[1]
    f.rewind(37, int(head[0]))
    g = f.fork()
    a, _ = g.decode(20, p)
    ref = m.session()
    ref.prefill(prompt)
    ref.rewind(37, int(head[0]))
    b, _ = ref.decode(20, p)
    assert a.tolist() == b.tolist()
    again, _ = forks[0].decode(5, p)
    tail, _ = src.decode(5, p)
    assert again.tolist() == tail.tolist()


def test_fork_refusals():
    shape = si.tiny_shape()
    w = si.make_weights(shape, 3)
    m, other = gpu_model(shape, w, 64), gpu_model(shape, w, 64)
    a, b = m.session(), m.session()
    with pytest.raises(sb.SbError) as e:
        b.fork_from(a)
    assert e.value.code == sb.ESTATE
    a.prefill(si.make_prompt(shape.vocab, 7, 1))
    for dst, src in ((a, a), (other.session(), a)):
        with pytest.raises(sb.SbError) as e:
            dst.fork_from(src)
        assert e.value.code == sb.EINVAL
    p = gpu_params(2, 4, threshold=0.0)
    a.draft_step(p)
    with pytest.raises(sb.SbError) as e:
        b.fork_from(a)
    assert e.value.code == sb.ESTATE
    a.verify(p)
    b.fork_from(a)
    # a destination with an open round drops it
    b.draft_step(p)
    b.fork_from(a)
    assert b.open_rows() == 0 and b.committed_len() == a.committed_len()
    x, _ = a.decode(12, p)
    y, _ = b.decode(12, p)
    assert x.tolist() == y.tolist()


# ---------------------------------------------------------------- all of them together
@pytest.mark.parametrize("fp32", [True, False], ids=["fp32", "bf16"])
def test_a_serving_loop(fp32):
    """Prompts of two sequences, one of them forked twice (full pages shared, the last one copied), tokens one at a time, a
    sequence that ends, a compacted cache: every output is attention over that sequence's own history."""
    hq, hkv, hd, n_pages, layers = 8, 2, 64, 64, 2
    dt = torch.float32 if fp32 else torch.bfloat16
    pool = torch.full((layers, 2, n_pages, hkv, PAGE, hd), math.nan, dtype=torch.bfloat16, device=DEV)
    pages = sb.Pages(n_pages)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in sb.rope_table_scaled(hd, 10000.0, 256, sb.ROPE_PARTS, 4.0, 64))
    gain = 1 + 0.1 * randn(1, hd)
    seqs = {}      # name -> (pages, per layer the float64 history of rounded k and v)
    step = [0]

    def run(batch):   # batch: {name: new rows}
        names = list(batch)
        rows = [batch[n] for n in names]
        for n in names:
            s = seqs.setdefault(n, dict(pages=[], k=[[], []], v=[[], []], len=0))
            s["len"] += batch[n]
            while len(s["pages"]) * PAGE < s["len"]:
                s["pages"] += pages.alloc(1).tolist()
        table = torch.zeros((len(names), 16), dtype=torch.int32)
        for b, n in enumerate(names):
            table[b, :len(seqs[n]["pages"])] = torch.tensor(seqs[n]["pages"], dtype=torch.int32)
        starts = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device=DEV)
        lens = torch.tensor([seqs[n]["len"] for n in names], dtype=torch.int32, device=DEV)
        kv = sb.Paged(pool, table.to(DEV), starts, lens, n_rows=sum(rows))
        for layer in range(layers):
            step[0] += 1
            qkv = randn(100 + step[0], sum(rows), (hq + 2 * hkv) * hd).to(dt)
            q = sb.op_rope_append(kv, qkv, hq, cos, sin, q_gain=gain, k_gain=gain, layer=layer)
            out = sb.op_paged_attention(kv, q, hq, softcap=20.0, window=100, layer=layer)
            at = 0
            for b, n in enumerate(names):
                s = seqs[n]
                c = Case([rows[b]], [s["len"]], hq, hkv, hd, dt, seed=0)
                pos = torch.arange(s["len"] - rows[b], s["len"], device=DEV)
                pg = torch.tensor(s["pages"], device=DEV)[pos // PAGE]
                s["k"][layer].append(pool[layer, 0][pg, :, pos % PAGE].clone())
                s["v"][layer].append(pool[layer, 1].view(n_pages, hkv, hd, PAGE)[pg, :, :, pos % PAGE].clone())
                want_v = qkv[at:at + rows[b]].view(rows[b], -1, hd)[:, hq + hkv:].to(torch.bfloat16)
                assert torch.equal(s["v"][layer][-1], want_v)
                # the history as it was written, in a cache of its own
                k, v = torch.cat(s["k"][layer]), torch.cat(s["v"][layer])
                allpos = torch.arange(s["len"], device=DEV)
                own = c.table[0].long()[allpos // PAGE]
                c.pool[0, 0][own, :, allpos % PAGE] = k
                c.pool[0, 1].view(c.n_pages, hkv, hd, PAGE)[own, :, :, allpos % PAGE] = v
                want, tol = attention_reference(c, q[at:at + rows[b]], cap=20.0, window=100)
                assert ((out[at:at + rows[b]].double() - want).abs() <= tol).all(), (n, layer)
                at += rows[b]

    def fork(src, dst):
        s = seqs[src]
        full = s["len"] // PAGE
        pages.share(s["pages"][:full])
        new = s["pages"][:full]
        if s["len"] % PAGE:
            last = pages.alloc(1).tolist()
            sb.op_copy_pages(pool, pool, last, s["pages"][full:full + 1])
            new = new + last
        seqs[dst] = dict(pages=new, k=[list(x) for x in s["k"]], v=[list(x) for x in s["v"]], len=s["len"])

    run({"a": 45, "b": 130})
    fork("a", "c")
    fork("a", "d")
    for _ in range(5):
        run({"a": 1, "b": 1, "c": 1, "d": 2})
    pages.release(seqs.pop("b")["pages"])
    run({"e": 20, "c": 1})
    pages.release(seqs.pop("a")["pages"])
    src, dst = pages.compact()
    assert len(src)
    sb.op_copy_pages(pool, pool, dst, src)
    move = dict(zip(src.tolist(), dst.tolist()))
    for s in seqs.values():
        s["pages"] = [move.get(p, p) for p in s["pages"]]
    pool[:, :, pages.used():] = math.nan
    for _ in range(3):
        run({"c": 1, "e": 3, "d": 1})
