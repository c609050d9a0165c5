"""Operators on a paged cache, what needs no GPU: refusals before anything is launched, the bookkeeping of shared pages,
rotary tables for long contexts."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2604_12247_amd as sb
from paper_2604_12247_amd import binding as B

P = 0x7f0000000000   # an aligned address: every call below is refused before it is looked at


def paged(**kw):
    d = dict(pool=P, table=P + (1 << 32), row_start=P + (2 << 32), kv_len=P + (3 << 32), n_pages=64, n_kv_heads=8, head_dim=128, n_seq=3,
             n_rows=10, table_ld=16, max_len=256)
    d.update(kw)
    return B.sb_paged(**d)


Q, KV_ROW, Q_ROW = P + (4 << 32), (32 + 16) * 128, 32 * 128
OUT, TAB, SCRATCH = P + (5 << 32), P + (6 << 32), P + (7 << 32)


def rope(kv=None, **kw):
    a = dict(layer=0, qkv=Q, x_dtype=sb.FP32, ld_qkv=KV_ROW, n_heads=32, q_gain=None, k_gain=None, eps=1e-6, cos=TAB, sin=TAB, n_pos=256,
             rot=128, layout=0, q_out=OUT, ld_q=Q_ROW)
    a.update(kw)
    return sb.lib().sb_op_rope_append(C.byref(kv or paged()), *a.values(), None)


def attention(kv=None, rule=None, **kw):
    a = dict(layer=0, q=Q, x_dtype=sb.BF16, ld_q=Q_ROW, n_heads=32, rule=rule, out=OUT, ld_out=Q_ROW, scratch=SCRATCH, n=1 << 40)
    a.update(kw)
    if a["rule"] is not None:
        a["rule"] = C.byref(a["rule"])
    return sb.lib().sb_op_paged_attention(C.byref(kv or paged()), *a.values(), None)


BAD_PAGED = [dict(head_dim=96), dict(n_kv_heads=0), dict(n_kv_heads=5), dict(n_seq=-1), dict(n_rows=-1), dict(n_pages=0), dict(table_ld=0),
             dict(max_len=0), dict(max_len=257), dict(pool=None), dict(table=None), dict(row_start=None), dict(kv_len=None),
             dict(pool=P + 8), dict(table=P + 2), dict(n_rows=1 << 30), dict(n_seq=1 << 30),
             dict(table_ld=1 << 21, max_len=(1 << 24) + 1)]


@pytest.mark.parametrize("bad", BAD_PAGED, ids=str)
def test_a_bad_cache_is_refused(bad):
    assert rope(paged(**bad)) == sb.EINVAL
    assert attention(paged(**bad)) == sb.EINVAL
    assert sb.lib().sb_last_error().startswith(b"op_")


@pytest.mark.parametrize("bad", [
    dict(layer=-1), dict(x_dtype=2), dict(n_heads=0), dict(n_heads=33), dict(n_heads=1 << 20), dict(qkv=None), dict(q_out=None), dict(qkv=Q + 8),
    dict(q_out=OUT + 4), dict(ld_qkv=KV_ROW - 4), dict(ld_qkv=KV_ROW + 2), dict(ld_q=Q_ROW - 4), dict(ld_q=Q_ROW + 3), dict(ld_qkv=1 << 50),
    dict(rot=-8), dict(rot=12), dict(rot=136), dict(layout=2), dict(cos=None), dict(sin=None), dict(cos=TAB + 4), dict(n_pos=0),
    dict(q_gain=TAB, eps=-1.0), dict(k_gain=TAB, eps=math.nan), dict(q_gain=TAB + 4), dict(q_out=Q + 16), dict(q_out=Q, ld_q=Q_ROW),
    dict(q_out=Q + 4 * Q_ROW, ld_q=KV_ROW), dict(q_out=P + 1024), dict(qkv=P + 1024)], ids=str)
def test_rope_append_refusals(bad):
    assert rope(**bad) == sb.EINVAL


@pytest.mark.parametrize("bad", [
    dict(layer=-1), dict(x_dtype=7), dict(n_heads=0), dict(n_heads=20), dict(q=None), dict(out=None), dict(q=Q + 2), dict(out=OUT + 8),
    dict(ld_q=Q_ROW - 8), dict(ld_q=Q_ROW + 4), dict(ld_out=Q_ROW + 1), dict(out=Q + 16), dict(out=Q, ld_out=2 * Q_ROW), dict(out=P),
    dict(rule=B.sb_attn_rule(scale=-1.0)), dict(rule=B.sb_attn_rule(scale=math.nan)), dict(rule=B.sb_attn_rule(scale=math.inf)),
    dict(rule=B.sb_attn_rule(softcap=-1.0)), dict(rule=B.sb_attn_rule(softcap=math.inf)), dict(rule=B.sb_attn_rule(window=-1)),
    dict(rule=B.sb_attn_rule(slopes=TAB + 2)), dict(rule=B.sb_attn_rule(prefix_len=TAB + 1)), dict(rule=B.sb_attn_rule(doc_start=TAB + 3))],
    ids=lambda d: str({k: [getattr(v, f) for f, _ in v._fields_] if k == "rule" else v for k, v in d.items()}))
def test_paged_attention_refusals(bad):
    assert attention(**bad) == sb.EINVAL


@pytest.mark.parametrize("rule", [dict(softcap=2e30), dict(scale=4.0, softcap=1e-6), dict(scale=1e-20, softcap=1e15), dict(scale=2e38)], ids=str)
def test_paged_attention_refuses_caps_that_floats_cannot_hold(rule):
    """cap tanh(scale q.k / cap) needs scale / cap and log2(e) cap."""
    assert attention(rule=B.sb_attn_rule(**rule)) == sb.EINVAL


def test_paged_attention_scratch_refusals():
    kv = paged(max_len=16 * 4096, table_ld=4096)   # (long enough that the keys are split)
    n = sb.lib().sb_op_paged_attention_scratch_bytes(C.byref(kv), 32)
    if n:
        assert attention(kv, scratch=None) == sb.EINVAL
        assert attention(kv, scratch=SCRATCH + 16) == sb.EINVAL
        assert attention(kv, n=n - 1) == sb.ENOMEM
        assert attention(kv, scratch=Q) == sb.EINVAL
        assert attention(kv, scratch=OUT) == sb.EINVAL
        assert attention(kv, scratch=P) == sb.EINVAL
    assert sb.lib().sb_op_paged_attention_scratch_bytes(C.byref(paged(head_dim=80)), 32) == 0


def test_nothing_to_do_is_done():
    for kv in (paged(n_rows=0, pool=None, table=None, row_start=None, kv_len=None), paged(n_seq=0, table=None, kv_len=None)):
        assert rope(kv, qkv=None, q_out=None) == sb.OK
        assert attention(kv, q=None, out=None, scratch=None, n=0) == sb.OK
        assert sb.lib().sb_op_paged_attention_scratch_bytes(C.byref(kv), 32) == 0


def copy(dst=P, dn=8, src=Q, sn=9, page=1024, slabs=4, to=(0, 1), frm=(3, 3), n=None):
    t, f = np.array(to, dtype=np.int32), np.array(frm, dtype=np.int32)
    return sb.lib().sb_op_copy_pages(dst, dn, src, sn, page, slabs, t.ctypes.data, f.ctypes.data, len(to) if n is None else n, None)


@pytest.mark.parametrize("bad", [
    dict(dn=0), dict(sn=0), dict(slabs=0), dict(slabs=70000), dict(n=-1), dict(page=8), dict(page=24), dict(dst=None), dict(src=None),
    dict(dst=P + 8), dict(src=Q + 4), dict(to=(0, 8)), dict(to=(-1, 1)), dict(frm=(0, 9)), dict(frm=(-1, 2)), dict(to=(2, 2)),
    dict(src=P + 1024), dict(src=P, sn=9), dict(src=P, sn=8, to=(0, 1), frm=(1, 2)), dict(src=P, sn=8, to=(0, 1), frm=(5, 0)),
    dict(src=P, sn=8, to=(4, 1), frm=(4, 2)), dict(to=tuple(range(8)) + (0,), frm=(1,) * 9)], ids=str)
def test_copy_pages_refusals(bad):
    assert copy(**bad) == sb.EINVAL


def test_copy_pages_refuses_pages_of_more_than_a_launch_counts():
    assert copy(page=(1 << 27) + 16, dn=1, sn=1, slabs=1, src=P + (1 << 40), to=(0,), frm=(0,)) == sb.EINVAL


def test_page_lists_that_32_bits_cannot_hold():
    p = sb.Pages(4)
    p.alloc(4)
    for bad in ([1 << 32], np.array([(1 << 32) + 1]), np.array([-(1 << 40)])):
        with pytest.raises(ValueError):
            p.share(bad)
    for bad in ([1.0], np.array([0.5])):
        with pytest.raises(TypeError):
            p.release(bad)
    p.share(np.array([2, 3], dtype=np.int64))
    p.share([])
    assert [p.users(i) for i in range(4)] == [1, 1, 2, 2]


def test_copy_of_no_pages_is_done():
    assert copy(to=(), frm=()) == sb.OK


def test_fork_session_refusals():
    assert sb.lib().sb_fork_session(None, None) == sb.EINVAL


# ---------------------------------------------------------------- bookkeeping
def test_pages_are_handed_out_shared_and_freed():
    p = sb.Pages(6)
    a, b = p.alloc(3), p.alloc(2)
    assert a.tolist() == [0, 1, 2] and b.tolist() == [3, 4] and p.used() == 5
    with pytest.raises(sb.SbError) as e:
        p.alloc(2)
    assert e.value.code == sb.ECAPACITY and p.used() == 5
    p.share(a[:2])
    p.release(a)
    assert [p.users(i) for i in range(6)] == [1, 1, 0, 1, 1, 0] and p.used() == 4
    assert p.alloc(2).tolist() == [2, 5]
    assert p.alloc(0).tolist() == []


def test_a_failing_call_changes_nothing():
    p = sb.Pages(4)
    p.alloc(3)
    p.share([1])
    before = [p.users(i) for i in range(4)]
    for bad in ([0, 0], [1, 1, 1], [0, 3], [0, 4], [-1], [2, 1, 0, 2]):
        with pytest.raises(sb.SbError) as e:
            p.release(bad)
        assert e.value.code == sb.EINVAL
        assert [p.users(i) for i in range(4)] == before and p.used() == 3
    for bad in ([0, 3], [4], [-2]):
        with pytest.raises(sb.SbError):
            p.share(bad)
        assert [p.users(i) for i in range(4)] == before
    p.release([1, 1, 0, 2])   # as often as they are used
    assert p.used() == 0
    for bad in (-1, 4):
        with pytest.raises(sb.SbError):
            p.users(bad)
    with pytest.raises(sb.SbError):
        p.alloc(-1)
    with pytest.raises(sb.SbError):
        sb.Pages(0)


@pytest.mark.parametrize("seed", range(8))
def test_compaction_against_a_plain_model(seed):
    r = np.random.default_rng(seed)
    n = int(r.integers(1, 60))
    p = sb.Pages(n)
    users = {int(x): 1 for x in p.alloc(int(r.integers(0, n + 1)))}
    for x in list(users):
        if r.random() < 0.5:
            p.release([x])
            del users[x]
        elif r.random() < 0.4:
            p.share([x, x])
            users[x] += 2
    src, dst = p.compact()
    live = len(users)
    assert sorted(src.tolist()) == sorted(x for x in users if x >= live)
    assert len(set(dst.tolist())) == len(dst) and all(d < live and d not in users for d in dst.tolist())
    move = dict(zip(src.tolist(), dst.tolist()))
    after = {move.get(x, x): u for x, u in users.items()}
    assert [p.users(i) for i in range(n)] == [after.get(i, 0) for i in range(n)] and p.used() == live
    assert sorted(after) == list(range(live))
    assert p.compact()[0].size == 0


def test_compaction_without_room_says_how_many_moves():
    p = sb.Pages(5)
    p.alloc(5)
    p.release([0, 2])
    n, buf = C.c_int32(), np.zeros(5, dtype=np.int32)
    assert sb.lib().sb_pages_compact(p.h, buf.ctypes.data, buf.ctypes.data, 1, C.byref(n)) == sb.ECAPACITY and n.value == 2
    assert [p.users(i) for i in range(5)] == [0, 1, 0, 1, 1]
    assert sb.lib().sb_pages_compact(p.h, None, None, 2, C.byref(n)) == sb.EINVAL
    assert sb.lib().sb_pages_compact(p.h, buf.ctypes.data, buf.ctypes.data, 5, None) == sb.EINVAL


# ---------------------------------------------------------------- rotary tables
def freq(rot, base, kind, factor, orig, slow, fast):
    i = np.arange(rot // 2, dtype=np.float64)
    b = np.float64(np.float32(base))
    if kind == sb.ROPE_BASE:
        b = b * factor ** (rot / (rot - 2))
    f = b ** (-2 * i / rot)
    if kind == sb.ROPE_LINEAR:
        f = f / factor
    if kind == sb.ROPE_PARTS:
        t = np.clip((orig * f / (2 * np.pi) - slow) / (fast - slow), 0, 1)
        f = (1 - t) * f / factor + t * f
    return f


@pytest.mark.parametrize("rot,base", [(128, 500000.0), (64, 10000.0), (24, 10000.0), (4, 100.0)])
@pytest.mark.parametrize("kind,factor,mag", [(sb.ROPE_PLAIN, 1.0, 1.0), (sb.ROPE_LINEAR, 4.0, 1.0), (sb.ROPE_BASE, 8.0, 1.0),
                                             (sb.ROPE_PARTS, 8.0, 1.25), (sb.ROPE_PARTS, 1.0, 1.0)])
def test_scaled_rope_tables(rot, base, kind, factor, mag):
    n = 3001
    c, s = sb.rope_table_scaled(rot, base, n, kind, factor, 1024, 1.0, 32.0, mag)
    a = np.arange(n)[:, None] * freq(rot, base, kind, factor, 1024, 1.0, 32.0)[None]
    # the angle's own error is some 2^-52 of 3000, the rounding to float half a step of a value up to `mag`
    tol = mag * (2.0 ** -24 + 3000 * 2.0 ** -50)
    assert np.abs(c - np.cos(a) * mag).max() <= tol and np.abs(s - np.sin(a) * mag).max() <= tol


def test_a_plain_scaled_table_is_the_plain_table():
    for a, b in zip(sb.rope_table_scaled(64, 10000.0, 500), sb.rope_table(64, 10000.0, 500)):
        assert np.array_equal(a, b)
    c, _ = sb.rope_table_scaled(64, 10000.0, 0)
    assert c.shape == (0, 32)


@pytest.mark.parametrize("bad", [dict(rot_dim=3), dict(rot_dim=0), dict(base=0.0), dict(kind=4), dict(kind=-1), dict(magnitude=0.0), dict(factor=0.5, kind=1),
                                 dict(factor=math.nan, kind=2), dict(kind=2, factor=2.0, rot_dim=2), dict(kind=3, factor=2.0, orig_len=0),
                                 dict(kind=3, factor=2.0, orig_len=64, slow=4.0, fast=4.0), dict(kind=3, factor=2.0, orig_len=64, slow=-1.0)], ids=str)
def test_scaled_rope_table_refusals(bad):
    a = dict(rot_dim=64, base=10000.0, n_pos=4)
    a.update(bad)
    with pytest.raises(sb.SbError) as e:
        sb.rope_table_scaled(**a)
    assert e.value.code == sb.EINVAL
