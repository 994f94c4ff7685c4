"""Chunks of new tokens over the paged cache: pages and slots, norms with the
rotation and the cache write, and the attention, each against the 64-bit oracle
(GPU), and what each refuses (no GPU: nothing is launched)."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import chunk as C
from paper_2607_18839_gb300 import build as B
from paper_2607_18839_gb300 import hpd as H

gpu = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module")
def lib():
    B.build()
    return H.load()


@pytest.fixture(scope="module")
def torch(lib):
    t = pytest.importorskip("torch")
    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    return t


# ---------------------------------------------------------------- refusals --

SLOT_PTRS = ("new_len", "seq_len", "page_table", "free_pages", "free_top", "seq_len_out", "free_top_out",
             "chunk_cu", "slot")
ROPE_PTRS = ("q", "k", "v", "rope", "pos", "slot", "q_out", "k_cache", "v_cache")
ATTN_PTRS = ("q", "chunk_cu", "seq_len", "k_cache", "v_cache", "page_table", "out")


def _struct(kind, ptrs, base, kw):
    a = kind()
    for p in ptrs:
        setattr(a, p, 4096)
    a.workspace = 4096
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def slot_args(**kw):
    return _struct(H.hpd_chunk_slots_args, SLOT_PTRS, dict(S=4, max_pages=8, num_pages=32, max_tokens=64), kw)


def rope_args(axis=None, **kw):
    a = _struct(H.hpd_qk_norm_rope_args, ROPE_PTRS,
                dict(T=4, H_q=8, H_kv=2, D=64, n_axes=1, max_pos=32, num_slots=64, eps=1e-6, q_stride=768,
                     k_stride=768, v_stride=768), kw)
    for i, x in (axis or {}).items():
        a.axis[i] = x
    return a


def attn_args(**kw):
    return _struct(H.hpd_chunk_attn_args, ATTN_PTRS,
                   dict(S=4, T=64, H_q=8, H_kv=2, D=64, num_pages=32, max_pages=8, workspace_bytes=1 << 30), kw)


@pytest.mark.parametrize("call,make,ptrs", [("hpd_chunk_slots", slot_args, SLOT_PTRS),
                                            ("hpd_qk_norm_rope", rope_args, ROPE_PTRS),
                                            ("hpd_chunk_attn", attn_args, ATTN_PTRS)])
def test_missing_pointers_and_workspaces_are_refused(lib, call, make, ptrs):
    for p in ptrs:
        with pytest.raises(H.HpdError) as e:
            getattr(H, call)(make(**{p: None}), None)
        assert e.value.status == 1, p
        with pytest.raises(H.HpdError) as e:
            getattr(H, call)(make(**{p: 4097}), None)  # no type is that narrow
        assert e.value.status == 1, p
    for bad in (None, 4096 + 16):
        with pytest.raises(H.HpdError) as e:
            getattr(H, call)(make(workspace=bad), None)
        assert e.value.status == 3


@pytest.mark.parametrize("bad,status", [
    (dict(S=0), 1), (dict(S=16385), 2), (dict(max_pages=0), 1), (dict(num_pages=0), 1), (dict(max_tokens=0), 1),
    (dict(max_pages=1 << 28), 2), (dict(num_pages=1 << 28), 2), (dict(pos=4098), 1)])
def test_slots_refuses(lib, bad, status):
    with pytest.raises(H.HpdError) as e:
        H.hpd_chunk_slots(slot_args(**bad), None)
    assert e.value.status == status


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), 1), (dict(H_q=0), 1), (dict(H_kv=0), 1), (dict(D=96), 2), (dict(n_axes=0), 1), (dict(n_axes=5), 1),
    (dict(max_pos=0), 1), (dict(num_slots=0), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
    (dict(eps=float("inf")), 1), (dict(q_stride=772), 1), (dict(v_stride=4), 1), (dict(q_weight=4104), 1),
    (dict(axis={31: 1}), 1), (dict(axis={0: 2}, n_axes=2), 1)])
def test_norm_rope_refuses(lib, bad, status):
    with pytest.raises(H.HpdError) as e:
        H.hpd_qk_norm_rope(rope_args(**bad), None)
    assert e.value.status == status


@pytest.mark.parametrize("bad,status", [
    (dict(S=0), 1), (dict(T=0), 1), (dict(H_q=9), 1), (dict(H_q=34), 2), (dict(D=32), 2), (dict(num_pages=0), 1),
    (dict(max_pages=0), 1), (dict(max_seq_len=-1), 1), (dict(scale=float("inf")), 1), (dict(q_stride=516), 1),
    (dict(q_stride=256), 1), (dict(max_pages=1 << 27), 2), (dict(workspace_bytes=255), 3), (dict(lse=4098), 1),
    (dict(full_len=4098), 1)])
def test_attn_refuses(lib, bad, status):
    a = attn_args(**bad)
    with pytest.raises(H.HpdError) as e:
        H.hpd_chunk_attn(a, None)
    assert e.value.status == status
    if status != 3 and not ({"lse", "full_len"} & set(bad)):
        assert H.hpd_chunk_attn_workspace_size(a) == 0


@pytest.mark.parametrize("S,H_q,H_kv,D,max_pages", [(4, 32, 8, 128, 1024), (1, 16, 2, 64, 64), (300, 8, 8, 128, 512),
                                                    (64, 40, 8, 128, 30), (2, 8, 1, 128, 3)])
def test_attn_workspace_serves_calls_of_fewer_rows(lib, S, H_q, H_kv, D, max_pages):
    size = [H.hpd_chunk_attn_workspace_size(attn_args(S=S, T=T, H_q=H_q, H_kv=H_kv, D=D, max_pages=max_pages,
                                                      num_pages=4096)) for T in range(1, 5000, 7)]
    assert all(0 < a <= b for a, b in zip(size, size[1:]))


def test_struct_layouts_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("hpd_chunk_slots_args", "hpd_qk_norm_rope_args", "hpd_chunk_attn_args")
    body = ""
    for n in names:
        body += f'  printf("%zu", sizeof({n}));\n'
        for f, _ in getattr(H, n)._fields_:
            body += f'  printf(" %zu", offsetof({n}, {f}));\n'
        body += '  printf("\\n");\n'
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hpd.h"\nint main(void) {\n' + body +
                   "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    lines = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.strip().split("\n")
    for n, line in zip(names, lines):
        k = getattr(H, n)
        assert [int(x) for x in line.split()] == [ctypes.sizeof(k)] + [getattr(k, f).offset for f, _ in k._fields_]


@gpu
def test_tensors_of_the_wrong_kind_are_refused(torch):
    i32 = lambda *a: torch.zeros(*a, dtype=torch.int32, device="cuda")  # noqa: E731
    bf = lambda *a: torch.zeros(*a, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    sl = H.ChunkSlots(i32(2, 4), i32(2), i32(8), i32(1), max_tokens=8)
    rope = H.QkNormRope(4, 2, 64, None, None, H.rope_table(8, 64))
    at = H.ChunkAttn(4, bf(8, 16, 2, 64), bf(8, 16, 2, 64), i32(2, 4), max_tokens=8)
    for bad in (lambda: sl(i32(3)), lambda: sl(i32(2).long()), lambda: sl(i32(2).cpu()),
                lambda: rope(bf(4, 511), i32(4), i32(4), bf(8, 16, 2, 64), bf(8, 16, 2, 64)),
                lambda: rope(bf(4, 512), i32(3), i32(4), bf(8, 16, 2, 64), bf(8, 16, 2, 64)),
                lambda: rope(bf(4, 512), i32(4), i32(3), bf(8, 16, 2, 64), bf(8, 16, 2, 64)),
                lambda: rope(bf(4, 512), i32(4), i32(4), bf(8, 16, 3, 64), bf(8, 16, 3, 64)),
                lambda: rope(bf(512, 4).T, i32(4), i32(4), bf(8, 16, 2, 64), bf(8, 16, 2, 64)),
                lambda: H.QkNormRope(4, 2, 64, None, None, H.rope_table(8, 64), sections=(8, 8)),
                lambda: H.QkNormRope(4, 2, 64, bf(32), None, H.rope_table(8, 64)),
                lambda: at(bf(9, 4, 64), i32(3), i32(2)), lambda: at(bf(8, 4, 128), i32(3), i32(2)),
                lambda: at(bf(8, 4, 64).float(), i32(3), i32(2)), lambda: at(bf(8, 4, 64), i32(2), i32(2)),
                lambda: at(bf(8, 4, 64), i32(3), i32(2), i32(1)), lambda: at(bf(4, 8, 64).transpose(0, 1), i32(3), i32(2))):
        with pytest.raises(H.HpdError) as e:
            bad()
        assert e.value.status == 1


# ------------------------------------------------------------ pages and slots --

def _slot_case(new_len, seq_len, max_pages, extra, seed, top=None):
    rng = np.random.default_rng(seed)
    new_len, seq_len = np.asarray(new_len, np.int64), np.asarray(seq_len, np.int64)
    held = [C.pages_of(max(l, 0)) if l <= max_pages * PAGE else 0 for l in seq_len]
    need = [max(0, C.pages_of(l + n) - h) for l, n, h in zip(seq_len, new_len, held)]
    num_pages = sum(held) + sum(need) + extra
    ids = rng.permutation(num_pages).astype(np.int32)
    table = np.full((len(new_len), max_pages), -1, np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = ids[at: at + h]
        at += h
    free = np.concatenate((ids[at:], rng.integers(0, num_pages, at).astype(np.int32)))
    return dict(new_len=new_len.astype(np.int32), seq_len=seq_len.astype(np.int32), page_table=table, free=free,
                top=num_pages - at if top is None else top)


def _run_slots(torch, c, max_tokens, in_place):
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    ins = dict(page_table=t(c["page_table"]), seq_len=t(c["seq_len"]), free_pages=t(c["free"]),
               free_top=t(np.array([c["top"]], np.int32)))
    op = H.ChunkSlots(*ins.values(), max_tokens=max_tokens, in_place=in_place)
    for x in (op.slot, op.pos, op.chunk_cu):
        x.fill_(12345)
    op(t(c["new_len"]))
    torch.cuda.synchronize()
    if not in_place:
        assert np.array_equal(ins["seq_len"].cpu().numpy(), c["seq_len"])
        assert int(ins["free_top"]) == c["top"]
    got = {k: getattr(op, k).cpu().numpy() for k in ("chunk_cu", "slot", "pos", "seq_len", "page_table")}
    got["free_top"] = int(op.free_top)
    assert np.array_equal(ins["free_pages"].cpu().numpy(), c["free"])
    return op, got


def _check_slots(torch, c, max_tokens, err=0):
    for in_place in (False, True):
        ref, e = C.slots(c["new_len"], c["seq_len"], c["page_table"], c["free"], c["top"], max_tokens)
        assert e == err
        op, got = _run_slots(torch, c, max_tokens, in_place)
        assert op.errors() == err
        for k, v in ref.items():
            assert np.array_equal(got[k], v), k


def _random_lengths(S, hi_new, hi_ctx, seed):
    rng = np.random.default_rng(seed)
    new = np.where(rng.random(S) < 0.4, rng.integers(0, 2, S), rng.integers(0, hi_new + 1, S))
    return new, rng.integers(0, hi_ctx + 1, S)


@gpu
@pytest.mark.parametrize("S,hi_new,hi_ctx,spare", [
    (1, 1, 0, 0), (1, 40, 15, 3), (4, 33, 100, 0), (31, 16, 17, 5), (33, 3, 60, 1), (511, 50, 200, 2),
    (512, 9, 40, 0), (513, 100, 300, 7), (2000, 40, 90, 1), (4500, 3, 20, 11), (16384, 2, 33, 0), (3, 5000, 900, 2)])
def test_gpu_slots(torch, S, hi_new, hi_ctx, spare):
    new, ctx = _random_lengths(S, hi_new, hi_ctx, seed=S)
    c = _slot_case(new, ctx, -(-(hi_new + hi_ctx) // PAGE) + 1, extra=4, seed=S + 1)
    _check_slots(torch, c, max(1, int(new.sum()) + spare))


@gpu
def test_gpu_slots_of_no_new_tokens_and_of_the_last_free_page(torch):
    _check_slots(torch, _slot_case([0, 0, 0], [0, 16, 5], 4, extra=0, seed=1), 4)
    _check_slots(torch, _slot_case([64, 0, 1], [0, 64, 63], 4, extra=0, seed=2), 65)


@gpu
@pytest.mark.parametrize("new,ctx,tokens,top,err", [
    ([4, -1, 3], [5, 6, 7], 64, None, C.ERR_LEN), ([4, 1, 3], [5, -6, 7], 64, None, C.ERR_LEN),
    ([4, 40, 3], [5, 30, 7], 64, None, C.ERR_LEN), ([4, 2 ** 31 - 1, 3], [5, 3, 7], 64, None, C.ERR_LEN),
    ([40, 20, 5], [5, 6, 7], 64, None, C.ERR_CAP), ([20, 20, 20], [5, 6, 7], 64, 3, 0),
    ([20, 20, 20], [5, 6, 7], 64, 2, C.ERR_POOL),
    ([20, 20, 20], [5, 6, 7], 64, -1, C.ERR_POOL), ([20, 20, 20], [5, 6, 7], 64, 1000, C.ERR_POOL)])
def test_gpu_slots_all_or_nothing(torch, new, ctx, tokens, top, err):
    c = _slot_case(np.clip(new, -1, 60), np.clip(ctx, 0, 64), 4, extra=9, seed=3, top=top)
    c["new_len"], c["seq_len"] = np.array(new, np.int32), np.array(ctx, np.int32)
    _check_slots(torch, c, tokens, err)


@gpu
def test_gpu_slots_totals_beyond_32_bits_are_refused(torch):
    # 200 sequences of 2^27 - 16 new tokens: their sum passes 2^32
    S, mp = 200, (1 << 27) // PAGE
    i32 = lambda *a: torch.zeros(*a, dtype=torch.int32, device="cuda")  # noqa: E731
    op = H.ChunkSlots(i32(1, 1), i32(1), i32(8), i32(1), max_tokens=32)
    # (the table of such sequences is never touched: only its width is stated)
    op.args.S, op.args.max_pages = S, mp
    new, old, cu = torch.full((S,), mp * PAGE - PAGE, dtype=torch.int32, device="cuda"), i32(S), i32(S + 1)
    op.args.seq_len = op.args.seq_len_out = old.data_ptr()
    op.args.chunk_cu = cu.data_ptr()
    op(new)
    torch.cuda.synchronize()
    assert op.errors() == C.ERR_CAP and int(op.slot.max()) == -1 and int(old.abs().max()) == 0


@gpu
def test_gpu_slots_flags_page_ids_out_of_range(torch):
    c = _slot_case([3, 20], [5, 0], 4, extra=2, seed=4)
    c["page_table"][0, 0] = 1 << 20
    c["free"][c["top"] - 1] = -7  # the last page taken
    op, got = _run_slots(torch, c, 32, in_place=False)
    assert op.errors() == 0x8
    assert list(got["slot"][:3]) == [-1, -1, -1] and (got["slot"][3:19] >= 0).all()
    assert (got["slot"][19:23] == -1).all()


@gpu
def test_gpu_slots_step_after_step(torch):
    """Several steps in place, the state carried on the device."""
    rng = np.random.default_rng(5)
    c = _slot_case(np.zeros(40, int), rng.integers(0, 50, 40), 40, extra=1500, seed=6)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    op = H.ChunkSlots(t(c["page_table"]), t(c["seq_len"]), t(c["free"]), t(np.array([c["top"]], np.int32)), 2400)
    st = dict(page_table=c["page_table"], seq_len=c["seq_len"], free_top=c["top"])
    for _ in range(6):
        new = rng.integers(0, 60, 40).astype(np.int32)
        st, e = C.slots(new, st["seq_len"], st["page_table"], c["free"], st["free_top"], 2400)
        assert e == 0
        op(t(new))
        torch.cuda.synchronize()
        for k in ("chunk_cu", "slot", "pos", "seq_len", "page_table"):
            assert np.array_equal(getattr(op, k).cpu().numpy(), st[k]), k
        assert int(op.free_top) == st["free_top"] and op.errors() == 0


# --------------------------------------------------- norms, rotation, write --

def _bf(torch, rng, *shape, std=1.0):
    x = torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).cuda()
    return x.to(torch.bfloat16)


def _np(x):
    return x.float().cpu().numpy()


def _run_rope(torch, T, hq, hkv, D, axes, pad, seed, weights=True, std=1.0, axis=None, neg=0):
    rng = np.random.default_rng(seed)
    qkv = _bf(torch, rng, T, (hq + 2 * hkv) * D + pad, std=std)
    qw, kw = (_bf(torch, rng, D) for _ in range(2)) if weights else (None, None)
    max_pos = 500
    table = H.rope_table(max_pos, D, 1e4)
    pos = rng.integers(0, max_pos, (axes, T)).astype(np.int32)
    pages = T // PAGE + 3
    slot = rng.permutation(pages * PAGE)[:T].astype(np.int32)
    if neg:
        slot[rng.permutation(T)[:neg]] = -1
    kc, vc = _bf(torch, rng, pages, PAGE, hkv, D), _bf(torch, rng, pages, PAGE, hkv, D)
    if axis is None:
        axis = list(rng.integers(0, axes, D // 2)) if axes > 1 else [0] * (D // 2)
        axis[0] = axes - 1
    kref, vref = _np(kc).reshape(-1, hkv, D).astype(np.float64), _np(vc).reshape(-1, hkv, D)
    op = H.QkNormRope(hq, hkv, D, qw, kw, table, axis=[int(a) for a in axis])
    p = torch.from_numpy(pos).cuda()
    q = op(qkv, p[0].contiguous() if axes == 1 else p, torch.from_numpy(slot).cuda(), kc, vc)
    torch.cuda.synchronize()
    assert op.errors() == 0
    x = _np(qkv)[:, : (hq + 2 * hkv) * D].reshape(T, -1, D)
    tab = table.cpu().numpy().astype(np.float64)
    rot = tab[pos[np.array(axis)].T, np.arange(D // 2)]
    w = [None if a is None else _np(a) for a in (qw, kw)]
    qr, qs = C.norm_rope(x[:, :hq], w[0], rot[..., 0], rot[..., 1], 1e-6)
    kr, ks = C.norm_rope(x[:, hq: hq + hkv], w[1], rot[..., 0], rot[..., 1], 1e-6)
    # one rounding to bf16 (2^-8 of the value at most), and 32-bit arithmetic:
    # a sum of D squares, a root and some six products, of 2^-24 each, against
    # the size of the two terms of a rotated value
    near = lambda got, ref, size: np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * size + 1e-30  # noqa: E731
    assert near(_np(q), qr, qs).all()
    on = slot >= 0
    kgot, vgot = _np(kc).reshape(-1, hkv, D), _np(vc).reshape(-1, hkv, D)
    assert near(kgot[slot[on]], kr[on], ks[on]).all()
    assert np.array_equal(vgot[slot[on]], x[on][:, hq + hkv:])
    rest = np.setdiff1d(np.arange(pages * PAGE), slot[on])
    assert np.array_equal(kgot[rest], kref[rest]) and np.array_equal(vgot[rest], vref[rest])
    return q


@gpu
@pytest.mark.parametrize("T,hq,hkv,D,axes,pad,weights", [
    (1, 8, 2, 64, 1, 0, True), (1, 1, 1, 128, 1, 0, False), (7, 16, 2, 128, 1, 8, True), (64, 16, 2, 128, 3, 0, True),
    (65, 5, 1, 64, 2, 24, True), (130, 40, 8, 128, 3, 64, True), (33, 14, 2, 64, 4, 0, False), (300, 3, 3, 128, 1, 0, True),
    (1000, 32, 8, 128, 3, 0, True), (2049, 16, 4, 64, 1, 40, True), (3, 128, 16, 128, 1, 0, True)])
def test_gpu_norm_rope(torch, T, hq, hkv, D, axes, pad, weights):
    _run_rope(torch, T, hq, hkv, D, axes, pad, seed=T + hq, weights=weights)


@gpu
def test_gpu_norm_rope_extremes(torch):
    _run_rope(torch, 40, 8, 2, 128, 1, 0, seed=1, std=1e-5)   # eps of the size of the squares
    _run_rope(torch, 40, 8, 2, 64, 1, 0, seed=2, std=1e15)    # squares sum to 1e32
    _run_rope(torch, 50, 8, 2, 128, 1, 0, seed=3, neg=20)     # rows that are padding
    # sections of whole groups of frequencies, and of parts of them
    _run_rope(torch, 20, 4, 2, 128, 3, 0, seed=4, axis=[0] * 16 + [1] * 24 + [2] * 24)
    _run_rope(torch, 20, 4, 2, 128, 3, 0, seed=5, axis=[0] * 21 + [1] * 21 + [2] * 22)


@gpu
def test_gpu_norm_rope_of_a_zero_row_in_place_and_out_of_range(torch):
    rng = np.random.default_rng(6)
    D, table = 64, H.rope_table(16, 64)
    qkv = _bf(torch, rng, 3, 6 * D)
    qkv[1] = 0
    kc, vc = _bf(torch, rng, 2, PAGE, 1, D), _bf(torch, rng, 2, PAGE, 1, D)
    op = H.QkNormRope(4, 1, D, None, None, table)
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q = op(qkv, i(1, 2, 3), i(0, 1, 2), kc, vc)
    torch.cuda.synchronize()
    assert float(q[1].float().abs().max()) == 0.0 and op.errors() == 0
    before = kc.clone()
    op(qkv, i(1, 2, 3), i(3, 32, -5), kc, vc)  # row 32 is past the cache
    torch.cuda.synchronize()
    assert op.errors() == 0x8 and torch.equal(kc.view(-1, D)[4:], before.view(-1, D)[4:])
    op.workspace.zero_()
    a = op(qkv, i(-3, 2, 99), i(-1, -1, -1), kc, vc).clone()
    b = op(qkv, i(0, 2, 15), i(-1, -1, -1), kc, vc)
    torch.cuda.synchronize()
    assert op.errors() == 0x400 and torch.equal(a, b)
    # queries rotated where they are: rows of queries alone
    x = qkv[:, : 4 * D].contiguous()
    op.args.q = op.args.q_out = x.data_ptr()
    op.args.q_stride = 4 * D
    op.args.pos = (p := i(0, 2, 15)).data_ptr()
    H.hpd_qk_norm_rope(op.args, H._stream_handle(None))
    torch.cuda.synchronize()
    assert torch.equal(x.view(3, 4, D), b) and p is not None


# ---------------------------------------------------------------- attention --

def _attn_case(torch, new, total, hq, hkv, D, seed, full=None, spare_rows=0, pad_q=0, std=1.0, scale=0.0,
               stale=float("nan"), max_pages=None, max_seq_len=0):
    rng = np.random.default_rng(seed)
    new, total = np.asarray(new), np.asarray(total)
    pages = [C.pages_of(l) for l in total]
    num_pages = sum(pages) + 2
    ids = rng.permutation(num_pages).astype(np.int32)
    mp = max_pages or max(1, max(pages))
    table = np.full((len(new), mp), -1, np.int32)
    at = 0
    for s, h in enumerate(pages):
        table[s, :h] = ids[at: at + h]
        at += h
    T = int(new.sum()) + spare_rows
    kc, vc = _bf(torch, rng, num_pages, PAGE, hkv, D, std=std), _bf(torch, rng, num_pages, PAGE, hkv, D)
    # whatever no sequence holds may be anything
    held = np.zeros((num_pages, PAGE), bool)
    for s, l in enumerate(total):
        for j in range(int(l)):
            held[table[s, j // PAGE], j % PAGE] = True
    off = torch.from_numpy(~held).cuda()
    kc[off] = stale
    vc[off] = stale
    q = _bf(torch, rng, max(T, 1), hq * D + pad_q, std=std)
    q = q[:, : hq * D].unflatten(1, (hq, D))
    cu = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    return dict(q=q, kc=kc, vc=vc, table=t(table), cu=t(cu), total=t(total), full=None if full is None else t(full),
                scale=scale, max_seq_len=max_seq_len)


def _check_attn(torch, c, sample=None, seed=0):
    hq = c["q"].shape[1]
    op = H.ChunkAttn(hq, c["kc"], c["vc"], c["table"], max_tokens=c["q"].shape[0], max_seq_len=c["max_seq_len"],
                     scale=c["scale"])
    op.out.fill_(7.0)
    op.lse.fill_(7.0)
    out, lse = op(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    assert op.errors() == 0
    again = op(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    cu, total = c["cu"].cpu().numpy(), c["total"].cpu().numpy()
    n = int(cu[-1])
    out, lse = _np(out), lse.cpu().numpy()
    assert np.array_equal(_np(again[0]), out, equal_nan=True) and np.array_equal(again[1].cpu().numpy(), lse)
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()  # rows of no sequence
    z = np.nan_to_num
    ref, rl, size, reach = C.attn(_np(c["q"])[:n], z(_np(c["kc"])), z(_np(c["vc"])), c["table"].cpu().numpy(), cu, total,
                                  None if c["full"] is None else c["full"].cpu().numpy(), c["scale"])
    assert np.array_equal(np.isneginf(lse[:n]), np.isneginf(rl))
    fin = np.isfinite(rl)
    # scores: D products summed in 32 bits, off by some 2^-21 of the sum of their
    # sizes; lse by as much, and by the exponentials' and the log's 2^-21
    slip = 2.0 ** -20 * reach + 2.0 ** -19
    assert (np.abs(lse[:n][fin] - rl[fin]) <= slip[fin] + 2.0 ** -21 * np.abs(rl[fin])).all()
    # out: one rounding to bf16 of each weight and of the result, 2^-8 each, and
    # what the scores are off
    tol = 2.0 ** -8 * (np.abs(ref) + size) * 1.02 + 2 * slip[..., None] * size
    bad = np.abs(out[:n] - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(out[:n] - ref).max())
    return op


ATTN = [  # new, total, H_q, H_kv, D
    ([1], [1], 8, 2, 64), ([1], [256], 8, 2, 64), ([1], [129], 16, 2, 128), ([5], [5], 16, 2, 128),
    ([17], [145], 4, 4, 128), ([129], [129], 8, 8, 64), ([200], [200], 16, 1, 128), ([33], [1000], 32, 8, 128),
    ([0, 3, 1, 0, 70], [9, 3, 40, 0, 200], 16, 2, 128), ([1] * 40, list(range(1, 400, 10)), 16, 4, 64),
    ([1, 2, 130, 64], [16, 34, 130, 640], 10, 2, 128), ([40, 41], [100, 41], 6, 2, 64), ([13, 7, 1], [2000, 7, 17], 14, 2, 64),
    ([9, 22], [300, 22], 22, 2, 128), ([128, 128], [256, 128], 2, 2, 128), ([300], [1500], 40, 8, 128),
    ([1, 1, 1], [5000, 3, 800], 16, 2, 128), ([1], [9000], 8, 8, 64), ([2] * 70, [130 + i for i in range(70)], 32, 2, 64)]


@gpu
@pytest.mark.parametrize("new,total,hq,hkv,D", ATTN)
def test_gpu_attn(torch, new, total, hq, hkv, D):
    _check_attn(torch, _attn_case(torch, new, total, hq, hkv, D, seed=len(new) + hq))


@gpu
@pytest.mark.parametrize("new,total,full,hq,hkv,D", [
    ([100, 1, 30], [100, 50, 130], [64, 50, 0], 16, 2, 128), ([70, 70], [200, 70], [130, 70], 10, 2, 64),
    ([40], [40], [1000], 8, 2, 128), ([40, 3], [400, 3], [-5, 2], 8, 2, 64), ([260], [300], [129], 16, 1, 128)])
def test_gpu_attn_prefix_mask(torch, new, total, full, hq, hkv, D):
    _check_attn(torch, _attn_case(torch, new, total, hq, hkv, D, seed=9, full=full))


@gpu
def test_gpu_attn_rows_without_keys(torch):
    # more new tokens than the sequence has: the first see nothing; none at all
    _check_attn(torch, _attn_case(torch, [20, 5, 150], [7, 0, 20], 8, 2, 128, seed=3))
    _check_attn(torch, _attn_case(torch, [20, 5], [7, 0], 6, 2, 64, seed=4, spare_rows=9))
    _check_attn(torch, _attn_case(torch, [0, 0], [7, 0], 6, 2, 64, seed=5, spare_rows=3))


@gpu
def test_gpu_attn_strided_queries_scales_and_spare_rows(torch):
    _check_attn(torch, _attn_case(torch, [60, 1], [300, 90], 16, 2, 128, seed=6, pad_q=4 * 128, spare_rows=70))
    _check_attn(torch, _attn_case(torch, [60, 1], [300, 90], 16, 2, 128, seed=7, scale=0.3, max_pages=100))
    _check_attn(torch, _attn_case(torch, [60, 1], [300, 90], 16, 2, 64, seed=8, scale=-0.2, max_seq_len=300))


@gpu
def test_gpu_attn_rising_scores_and_stale_rows(torch):
    # scores that rise by hundreds along the keys, so that early weights vanish
    c = _attn_case(torch, [50, 1], [700, 650], 8, 2, 128, seed=10, stale=float("inf"))
    for s, l in ((0, 700), (1, 650)):
        row = c["table"][s].cpu().numpy()
        for j in range(l):
            c["kc"][row[j // PAGE], j % PAGE, :, 0] = j / 8.0
    c["q"][..., 0] = 16.0
    op = _check_attn(torch, c)
    # values that overflow 32 bits where weights of 2^64 meet them stay finite
    c["vc"] *= 2.0 ** 80
    out, _ = H.ChunkAttn(8, c["kc"], c["vc"], c["table"], max_tokens=51)(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out.float()).all()) and op is not None


@gpu
def test_gpu_attn_nan_among_the_keys_stays_where_it_is_seen(torch):
    c = _attn_case(torch, [40, 30], [300, 200], 8, 2, 128, seed=11)
    row = c["table"][0].cpu().numpy()
    c["kc"][row[280 // PAGE], 280 % PAGE, 1] = float("nan")  # key 280 of KV head 1: seen from token 20 on
    op = H.ChunkAttn(8, c["kc"], c["vc"], c["table"], max_tokens=70)
    out, lse = op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    nan = torch.isnan(lse).cpu().numpy()
    want = np.zeros((70, 8), bool)
    want[20:40, 4:] = True
    assert np.array_equal(nan, want)
    assert np.array_equal(torch.isnan(out.float()).any(-1).cpu().numpy(), want)


@gpu
def test_gpu_attn_flags_and_clamps_device_data(torch):
    c = _attn_case(torch, [4, 6], [40, 60], 8, 2, 64, seed=12, stale=0.0)
    good = lambda: H.ChunkAttn(8, c["kc"], c["vc"], c["table"], max_tokens=10)  # noqa: E731
    for what, bad, flag in (("total", [40, 5000], 0x4), ("total", [-3, 60], 0x4), ("cu", [0, 4, 11], 0x2),
                            ("cu", [0, 7, 3], 0x2), ("cu", [-2, 4, 10], 0x2)):
        op = good()
        args = dict(c, **{what: torch.tensor(bad, dtype=torch.int32, device="cuda")})
        op(args["q"], args["cu"], args["total"])
        torch.cuda.synchronize()
        assert op.errors() & flag, (what, bad)
    c["table"][1, 0] = 1 << 24
    op = good()
    op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0x8


@gpu
def test_gpu_attn_on_another_stream_and_in_a_graph(torch):
    c = _attn_case(torch, [30, 1, 9], [500, 77, 9], 16, 2, 128, seed=13)
    op = H.ChunkAttn(16, c["kc"], c["vc"], c["table"], max_tokens=40)
    ref = [x.clone() for x in op(c["q"], c["cu"], c["total"])]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    op.out.zero_()
    torch.cuda.synchronize()
    op(c["q"], c["cu"], c["total"], stream=s)
    s.synchronize()
    assert torch.equal(op.out, ref[0]) and torch.equal(op.lse, ref[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op(c["q"], c["cu"], c["total"])
    op.out.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(op.out, ref[0]) and torch.equal(op.lse, ref[1])


@gpu
@pytest.mark.parametrize("hq,hkv,D", [(32, 8, 128), (8, 8, 64)])
def test_gpu_attn_many_short_units_one_after_another(torch, hq, hkv, D):
    # some twenty units of one or two blocks on every SM, whose roles may be units
    # apart: every call gives the first one's bits, and those the oracle's values
    rng = np.random.default_rng(21)
    S = 3200 // hkv
    new, total = np.full(S, 2), rng.integers(2, 250, S)
    c = _attn_case(torch, new, total, hq, hkv, D, seed=14)
    op = _check_attn(torch, c)
    first = op.out.clone(), op.lse.clone()
    for _ in range(50):
        op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0
    assert torch.equal(op.out, first[0]) and torch.equal(op.lse, first[1])


@gpu
@pytest.mark.parametrize("new,total,hq,hkv,D", [
    ([700], [3000], 40, 8, 128),            # 27 x 8 units on 152 SMs: some whole, the rest split
    ([1], [20000], 32, 8, 128),             # nothing but splits
    ([640, 3], [2500, 4000], 16, 4, 64),
    ([1, 1, 1], [9000, 40, 0], 8, 2, 128),  # splits of one sequence, none of the others
    ([300, 290], [2300, 300], 16, 16, 128)])
def test_gpu_attn_split_tiles(torch, new, total, hq, hkv, D):
    c = _attn_case(torch, new, total, hq, hkv, D, seed=15)
    _check_attn(torch, c)
    # offsets out of order beside splits: flagged, in bounds
    op = H.ChunkAttn(hq, c["kc"], c["vc"], c["table"], max_tokens=c["q"].shape[0])
    if len(new) > 1:
        bad = c["cu"].clone()
        bad[1] = c["q"].shape[0] + 5
        op(c["q"], bad, c["total"])
        torch.cuda.synchronize()
        assert op.errors() & 0x2


def _near_oracle(c, rows, out, lse):
    """These rows of a call against the oracle, whatever the others hold."""
    z = np.nan_to_num
    ref, rl, size, reach = C.attn(_np(c["q"]), z(_np(c["kc"])), z(_np(c["vc"]), posinf=0.0, neginf=0.0),
                                  c["table"].cpu().numpy(), c["cu"].cpu().numpy(), c["total"].cpu().numpy(),
                                  None if c["full"] is None else c["full"].cpu().numpy(), c["scale"])
    slip = 2.0 ** -20 * reach + 2.0 ** -19  # as in _check_attn
    assert (np.abs(lse - rl)[rows] <= (slip + 2.0 ** -21 * np.abs(rl))[rows]).all()
    assert (np.abs(out - ref)[rows] <= (2.0 ** -8 * (np.abs(ref) + size) * 1.02 + 2 * slip[..., None] * size)[rows]).all()


@gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("new,total,hq,hkv,D", [([40, 30], [300, 200], 8, 2, 128), ([40, 30], [300, 200], 8, 2, 64),
                                                ([30], [6000], 8, 2, 128), ([300, 9], [700, 50], 32, 8, 128)])
def test_gpu_attn_values_not_finite_stay_where_they_are_seen(torch, value, new, total, hq, hkv, D):
    # a value in a chunk's own keys: the tokens before it share its tiles and must
    # not see it (0 times it is not 0); lse knows nothing of values
    c = _attn_case(torch, new, total, hq, hkv, D, seed=16)
    G, first = hq // hkv, 20
    at = total[0] - new[0] + first
    c["vc"][int(c["table"][0, at // PAGE]), at % PAGE, 1, 5] = value
    op = H.ChunkAttn(hq, c["kc"], c["vc"], c["table"], max_tokens=sum(new))
    out, lse = op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0
    out, lse = _np(out), lse.cpu().numpy()
    want = np.zeros(out.shape, bool)
    want[first: new[0], G: 2 * G, 5] = True
    assert np.array_equal(~np.isfinite(out), want)
    seen = want.any(-1)
    assert np.isfinite(lse).all()
    # (rows that see it: their other columns are as good as any)
    _near_oracle(c, ~seen, out, lse)
    if value != value:
        assert np.isnan(out[want]).all()
    else:
        assert (out[want] == value).all()


@gpu
def test_gpu_attn_scores_of_minus_infinity_before_the_others(torch):
    # the keys whose scores give a tile its base at minus infinity, the others so low
    # that no weight of base 0 is left: the softmax is of the others all the same
    c = _attn_case(torch, [3, 2], [400, 128], 4, 2, 128, seed=17, scale=1.0)
    c["q"].zero_()
    c["q"][..., 0] = 16.0
    for s, l in ((0, 400), (1, 128)):
        for j in range(l):
            low = (j % 128 < 32 or 64 <= j % 128 < 96) and j < 128
            page = int(c["table"][s, j // PAGE])
            c["kc"][page, j % PAGE, :, 0] = -3e38 if low else -12.5
            c["vc"][page, j % PAGE] = 1000.0 if low else 3.0
    op = H.ChunkAttn(4, c["kc"], c["vc"], c["table"], max_tokens=5, scale=1.0)
    out, lse = op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0 and bool((out == 3.0).all())
    keys = np.array([398 - 64, 399 - 64, 400 - 64, 127 - 64, 128 - 64])
    assert np.abs(lse.cpu().numpy() - (np.log(keys) - 200.0)[:, None]).max() <= 2.0 ** -12


@gpu
def test_gpu_attn_output_at_an_odd_multiple_of_16_bytes(torch):
    c = _attn_case(torch, [60, 1], [300, 2900], 16, 2, 128, seed=18)
    op = H.ChunkAttn(16, c["kc"], c["vc"], c["table"], max_tokens=61)
    want = op(c["q"], c["cu"], c["total"])[0].clone()
    room = torch.full((61 * 16 * 128 + 16,), 7.0, dtype=torch.bfloat16, device="cuda")
    op.args.out = room.data_ptr() + 16
    op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0 and torch.equal(room[8:-8].view_as(want), want)
    assert bool((room[:8] == 7.0).all()) and bool((room[-8:] == 7.0).all())


@gpu
def test_gpu_pages_beyond_32_bits_of_a_long_cache(torch):
    # rows past 2^32 values (2^33 bytes) of the pool, written by the rotation and
    # read by the attention; the same in a small pool gives the same bits
    hq, hkv, D, new, total = 16, 8, 128, [37, 5], [37, 133]
    far, pages = 264_000, sum(C.pages_of(l) for l in total)
    assert far * PAGE * hkv * D > 2 ** 32
    rng = np.random.default_rng(19)
    qkv = _bf(torch, rng, sum(new), (hq + 2 * hkv) * D)
    old = _bf(torch, rng, 2, pages, PAGE, hkv, D)
    table, i32 = H.rope_table(200, D), dict(dtype=torch.int32, device="cuda")
    got = []
    for base in (0, far):
        kc, vc = (torch.empty(base + pages, PAGE, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        kc[base:], vc[base:] = old[0], old[1]
        top = torch.tensor([pages], **i32)
        free = torch.arange(base + pages, **i32)[-pages:].flip(0).repeat(2)  # the last pages of the pool
        pt = torch.zeros(2, 9, **i32)
        pt[1, :8] = free[:8]
        slots = H.ChunkSlots(pt, torch.tensor([0, 128], **i32), free, top, max_tokens=42)
        # (ids up to the stack's size are valid to it: state the pool's)
        slots.args.num_pages = base + pages
        slots(torch.tensor(new, **i32))
        rope = H.QkNormRope(hq, hkv, D, None, None, table)
        q = rope(qkv, slots.pos, slots.slot, kc, vc)
        op = H.ChunkAttn(hq, kc, vc, pt, max_tokens=42)
        out, lse = op(q, slots.chunk_cu, slots.seq_len)
        torch.cuda.synchronize()
        assert slots.errors() == rope.errors() == op.errors() == 0
        assert int(slots.slot.min()) >= base * PAGE
        got.append((out.clone(), lse.clone(), kc[base:].clone(), vc[base:].clone()))
        del kc, vc, op
    for a, b in zip(*got):
        assert torch.equal(a, b)


@gpu
def test_gpu_norm_rope_keeps_its_output_while_it_grows(torch):
    rng = np.random.default_rng(20)
    kc, vc = (torch.zeros(8, PAGE, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    op = H.QkNormRope(4, 2, 64, None, None, H.rope_table(64, 64))
    i32 = dict(dtype=torch.int32, device="cuda")
    x = _bf(torch, rng, 40, 8 * 64)
    run = lambda n: op(x[:n], torch.arange(n, **i32), torch.arange(n, **i32), kc, vc)  # noqa: E731
    pos = torch.arange(4, **i32)
    want = run(4).clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q = op(x[:4], pos, pos, kc, vc)
    big = run(40).clone()
    q.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(q, want) and torch.equal(big[:4], want) and torch.equal(run(40), big)


# ----------------------------------------- prefill of pages, then a decode step --

@pytest.fixture(scope="module")
def example():
    import importlib.util
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                        "prefill_then_decode.py")
    spec = importlib.util.spec_from_file_location("prefill_then_decode", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@gpu
def test_gpu_prefill_in_chunks_then_decode(torch, example):
    import oracle
    from paper_2607_18839_gb300 import workloads as W
    make = lambda room: example.Pages(example.Shape(), [(5, 7), (9, 9), (1, 1)], [30, 3, 77], room)  # noqa: E731
    whole, parts = make(300), make(97)
    a, b = whole.prefill(per_step=100), parts.prefill(per_step=11)
    torch.cuda.synchronize()
    # the same hidden states, but for what two layers' roundings to bf16 make of
    # scores summed in other orders: 2^-8 of values of some units each
    for x, y, n in zip(a, b, whole.total):
        assert x.shape == (n, 256) and float((x.float() - y.float()).abs().max()) <= 8 * 2.0 ** -8 * float(x.abs().max())
    assert int(whole.top) == int(parts.top) == 64
    op = parts.branches(per_doc=3, m=4)
    d, host = op.d, lambda t: t.cpu().numpy()  # noqa: E731
    bits = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    cu, pt = host(d.prefix_cu), host(d.prefix_page_table)
    rows = [[int(pt[s, j // PAGE]) * PAGE + j % PAGE for j in range(n)] for s, n in enumerate(parts.total)]
    at = np.concatenate(rows)
    inp = W.BranchDecodeInputs(
        n_docs=3, B=9, m=4, H_q=16, H_kv=2, D=128, num_pages=d.num_pages, max_pages=d.max_pages, q=bits(d.q),
        prefix_k=bits(d.k_cache).reshape(-1, 2, 128)[at], prefix_v=bits(d.v_cache).reshape(-1, 2, 128)[at],
        prefix_cu=cu, branch_cu=host(d.branch_cu), k_cache=bits(d.k_cache), v_cache=bits(d.v_cache),
        page_table=host(d.page_table), branch_len=host(d.branch_len), branch_prefix_len=host(d.branch_prefix_len))
    ref, rl = oracle.branch_attn(inp)
    assert np.abs(_np(op.out) - ref).max() <= 1e-2 and np.abs(host(op.lse) - rl).max() <= 1e-3
    # (every branch has a page of its own)
    assert (host(d.branch_len) == 4).all() and len(set(host(d.page_table)[:, 0])) == 9


@gpu
def test_gpu_prefill_refuses_what_has_no_room(torch, example):
    pages = example.Pages(example.Shape(layers=1), [(9, 9)], [3], room=40)
    with pytest.raises(ValueError):
        pages.prefill(per_step=10)


@gpu
def test_gpu_attn_calls_of_fewer_rows_than_the_operator_was_made_for(torch):
    # 4,096 rows leave no SM idle, one row of a long context is split over all: the
    # same operator, the oracle's values
    c = _attn_case(torch, [1, 0], [3000, 9], 32, 8, 128, seed=22)
    want, lse = H.ChunkAttn(32, c["kc"], c["vc"], c["table"], max_tokens=1)(c["q"], c["cu"], c["total"])
    op = H.ChunkAttn(32, c["kc"], c["vc"], c["table"], max_tokens=4096)
    for _ in range(2):
        got = op(c["q"], c["cu"], c["total"])
        torch.cuda.synchronize()
        assert op.errors() == 0 and got[0].shape == want.shape
        assert torch.equal(got[0], want) and torch.equal(got[1], lse)
    _check_attn(torch, c)
