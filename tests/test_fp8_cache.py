"""The paged cache in 8 bits: its write with norms and rotation, and the attention
over it, against the 64-bit oracle (GPU), and what each refuses (no GPU: nothing is
launched)."""
import contextlib
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import test_chunk_ops as K
import test_chunk_ops_edges as E
from oracle import chunk as C
from oracle import fp8 as F
from paper_2607_18839_gb300 import build as B
from paper_2607_18839_gb300 import hpd as H

gpu = pytest.mark.gpu
PAGE = 16
INF, NAN = float("inf"), float("nan")
NEED_CURRENT = H._need_current


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


def test_the_oracles_codes():
    torch = pytest.importorskip("torch")
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).double().numpy(), F.VALUES, equal_nan=True)
    rng = np.random.default_rng(0)
    v = F._POSITIVE
    x = np.concatenate((F.VALUES, (v[1:] + v[:-1]) / 2, rng.standard_normal(5000) * 100, rng.standard_normal(5000) * 0.01,
                        [500.0, -1e30, 0.0, -0.0, 2.0 ** -10, 2.0 ** -11]))
    want = torch.from_numpy(np.clip(x, -448, 448)).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(F.encode(x) & np.where(np.isnan(x), 127, 255), want & np.where(np.isnan(x), 127, 255))
    assert np.array_equal(F.encode([INF, -INF, NAN]) & 127, [127] * 3)


# ---------------------------------------------------------------- refusals --

def write_args(k_scale=4096, v_scale=4096, **kw):
    f = H.hpd_qk_norm_rope_fp8_args()
    f.rope = K.rope_args(**kw)
    f.k_scale, f.v_scale = k_scale, v_scale
    return f


def attn_args(k_scale=4096, v_scale=4096, **kw):
    f = H.hpd_chunk_attn_fp8_args()
    f.attn = K.attn_args(**kw)
    f.k_scale, f.v_scale = k_scale, v_scale
    return f


@pytest.mark.parametrize("call,make,ptrs", [("hpd_qk_norm_rope_fp8", write_args, K.ROPE_PTRS + ("k_scale", "v_scale")),
                                            ("hpd_chunk_attn_fp8", attn_args, K.ATTN_PTRS + ("k_scale", "v_scale"))])
def test_missing_pointers_and_workspaces_are_refused(lib, call, make, ptrs):
    for p in ptrs:
        for bad in (None, 4097, 4098):
            with pytest.raises(H.HpdError) as e:
                getattr(H, call)(make(**{p: bad}), None)
            assert e.value.status == 1, p
    for bad in (None, 4096 + 16):
        with pytest.raises(H.HpdError) as e:
            getattr(H, call)(make(workspace=bad), None)
        assert e.value.status == 3


@pytest.mark.parametrize("bad,status", [
    (dict(T=-1), 1), (dict(H_q=0), 1), (dict(H_kv=0), 1), (dict(D=96), 2), (dict(n_axes=5), 1), (dict(max_pos=0), 1),
    (dict(num_slots=0), 1), (dict(num_slots=24), 1), (dict(eps=NAN), 1), (dict(q_stride=772), 1),
    (dict(v_stride=4), 1), (dict(axis={31: 1}), 1)])
def test_write_refuses(lib, bad, status):
    with pytest.raises(H.HpdError) as e:
        H.hpd_qk_norm_rope_fp8(write_args(**bad), None)
    assert e.value.status == status


@pytest.mark.parametrize("bad,status", [
    (dict(S=0), 1), (dict(T=0), 1), (dict(H_q=9), 1), (dict(H_q=34), 2), (dict(D=32), 2), (dict(num_pages=0), 1),
    (dict(max_seq_len=-1), 1), (dict(scale=INF), 1), (dict(q_stride=256), 1), (dict(max_pages=1 << 27), 2),
    (dict(workspace_bytes=255), 3), (dict(lse=4098), 1), (dict(full_len=4098), 1)])
def test_attn_refuses(lib, bad, status):
    f = attn_args(**bad)
    with pytest.raises(H.HpdError) as e:
        H.hpd_chunk_attn_fp8(f, None)
    assert e.value.status == status
    if status != 3 and not ({"lse", "full_len"} & set(bad)):
        assert H.hpd_chunk_attn_fp8_workspace_size(f) == 0


@pytest.mark.parametrize("S,H_q,H_kv,D,max_pages", [(4, 32, 8, 128, 1024), (1, 16, 2, 64, 64), (300, 8, 8, 128, 512),
                                                    (64, 40, 8, 128, 30), (2, 8, 1, 128, 3)])
def test_attn_workspace_serves_calls_of_fewer_rows(lib, S, H_q, H_kv, D, max_pages):
    size = [H.hpd_chunk_attn_fp8_workspace_size(attn_args(S=S, T=T, H_q=H_q, H_kv=H_kv, D=D, max_pages=max_pages,
                                                          num_pages=4096)) for T in range(1, 5000, 7)]
    assert all(0 < a <= b for a, b in zip(size, size[1:]))


def test_write_of_no_rows(lib):
    H.hpd_qk_norm_rope_fp8(write_args(T=0, q=None, k=None, v=None, pos=None, slot=None, q_out=None), None)


def test_struct_layouts_match_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names, body = ("hpd_qk_norm_rope_fp8_args", "hpd_chunk_attn_fp8_args"), ""
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


class Host(E.Host):
    """The binding on host tensors, with an 8-bit cache among them."""

    def __init__(self, torch, monkeypatch):
        super().__init__(torch, monkeypatch)
        self.f32 = lambda *n: self.of(torch.zeros(n))
        self.code = lambda *n: self.of(torch.zeros(n, dtype=torch.uint8).view(torch.float8_e4m3fn))
        monkeypatch.setattr(H, "_need_current", lambda *a: None)
        for name in ("hpd_qk_norm_rope_fp8", "hpd_chunk_attn_fp8"):
            monkeypatch.setattr(H, name, lambda args, s, name=name: self.calls.append((name, args, s)))


@pytest.fixture
def host(lib, monkeypatch):
    return Host(pytest.importorskip("torch"), monkeypatch)


def test_caches_and_scales_of_the_wrong_kind_are_refused(host):
    bf, i32, f32, code = host.bf, host.i32, host.f32, host.code
    rope, good = host.rope(), dict(k_scale=f32(8, 2), v_scale=f32(8, 2))
    put = lambda k, v, **kw: rope(bf(4, 512), i32(4), i32(4), k, v, q_out=bf(4, 4, 64), **kw)  # noqa: E731
    attn = lambda k, v, **kw: H.ChunkAttn(4, k, v, i32(2, 4), max_tokens=8, **kw)  # noqa: E731
    for call in (put, attn):
        for bad in (lambda: call(bf(8, 16, 2, 64), bf(8, 16, 2, 64), **good),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64)),
                    lambda: call(code(8, 16, 2, 64), bf(8, 16, 2, 64), **good),
                    lambda: call(code(8, 16, 2, 64), code(9, 16, 2, 64), **good),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64), k_scale=f32(8, 2)),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64), v_scale=f32(8, 2)),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64), k_scale=f32(8, 2), v_scale=f32(8, 1)),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64), k_scale=f32(7, 2), v_scale=f32(8, 2)),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64), k_scale=bf(8, 2), v_scale=f32(8, 2)),
                    lambda: call(code(8, 16, 2, 64), code(8, 16, 2, 64), k_scale=f32(2, 8).T, v_scale=f32(8, 2))):
            with pytest.raises(H.HpdError) as e:
                bad()
            assert e.value.status == 1
    host.calls.clear()
    put(code(8, 16, 2, 64), code(8, 16, 2, 64), **good)
    name, f, _ = host.calls[-1]
    assert name == "hpd_qk_norm_rope_fp8" and f.k_scale == good["k_scale"].data_ptr() and f.rope.num_slots == 128
    # and the same object on a bf16 cache again
    put(bf(8, 16, 2, 64), bf(8, 16, 2, 64))
    assert host.calls[-1][0] == "hpd_qk_norm_rope"
    op = attn(code(8, 16, 2, 64), code(8, 16, 2, 64), **good)
    op(bf(8, 4, 64), i32(3), i32(2))
    assert host.calls[-1][0] == "hpd_chunk_attn_fp8" and host.calls[-1][1].v_scale == good["v_scale"].data_ptr()


def test_every_tensor_of_another_device_is_refused(host, monkeypatch):
    torch, bf, i32, f32, code = host.torch, host.bf, host.i32, host.f32, host.code

    class Far(type(bf(1))):
        get_device = lambda self: 1  # noqa: E731

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)  # (where the host's tensors are)
    monkeypatch.setattr(H, "_need_current", NEED_CURRENT)
    rope = host.rope()
    put = dict(qkv=bf(4, 512), pos=i32(4), slot=i32(4), k_cache=code(8, 16, 2, 64), v_cache=code(8, 16, 2, 64),
               q_out=bf(4, 4, 64), k_scale=f32(8, 2), v_scale=f32(8, 2))
    op = H.ChunkAttn(4, code(8, 16, 2, 64), code(8, 16, 2, 64), i32(2, 4), max_tokens=8, k_scale=f32(8, 2), v_scale=f32(8, 2))
    attn = dict(q=bf(4, 4, 64), chunk_cu=i32(3), seq_len=i32(2), full_len=i32(2))
    for call, kw in ((rope, put), (op, attn)):
        host.calls.clear()
        call(**kw)
        assert len(host.calls) == 1
        for name in kw:
            with pytest.raises(H.HpdError) as e:
                call(**{**kw, name: kw[name].as_subclass(Far)})
            assert e.value.status == 1 and len(host.calls) == 1, name
    # and what the object was made with
    far = H.QkNormRope(4, 2, 64, None, None, host.of(torch.zeros(8, 32, 2)).as_subclass(Far))
    with pytest.raises(H.HpdError):
        far(**put)


@gpu
def test_tensors_of_another_device_are_refused(torch):
    here = torch.cuda.current_device()
    with contextlib.ExitStack() as stack:
        if torch.cuda.device_count() > 1:
            stack.enter_context(torch.cuda.device(1 - min(here, 1)))
            x = torch.zeros(2, device=f"cuda:{here}")
        else:
            x = torch.zeros(2)  # of no device at all
        with pytest.raises(H.HpdError) as e:
            H._need_current("x", x)
        assert e.value.status == 1


# ------------------------------------------------------------------ the write --

def _codes(torch, x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().view(torch.float8_e4m3fn)


def _u8(x):
    import torch
    return x.view(torch.uint8).cpu().numpy()


def _cache(torch, rng, pages, hkv, D):
    """Codes of every kind and scales, some of them wrong for what they hold."""
    code = rng.integers(0, 256, (pages, PAGE, hkv, D)).astype(np.uint8)
    code[(code & 127) == 127] = 5
    code[rng.random(code.shape) < 1e-4] = 127
    scale = (2.0 ** rng.uniform(-12, -5, (pages, hkv))).astype(np.float32)
    return _codes(torch, code), torch.from_numpy(scale).cuda()


def _slots(rng, new, ctx, extra=3):
    pages = [C.pages_of(n + c) for n, c in zip(new, ctx)]
    ids = rng.permutation(sum(pages) + extra)
    slot, at = [], 0
    for n, c, p in zip(new, ctx, pages):
        slot += [int(ids[at + j // PAGE]) * PAGE + j % PAGE for j in range(c, c + n)]
        at += p
    return np.array(slot, np.int32), sum(pages) + extra


class Write:
    """A call of the write on random rows, and its check against the oracle."""

    def __init__(self, torch, slot, pages, hq, hkv, D, axes=1, pad=0, seed=0, weights=True, std=1.0):
        self.torch, self.slot, self.hq, self.hkv, self.D = torch, slot, hq, hkv, D
        rng, T = np.random.default_rng(seed), len(slot)
        self.qkv = K._bf(torch, rng, T, (hq + 2 * hkv) * D + pad, std=std)
        self.qw, self.kw = (K._bf(torch, rng, D) for _ in range(2)) if weights else (None, None)
        self.table = H.rope_table(500, D, 1e4)
        self.pos = rng.integers(0, 500, (axes, T)).astype(np.int32)
        self.axis = [int(a) for a in rng.integers(0, axes, D // 2)]
        self.axis[0] = axes - 1
        self.k, self.ks = _cache(torch, rng, pages, hkv, D)
        self.v, self.vs = _cache(torch, rng, pages, hkv, D)
        self.op = H.QkNormRope(hq, hkv, D, self.qw, self.kw, self.table, axis=self.axis)
        self.dev = lambda a: torch.from_numpy(a).cuda()

    def call(self, **kw):
        p = self.pos[0] if len(self.pos) == 1 else self.pos
        return self.op(self.qkv, self.dev(np.ascontiguousarray(p)), self.dev(self.slot), self.k, self.v,
                       k_scale=self.ks, v_scale=self.vs, **kw)

    def check(self, err=0, rows=None, **kw):
        hq, hkv, D, T = self.hq, self.hkv, self.D, len(self.slot)
        had = [(_u8(c), s.cpu().numpy()) for c, s in ((self.k, self.ks), (self.v, self.vs))]
        q = self.call(**kw)
        self.torch.cuda.synchronize()
        assert self.op.errors() == err
        x = K._np(self.qkv)[:, : (hq + 2 * hkv) * D].reshape(T, -1, D)
        rot = self.table.cpu().numpy().astype(np.float64)[self.pos[np.array(self.axis)].T, np.arange(D // 2)]
        w = [None if a is None else K._np(a) for a in (self.qw, self.kw)]
        with np.errstate(invalid="ignore", over="ignore"):
            qr, qs = C.norm_rope(x[:, :hq], w[0], rot[..., 0], rot[..., 1], 1e-6)
            kr, ksz = C.norm_rope(x[:, hq: hq + hkv], w[1], rot[..., 0], rot[..., 1], 1e-6)
        fine = np.isfinite(qr)
        tol = 2.0 ** -8 * np.abs(qr) + 2.0 ** -19 * qs + 1e-30
        assert (np.abs(K._np(q) - qr) <= tol)[fine].all()
        slot = self.slot if rows is None else np.where(rows, self.slot, -1)
        # values are exact, keys off by the 32-bit arithmetic of their norm and rotation, 2^-19
        # of the two terms (see the bf16 cache's test)
        for new, size, (codes, scale), got, got_s in ((kr, ksz, had[0], self.k, self.ks),
                                                      (x[:, hq + hkv:], 0 * kr, had[1], self.v, self.vs)):
            exact, want, want_s = F.put(new, slot, codes, scale)
            got, got_s = _u8(got), got_s.cpu().numpy()
            written = np.zeros(want.shape[:2], bool)
            slip = np.zeros(want.shape)
            for t, s in enumerate(slot):
                if s >= 0:
                    written[s // PAGE, s % PAGE] = True
                    slip[s // PAGE, s % PAGE] = size[t] / want_s[s // PAGE][:, None]
            # a scale is a quotient of the largest value (one rounding), or doublings of what was there
            assert (np.abs(got_s - want_s) <= want_s * (2.0 ** -23 + 2.0 ** -18 * (size.max() > 0))).all()
            # rows that were there: the same, or halved as often as the scale was doubled, to the bit
            assert np.array_equal(got[~written], want[~written])
            a, ok = F.decode(got), np.isfinite(exact)
            assert np.array_equal(np.isnan(a), ~ok)
            # half a step of e4m3: 2^-4 of the value, 2^-10 below its normal numbers; twice the
            # product's and the reciprocal's rounding; the key's own error and its scale's
            half = np.maximum(2.0 ** -4 * np.abs(exact), 2.0 ** -10) * (1 + 2.0 ** -20)
            half += 2.0 ** -22 * np.abs(exact) + (2.0 ** -19 * slip + 2.0 ** -18 * np.abs(exact) if size.max() > 0 else 0.0)
            with np.errstate(invalid="ignore"):
                bad = np.abs(a - exact) > half
            assert not (bad & ok & written[:, :, None, None]).any()
        return q


WRITES = [  # new, ctx, H_q, H_kv, D, axes, pad, weights
    ([1], [0], 4, 1, 64, 1, 0, True), ([1], [15], 4, 4, 128, 1, 8, True), ([16], [0], 8, 2, 64, 1, 0, False),
    ([17], [15], 16, 2, 128, 3, 0, True), ([1] * 33, list(range(33)), 16, 2, 128, 1, 0, True),
    ([5, 1, 40, 3, 1], [3, 31, 7, 13, 16], 6, 2, 64, 3, 64, True), ([300, 77], [0, 9], 32, 8, 128, 3, 64, True),
    ([1000], [5], 40, 8, 128, 1, 0, True), ([2] * 100, [14, 15, 16, 17] * 25, 8, 8, 64, 1, 0, False),
    ([3, 129], [16, 1], 2, 2, 128, 2, 0, True), ([700], [0], 1, 1, 64, 4, 0, True)]


@gpu
@pytest.mark.parametrize("new,ctx,hq,hkv,D,axes,pad,weights", WRITES)
def test_gpu_write(torch, new, ctx, hq, hkv, D, axes, pad, weights):
    slot, pages = _slots(np.random.default_rng(sum(new)), new, ctx)
    w = Write(torch, slot, pages, hq, hkv, D, axes, pad, seed=len(slot), weights=weights)
    w.check()
    w.check()  # the same rows once more: their pages' scales have grown already


@gpu
def test_gpu_write_leaves_out_rows_without_a_slot(torch):
    rng = np.random.default_rng(3)
    slot, pages = _slots(rng, [20, 1, 50], [5, 3, 0])
    slot[[0, 1, 9, 10, 19, 20]] = -1  # a run's first rows and last ones, a whole one
    slot[21 + 16: 21 + 32] = -1       # a whole page's
    Write(torch, slot, pages, 4, 2, 128).check()
    slot[:] = -1
    Write(torch, slot, pages, 4, 2, 64).check()
    # a slot past the cache is flagged, and nothing of its row is written
    slot, pages = _slots(rng, [20], [0])
    out = slot.copy()
    out[[15, 19]] = [pages * PAGE, pages * PAGE + 4000000]
    Write(torch, out, pages, 4, 2, 64).check(err=0x8, rows=out < pages * PAGE)


@gpu
@pytest.mark.parametrize("D", [64, 128])
def test_gpu_write_of_values_out_of_the_ordinary(torch, D):
    slot, pages = _slots(np.random.default_rng(4), [40, 3], [0, 5])
    w = Write(torch, slot, pages, 4, 2, D, weights=False)
    x = w.qkv.view(43, 8, D)
    x[0:16, 4:] = 0.0                       # a page of zeros
    x[16:32, 7, 3] = 3e38                   # a value that makes others vanish
    x[17, 6, 1], x[18, 6, 2], x[19, 6, 3] = INF, -INF, NAN
    x[20, 4, 5], x[21, 5, 0] = INF, NAN     # keys: their rows have no norm
    x[22, 6] *= 1e-38
    x[32:40, 6] = NAN                       # nothing finite in a page
    x[40, 7] = 1e30                         # a scale that grows by some hundred doublings
    x[41, 6] = 0.0
    w.check()
    assert (w.ks.cpu() > 0).all() and (w.vs.cpu() > 0).all()


@gpu
def test_gpu_write_grows_scales_without_rounding_twice(torch):
    # 16 tokens one by one, ever larger: every code is within half a step of its value's
    # quotient with the last scale, or what is left of it below the normal numbers
    rng = np.random.default_rng(5)
    hkv, D = 2, 64
    k, v, ks, vs = H.fp8_cache(3, hkv, D)
    op = H.QkNormRope(2, hkv, D, None, None, H.rope_table(32, D))
    rows = K._bf(torch, rng, 16, 4 * D + 2 * D) * torch.exp2(torch.arange(16, device="cuda") * 0.4)[:, None].bfloat16()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for t in range(16):
        op(rows[t: t + 1], i32(t), i32(16 + t), k, v, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    x = K._np(rows)[:, 4 * D:].reshape(16, 2, D)[:, :, :].astype(np.float64)
    s = vs[1].cpu().numpy().astype(np.float64)
    top = np.abs(x).max((0, 2)) / 448
    assert (s >= top * (1 - 2.0 ** -23)).all() and (s < 2 * top).all()
    got = F.decode(_u8(v)[1]) * s[:, None]
    # each halving below the normal numbers rounds once more, by half a step at most: 2^-10 of the scale
    # of that time, which the later ones double: in all less than twice the last
    assert (np.abs(got - x) <= 2.0 ** -4 * np.abs(x) * (1 + 2.0 ** -18) + 2.0 ** -9 * s[:, None]).all()
    assert not _u8(v)[[0, 2]].any()


@gpu
def test_gpu_write_keeps_the_largest_scales(torch):
    # doublings end below twice the largest value / 448, which may pass 2^120
    k, v, ks, vs = H.fp8_cache(1, 1, 64)
    op = H.QkNormRope(1, 1, 64, None, None, H.rope_table(8, 64))
    vs.fill_(1.1 * 2.0 ** -10)
    ks.fill_(1.0)
    rows = torch.ones(2, 3 * 64, dtype=torch.bfloat16, device="cuda")
    rows[0, 2 * 64:] = 3.38e38
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for t in range(2):
        op(rows[t: t + 1], i32(t), i32(5 + t), k, v, k_scale=ks, v_scale=vs)
    torch.cuda.synchronize()
    assert op.errors() == 0
    assert vs.item() == float(np.float32(1.1)) * 2.0 ** 120
    got, x = F.decode(_u8(v)[0, 5]), float(rows[0, -1]) / vs.item()
    assert (np.abs(got - x) <= 2.0 ** -4 * x).all() and not _u8(v)[0, 6].any()


@gpu
@pytest.mark.parametrize("bad", [0.0, -1.0, NAN, INF, 1e-35])
def test_gpu_write_flags_scales_that_are_none(torch, bad):
    slot, pages = _slots(np.random.default_rng(6), [3, 20], [5, 0])
    w = Write(torch, slot, pages, 4, 2, 64)
    w.ks[int(slot[0]) // PAGE, 1] = bad
    w.vs[int(slot[3]) // PAGE, 0] = bad     # of a page that is written from its first row on: not read
    w.check(err=0x800)


@gpu
def test_gpu_write_in_place_on_another_stream_and_in_a_graph(torch):
    slot, pages = _slots(np.random.default_rng(7), [30, 2, 9], [3, 20, 0])
    w = Write(torch, slot, pages, 4, 2, 128)
    first = [x.clone() for x in (w.k.view(torch.uint8), w.ks, w.v.view(torch.uint8), w.vs)]

    def again(call):
        for x, y in zip((w.k.view(torch.uint8), w.ks, w.v.view(torch.uint8), w.vs), first):
            x.copy_(y)
        torch.cuda.synchronize()
        q = call()
        torch.cuda.synchronize()
        return [q.clone()] + [x.clone() for x in (w.k.view(torch.uint8), w.ks, w.v.view(torch.uint8), w.vs)]

    want = again(w.call)
    side = torch.cuda.Stream()
    got = again(lambda: w.call(stream=side))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g, pos, sl = torch.cuda.CUDAGraph(), w.dev(w.pos[0].copy()), w.dev(w.slot)
    with torch.cuda.graph(g):
        q = w.op(w.qkv, pos, sl, w.k, w.v, k_scale=w.ks, v_scale=w.vs)
    got = again(lambda: (g.replay(), q)[1])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # the queries where they were
    qkv = w.qkv.clone()
    alone = qkv[:, : 4 * 128].contiguous()
    a = w.op.args
    w.op(qkv, pos, sl, w.k, w.v, k_scale=w.ks, v_scale=w.vs)
    a.q, a.q_stride, a.q_out = alone.data_ptr(), 4 * 128, alone.data_ptr()
    H.hpd_qk_norm_rope_fp8(w.op._fp8, H._stream_handle(None))
    torch.cuda.synchronize()
    assert torch.equal(alone.view(want[0].shape), want[0])


# -------------------------------------------------------------- the attention --

def _coded(torch, c, seed=0, spread=3.0):
    """The case's cache in 8 bits: rows that no sequence holds are codes of NaN, and so
    are the scales of pages that none holds."""
    rng = np.random.default_rng(seed)
    for name in ("k", "v"):
        x = c[name + "c"].float()
        top = torch.nan_to_num(x).abs().amax((1, 3))
        grow = torch.from_numpy((2.0 ** rng.uniform(0, spread, tuple(top.shape))).astype(np.float32)).cuda()
        scale = torch.where(top > 0, top / 448 * grow, 1.0)
        c[name + "8"] = (x / scale[:, None, :, None]).to(torch.float8_e4m3fn)
        held = torch.isfinite(x).any(-1).any(-1).any(-1)
        c[name + "s"] = torch.where(held[:, None], scale, NAN).contiguous()
        c[name + "c"] = c[name + "8"].double() * c[name + "s"].double()[:, None, :, None]
    return c


def _op(c, max_tokens=None):
    return H.ChunkAttn(c["q"].shape[1], c["k8"], c["v8"], c["table"], max_tokens=max_tokens or c["q"].shape[0],
                       max_seq_len=c["max_seq_len"], scale=c["scale"], k_scale=c["ks"], v_scale=c["vs"])


def _reference(c):
    z = lambda x: np.nan_to_num(x.double().cpu().numpy())  # noqa: E731
    cu, q = c["cu"].cpu().numpy(), K._np(c["q"])
    n = int(cu[-1])
    got = C.attn(q[:n], z(c["kc"]), z(c["vc"]), c["table"].cpu().numpy(), cu, c["total"].cpu().numpy(),
                 None if c["full"] is None else c["full"].cpu().numpy(), c["scale"])
    # a query is taken in two e4m3 parts of one power of two, the second to 2^-10 of 224 of its largest value at
    # least: a score is off by 2^-17 of that times the sum of the key's sizes
    D = q.shape[2]
    k = np.abs(z(c["kc"])).sum(-1).max()
    return got, 2.0 ** -17 * np.abs(q[:n]).max(-1) * k * (abs(c["scale"]) or D ** -0.5)


def _near(c, out, lse, rows=None):
    (ref, rl, size, reach), q_slip = _reference(c)
    rows = np.ones(rl.shape, bool) if rows is None else rows
    assert np.array_equal(np.isneginf(lse)[rows], np.isneginf(rl)[rows])
    fin = np.isfinite(rl) & rows
    # as with the bf16 cache: scores off by some 2^-21 of the sum of their products' sizes, lse by as much and by the
    # exponentials' and the log's 2^-21; out by a rounding to bf16 of each weight (with its value's scale in it) and
    # of the result, 2^-8 each
    slip = 2.0 ** -20 * reach + 2.0 ** -19 + q_slip
    assert (np.abs(lse - rl)[fin] <= slip[fin] + 2.0 ** -21 * np.abs(rl[fin])).all()
    tol = 2.0 ** -8 * (np.abs(ref) + size) * 1.02 + 2 * slip[..., None] * size
    bad = (np.abs(out - ref) > tol) & rows[..., None]
    assert not bad.any(), (np.argwhere(bad)[:5], np.abs(out - ref)[rows].max())


def _check(torch, c, err=0):
    op = _op(c)
    op.out.fill_(7.0)
    op.lse.fill_(7.0)
    out, lse = op(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    assert op.errors() == err
    out, lse = out.clone(), lse.clone()
    again = op(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    n = int(c["cu"][-1])
    out, lse = K._np(out), lse.cpu().numpy()
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()  # rows of no sequence
    _near(c, out[:n], lse[:n])
    return op


@gpu
@pytest.mark.parametrize("new,total,hq,hkv,D", K.ATTN + [([1] * 8, [1, 15, 16, 17, 127, 128, 129, 640], 8, 8, 128),
                                                         ([4, 4, 4], [500, 4, 33], 32, 2, 128)])
def test_gpu_attn(torch, new, total, hq, hkv, D):
    _check(torch, _coded(torch, K._attn_case(torch, new, total, hq, hkv, D, seed=sum(total) + D)))


@gpu
@pytest.mark.parametrize("new,total,full,hq,hkv,D", [
    ([200], [200], [150], 16, 2, 128), ([70, 5, 3], [300, 5, 90], [280, 5, 0], 8, 2, 64),
    ([33, 1], [161, 40], [140, 99], 10, 2, 128), ([129], [257], [257], 4, 4, 128)])
def test_gpu_attn_prefix_mask(torch, new, total, full, hq, hkv, D):
    _check(torch, _coded(torch, K._attn_case(torch, new, total, hq, hkv, D, seed=9, full=full)))


@gpu
def test_gpu_attn_rows_without_keys(torch):
    for hq, hkv, D in ((8, 2, 128), (6, 2, 64)):
        _check(torch, _coded(torch, K._attn_case(torch, [5, 3, 40, 2], [0, 1, 17, 2], hq, hkv, D, seed=1)))


@gpu
def test_gpu_attn_strided_queries_scales_and_spare_rows(torch):
    for scale in (0.3, -0.2, 0.0):
        _check(torch, _coded(torch, K._attn_case(torch, [20, 1, 70], [150, 33, 70], 16, 2, 128, seed=2, spare_rows=5,
                                                 pad_q=64, scale=scale, max_pages=50, max_seq_len=700)))


@gpu
@pytest.mark.parametrize("D", [64, 128])
def test_gpu_attn_scales_far_apart(torch, D):
    # pages of very small and very large keys and values side by side, and queries with an
    # outlier that takes the others' bits
    c = _coded(torch, K._attn_case(torch, [60, 2], [700, 300], 16, 2, D, seed=3))
    rng = np.random.default_rng(4)
    for name, lo, hi in (("k", -6, 2), ("v", -30, 20)):
        c[name + "s"] *= torch.from_numpy((2.0 ** rng.integers(lo, hi, tuple(c[name + "s"].shape))).astype(np.float32)).cuda()
        c[name + "c"] = c[name + "8"].double() * c[name + "s"].double()[:, None, :, None]
    c["q"][::3, :, 5] *= 50
    c["q"][1] = 0
    c["q"][2] *= 1e-30
    _check(torch, c)
    c["vs"][int(c["table"][0, 3])] = 0.0  # a page whose values are all 0
    c["vc"] = c["v8"].double() * c["vs"].double()[:, None, :, None]
    _check(torch, c)


@gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S,n", [(19, 1), (1, 608)])
@pytest.mark.parametrize("ratio,low,zeros,most", [
    (2.0 ** -10, 10, None, 1.0), (2.0 ** -13, 8, None, 1.0), (2.0 ** -13, 10, None, 1.0), (2.0 ** -13.9, 9, None, 1.0),
    (2.0 ** -13.9, 11, None, 1.0), (2.0 ** -13, 10, -1, 1.0), (2.0 ** -16, 10, None, 1.0), (2.0 ** 9, 11, None, 1.0),
    (2.0 ** -13, 10, None, 2.0 ** 127), (2.0 ** -13, 10, None, 2.0 ** -80), (2.0 ** -13, 10, 60, 1.0), (2.0 ** -3, 7, 80, 1.0),
    (1.0, 8, 88, 1.0)])
def test_gpu_attn_values_of_other_scales_than_the_first_blocks(torch, S, n, D, ratio, low, zeros, most):
    # 16,000 keys of equal weights, e^-low of the largest, whose values' scales are `ratio` times the second page's;
    # that has next to no weight, so that a row is of the small ones.  152 units of all keys: the sequences share
    # their pages, the queries are the same.  zeros: scores of pages of zeros with the least scale (weights that no
    # product has, or no sum of 32 bits).
    hq, hkv, L = 32, 8, 16400
    rng = np.random.default_rng(17)
    pages = C.pages_of(L)
    k, v = np.zeros((pages, PAGE, hkv, D)), 448.0 * 2.0 ** -rng.integers(0, 2, (pages, PAGE, hkv, D))
    vs = np.full((pages, hkv), ratio, np.float32)
    k[..., 0] = -low
    k[0, 3, :, 0] = 0
    k[1, :, :, 0], vs[1] = -40, 1.0
    vs *= np.float32(most)
    if zeros is not None:
        v[[20, 333]], vs[[20, 333]] = 0, 2.0 ** -100
        k[[20, 333], 5, :, 0] = zeros
    code = lambda x: torch.from_numpy(x).cuda().float().to(torch.float8_e4m3fn)  # noqa: E731
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    ids = rng.permutation(pages)
    back = np.argsort(ids)  # the page of a sequence that is held at a place of the cache
    op = H.ChunkAttn(hq, code(k[back]), code(v[back]), i32(np.tile(ids, (S, 1))), max_tokens=S * n, scale=1.0,
                     k_scale=torch.ones(pages, hkv, device="cuda"), v_scale=torch.from_numpy(vs[back]).cuda())
    q = torch.zeros(S * n, hq, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    out, lse = op(q, i32(np.arange(S + 1) * n), i32([L] * S))
    torch.cuda.synchronize()
    assert op.errors() == 0
    p = np.exp(k[..., 0].reshape(-1, hkv)[:L])
    x = (v * vs[:, None, :, None].astype(np.float64)).reshape(-1, hkv, D)[:L]
    lim = L - n + np.arange(n)
    tot = np.cumsum(p, 0)[lim]
    size = np.cumsum(p[..., None] * x, 0)[lim] / tot[..., None]  # (all values are positive: the output too)
    rows = lambda a: np.repeat(np.tile(a, (S,) + (1,) * (a.ndim - 1)), hq // hkv, 1)  # noqa: E731
    # roundings as in _near, of scores whose queries lose nothing, and 2^-28 a key of what the products (of weights
    # and scales) add up to, of the largest code
    slip = 2.0 ** -20 * max(40, zeros or 0) + 2.0 ** -19
    lost = 2.0 ** -28 * 448 * ((lim + 1) / tot.T * np.cumsum(p * np.repeat(vs, PAGE, 0)[:L], 0)[lim].T).T
    assert (np.abs(lse.cpu().numpy() - rows(np.log(tot))) <= slip + 2.0 ** -21 * np.abs(rows(np.log(tot)))).all()
    off = np.abs(K._np(out) - rows(size))
    assert (off <= (2.0 ** -7 * 1.02 + 2 * slip) * rows(size) + rows(lost)[..., None]).all(), (off / rows(size)).max()


@gpu
def test_gpu_attn_rising_scores(torch):
    # scores that rise by more than the window of a fixed base
    c = K._attn_case(torch, [64, 1], [900, 2000], 8, 2, 128, seed=5)
    c["kc"] = torch.where(torch.isfinite(c["kc"]), c["kc"] * 0.05, c["kc"])
    for s, t in enumerate((900, 2000)):
        for j in range(t):
            c["kc"][int(c["table"][s, j // PAGE]), j % PAGE, :, 0] = 0.3 * j
    c["q"][:, :, 0] = c["q"][:, :, 0].abs() + 1
    _check(torch, _coded(torch, c, spread=0.0))


@gpu
def test_gpu_attn_many_short_units_one_after_another(torch):
    for hq, hkv, D in ((32, 8, 128), (8, 8, 64)):
        S = 700
        c = _coded(torch, K._attn_case(torch, [1] * S, [1 + i % 37 for i in range(S)], hq, hkv, D, seed=6))
        _check(torch, c)


@gpu
@pytest.mark.parametrize("new,total,hq,hkv,D", [
    ([1], [20000], 16, 2, 128), ([1, 1], [9000, 30], 32, 8, 128), ([16], [9000], 16, 2, 64), ([500], [2500], 16, 4, 64),
    ([1] * 5, [3999, 1, 70, 2048, 2049], 8, 1, 128), ([700], [3000], 40, 8, 128),
    # groups of one and two sequences a lane of the scheduler, in order of their lengths and not, some empty
    ([1] * 33, [64 * i for i in range(33)], 8, 2, 64), ([i % 4 for i in range(64)], [9 + 40 * (i * 23 % 64) for i in range(64)], 32, 8, 128),
    ([1] * 64, [5 + 2000 * (i == 40) for i in range(64)], 4, 4, 64), ([60] * 32, [60 + 37 * (i * 7 % 32) for i in range(32)], 16, 4, 64)])
def test_gpu_attn_split_tiles(torch, new, total, hq, hkv, D):
    c = _coded(torch, K._attn_case(torch, new, total, hq, hkv, D, seed=7, max_seq_len=max(total)))
    _check(torch, c)


@gpu
@pytest.mark.parametrize("new,total,full,hq,hkv,D", [
    ([100, 3], [300, 90], None, 16, 2, 128), ([100, 3], [300, 90], None, 16, 2, 64), ([128], [150], None, 1, 1, 128),
    ([60], [3000], None, 40, 8, 128), ([90, 1], [200, 77], [150, 0], 10, 2, 128), ([1], [5000], None, 16, 2, 128)])
def test_gpu_attn_codes_of_nan_stay_where_they_are_seen(torch, new, total, full, hq, hkv, D):
    c = _coded(torch, K._attn_case(torch, new, total, hq, hkv, D, seed=8, full=full))
    L, n, G = total[0], new[0], hq // hkv
    at = [int(L - n + f * (n - 1)) for f in (0.2, 0.5, 0.95)]
    cols = (5, D - 1, 33)
    for j, col in zip(at, cols):
        c["v8"].view(torch.uint8)[int(c["table"][0, j // PAGE]), j % PAGE, hkv - 1, col] = 0x7F
    out, lse = _op(c)(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    out, lse = K._np(out), lse.cpu().numpy()
    lim = L - n + np.arange(n) + 1
    if full:
        lim = np.minimum(np.maximum(lim, full[0]), L)
    want = np.zeros(out.shape, bool)
    for j, col in zip(at, cols):
        want[np.flatnonzero(lim > j), (hkv - 1) * G:, col] = True
    assert np.array_equal(np.isnan(out), want) and np.isfinite(lse).all()
    _near(c, out, lse, rows=~want.any(-1))
    # a key of NaN: the rows that see it, all of them
    j = at[1]
    c["k8"].view(torch.uint8)[int(c["table"][0, j // PAGE]), j % PAGE, 0, 7] = 0xFF
    out, lse = _op(c)(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    rows = np.zeros(lse.shape, bool)
    rows[np.flatnonzero(lim > j), :G] = True
    assert np.array_equal(np.isnan(K._np(out)).all(-1) & (np.arange(hq) < G), rows)
    assert np.array_equal(np.isnan(lse.cpu().numpy()), rows)


@gpu
def test_gpu_attn_queries_that_are_not_finite(torch):
    c = _coded(torch, K._attn_case(torch, [40, 1], [300, 500], 8, 2, 128, seed=10))
    c["q"][3, 1, 5], c["q"][7, 0, 100], c["q"][40, 7, 0] = INF, NAN, -INF
    out, lse = _op(c)(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    out, lse = K._np(out), lse.cpu().numpy()
    off = np.zeros(lse.shape, bool)
    off[[3, 7, 40], [1, 0, 7]] = True
    assert np.array_equal(np.isnan(lse), off) and np.array_equal(np.isnan(out).all(-1), off)
    c["q"] = torch.nan_to_num(c["q"], posinf=0.0, neginf=0.0)
    _near(c, out, lse, rows=~off)


@gpu
def test_gpu_attn_flags_and_clamps_device_data(torch):
    c = _coded(torch, K._attn_case(torch, [20, 30], [100, 200], 8, 2, 64, seed=11))
    pages = c["k8"].shape[0]
    c["ks"], c["vs"] = torch.nan_to_num(c["ks"], nan=1.0), torch.nan_to_num(c["vs"], nan=1.0)
    op = _op(c)
    for bad in (-1.0, NAN, INF):
        keep = c["vs"].clone()
        page = int(c["table"][1, 2])
        c["vs"][page] = bad
        out, lse = op(c["q"], c["cu"], c["total"])
        torch.cuda.synchronize()
        assert op.errors() == 0x800
        c["vs"][page] = 0.0
        want = [x.clone() for x in (out, lse)]
        got = op(c["q"], c["cu"], c["total"])
        assert all(torch.equal(a, b) for a, b in zip(want, got))
        c["vs"].copy_(keep)
        H.hpd_workspace_init(op.workspace.data_ptr(), op.workspace.numel(), H._stream_handle(None))
    c["table"][0, 1] = pages + 7
    c["table"][1, 0] = -3
    op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0x8
    H.hpd_workspace_init(op.workspace.data_ptr(), op.workspace.numel(), H._stream_handle(None))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    op(c["q"], i32(0, 20, 70), i32(100, 1 << 20))
    torch.cuda.synchronize()
    assert op.errors() & 0x6 == 0x6


@gpu
def test_gpu_attn_on_another_stream_in_a_graph_and_of_fewer_rows(torch):
    c = _coded(torch, K._attn_case(torch, [20, 1, 9], [100, 4000, 9], 16, 2, 128, seed=12))
    op = _op(c, max_tokens=500)
    want = [x.clone() for x in op(c["q"], c["cu"], c["total"])]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = op(c["q"], c["cu"], c["total"], stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = op(c["q"], c["cu"], c["total"])
    c["q"].copy_(-c["q"])
    g.replay()
    torch.cuda.synchronize()
    _near(c, K._np(held[0]), held[1].cpu().numpy())


@gpu
@pytest.mark.parametrize("S", [20, 50, 100])
def test_gpu_attn_offsets_out_of_order(torch, S):
    # every second sequence begins at row 0 again: more tiles than there are rows for; a
    # sequence that has rows of its own alone keeps its results
    c = _coded(torch, K._attn_case(torch, [3] * S, [200 + i for i in range(S)], 8, 2, 64, seed=15))
    op = _op(c)
    want = [x.clone() for x in op(c["q"], c["cu"], c["total"])]
    cu = c["cu"].clone()
    cu[1:S:2] = 3 * S
    op(c["q"], cu, c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0x2
    H.hpd_workspace_init(op.workspace.data_ptr(), op.workspace.numel(), H._stream_handle(None))
    got = op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0 and all(torch.equal(a, b) for a, b in zip(want, got))


@gpu
def test_gpu_calls_at_once_and_graphs_that_share_a_workspace(torch):
    cases = [_coded(torch, K._attn_case(torch, new, total, 16, 2, 128, seed=16 + i))
             for i, (new, total) in enumerate((([300, 1], [1500, 4000]), ([1] * 40, list(range(30, 1230, 30)))))]
    ops = [_op(c) for c in cases]
    run = lambda i, **kw: ops[i](cases[i]["q"], cases[i]["cu"], cases[i]["total"], **kw)  # noqa: E731
    want = [[x.clone() for x in run(i)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for o in ops:
        o.out.zero_(), o.lse.zero_()
    torch.cuda.synchronize()
    for _ in range(20):  # an object a stream, at the same time
        for i in range(2):
            run(i, stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(want[i], (ops[i].out, ops[i].lse)))
    # one object in two graphs, of different numbers of rows, one after the other
    c, op = cases[0], ops[0]
    one = dict(cu=torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda"), total=c["total"])
    alone = [x.clone() for x in op(c["q"][:1], one["cu"], one["total"])]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        whole = op(c["q"], c["cu"], c["total"])
    with torch.cuda.graph(graphs[1]):
        first = op(c["q"][:1], one["cu"], one["total"])
    for _ in range(3):
        graphs[0].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want[0], whole))
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(alone, first))
    assert ops[0].errors() == ops[1].errors() == 0


@gpu
def test_gpu_pages_beyond_32_bits_of_a_long_cache(torch):
    # 1.2 million pages of one head of 128: codes past 2^31
    pages, D = 1200000, 128
    k = torch.zeros(pages, PAGE, 1, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros(pages, PAGE, 1, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks, vs = torch.ones(pages, 1, device="cuda"), torch.ones(pages, 1, device="cuda")
    far = [pages - 1, 5, pages - 3, 1 << 20]
    rng = np.random.default_rng(13)
    table = torch.tensor([far], dtype=torch.int32, device="cuda")
    slot = torch.tensor([far[j // PAGE] * PAGE + j % PAGE for j in range(60)], dtype=torch.int32, device="cuda")
    op = H.QkNormRope(4, 1, D, None, None, H.rope_table(64, D))
    qkv = K._bf(torch, rng, 60, 6 * D)
    q = op(qkv, torch.arange(60, dtype=torch.int32, device="cuda"), slot, k, v, k_scale=ks, v_scale=vs)
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    c = dict(q=q, k8=k, v8=v, ks=ks, vs=vs, table=table, cu=i32(0, 60), total=i32(60), full=None, scale=0.0, max_seq_len=60)
    out, lse = _op(c)(q, c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0
    near = dict(c, table=i32(0, 1, 2, 3)[None])
    for n in "kv":
        near[n + "c"] = c[n + "8"].view(torch.uint8)[far].view(torch.float8_e4m3fn).double() * c[n + "s"][far].double()[:, None, :, None]
    assert (near["vc"].float() != 0).any()
    _near(near, K._np(out), lse.cpu().numpy())


# ----------------------------------------------------------------- together --

@gpu
def test_gpu_prompts_then_tokens_with_their_log_probabilities(torch):
    # three sequences through slots, write and attention in chunks and then token by token,
    # and the log probabilities of what each step chose; the cache in bf16 beside it
    rng = np.random.default_rng(14)
    S, hq, hkv, D, V, steps = 3, 8, 2, 64, 900, 6
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    pages = 40
    free, top = i32(rng.permutation(pages)), i32([pages])
    table, seq = torch.zeros(S, 12, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    slots = H.ChunkSlots(table, seq, free, top, max_tokens=256)
    rope = H.QkNormRope(hq, hkv, D, K._bf(torch, rng, D), K._bf(torch, rng, D), H.rope_table(256, D))
    k, v, ks, vs = H.fp8_cache(pages, hkv, D)
    kb, vb = (torch.zeros(pages, PAGE, hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    a8 = H.ChunkAttn(hq, k, v, table, max_tokens=256, k_scale=ks, v_scale=vs)
    a16 = H.ChunkAttn(hq, kb, vb, table, max_tokens=256)
    head = K._bf(torch, rng, hq * D, V, std=0.2)
    total = np.zeros(S, int)
    for chunk in ([70, 1, 33], [9, 30, 0]) + ([1, 1, 1],) * steps:
        T = sum(chunk)
        c = slots(i32(chunk))
        qkv = K._bf(torch, rng, T, (hq + 2 * hkv) * D)
        q = rope(qkv, c.pos[:T], c.slot, k, v, k_scale=ks, v_scale=vs).clone()
        q16 = rope(qkv, c.pos[:T], c.slot, kb, vb)
        assert torch.equal(q, q16)
        out, lse = a8(q, c.chunk_cu, c.seq_len)
        out16, lse16 = a16(q, c.chunk_cu, c.seq_len)
        total += chunk
        case = dict(q=q, k8=k, v8=v, ks=ks, vs=vs, table=table, cu=c.chunk_cu, total=c.seq_len, full=None, scale=0.0,
                    max_seq_len=0, kc=k.double() * ks.double()[:, None, :, None], vc=v.double() * vs.double()[:, None, :, None])
        _near(case, K._np(out), lse.cpu().numpy())
        # codes are within 2^-4 of their values: so are weighted means of them, and scores by 2^-4 of their products
        assert float((out.float() - out16.float()).norm() / out16.float().norm()) < 0.1
        logits = (out.flatten(1) @ head)[:, :V]
        chosen, _ = H.pmtp_accept(logits[:, None].contiguous(), torch.zeros(T, 1, dtype=torch.int32, device="cuda"))
        r = H.token_logprobs(logits, chosen[:, 0].contiguous(), top=3)
        assert torch.equal(r.top_tokens[:, 0], chosen[:, 0])
        want = torch.log_softmax(logits.double(), -1).gather(1, chosen.long())[:, 0]
        assert float((r.logprob - want).abs().max()) < 1e-4
    assert a8.errors() == 0 and rope.errors() == 0 and seq.tolist() == total.tolist()
