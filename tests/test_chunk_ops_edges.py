"""Chunks of new tokens over the paged cache at their edges: sizes at a limit,
calls of no rows and of one, tensors that share their storage, streams, values
that are not finite among long contexts."""
import contextlib
import importlib.util
import os
import re
import subprocess
import sys
import textwrap

import numpy as np
import pytest

import test_chunk_ops as K
from paper_2607_18839_gb300 import build as B
from paper_2607_18839_gb300 import hpd as H

gpu = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


class Host:
    """The binding on host tensors that say they are on a device: C calls are
    recorded and not made, unless a test makes them."""

    def __init__(self, torch, monkeypatch):
        class OnDevice(torch.Tensor):
            is_cuda = property(lambda self: True)

        self.torch, self.calls, self.stream = torch, [], "current"
        self.of = lambda t: t.as_subclass(OnDevice)
        self.bf = lambda *n: self.of(torch.zeros(n, dtype=torch.bfloat16))
        self.i32 = lambda *n: self.of(torch.zeros(n, dtype=torch.int32))

        @contextlib.contextmanager
        def on(stream):
            before, self.stream = self.stream, stream or self.stream  # (None: no other)
            yield
            self.stream = before

        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: self.calls.append(("synchronize",)))
        monkeypatch.setattr(H, "_stream_handle", lambda s: s or self.stream)
        monkeypatch.setattr(H, "hpd_workspace_init", lambda *a: self.calls.append(("clear",) + a))
        for name in ("hpd_qk_norm_rope", "hpd_chunk_attn"):
            monkeypatch.setattr(H, name, lambda args, s, name=name: self.calls.append((name, args, s)))

    def rope(self, H_q=4, H_kv=2, D=64, **kw):
        return H.QkNormRope(H_q, H_kv, D, None, None, self.of(self.torch.zeros(8, D // 2, 2)), **kw)


@pytest.fixture
def host(lib, monkeypatch):
    return Host(pytest.importorskip("torch"), monkeypatch)


# ------------------------------------------------------------ pages and slots --

@gpu
def test_gpu_slots_sizes_where_shared_memory_passes_its_default(torch):
    # the lengths of some 4,090 sequences fill the default size; each in a process of
    # its own, as a larger call before lets a smaller one through
    body = """
        import sys, torch
        sys.path[:0] = [%r, %r]
        import test_chunk_ops as K
        S = int(sys.argv[1])
        new, ctx = K._random_lengths(S, 3, 20, seed=S)
        K._check_slots(torch, K._slot_case(new, ctx, 3, extra=4, seed=1), int(new.sum()) + 1)
    """ % (ROOT, os.path.join(ROOT, "tests"))
    for S in (4083, 4084, 4095, 4096):
        r = subprocess.run([sys.executable, "-c", textwrap.dedent(body), str(S)], capture_output=True, text=True)
        assert r.returncode == 0, (S, r.stderr[-400:])


# --------------------------------------------------- norms, rotation, write --

def test_norm_rope_of_no_rows(lib, host, monkeypatch):
    # nothing to do, and tensors of no rows have no address
    rows = dict.fromkeys(("q", "k", "v", "pos", "slot", "q_out"))
    assert lib.hpd_qk_norm_rope(K.rope_args(T=0, **rows), None) == 0
    assert lib.hpd_qk_norm_rope(K.rope_args(T=1, **rows), None) == 1
    monkeypatch.setattr(H, "hpd_qk_norm_rope",
                        lambda a, s: H._check("hpd_qk_norm_rope", lib.hpd_qk_norm_rope(a, None)))
    cache = host.bf(2, PAGE, 2, 64)
    op = host.rope()
    op.args.workspace = op.args.rope = 4096
    empty = host.bf(0, 8 * 64)
    assert empty.data_ptr() == 0
    for _ in range(2):
        assert op(empty, host.i32(0), host.i32(0), cache, cache).shape == (0, 4, 64)


def test_norm_rope_of_one_row_has_no_stride(host):
    # (a stride between rows that are not there need not be a multiple of 8)
    op, cache = host.rope(), host.bf(2, PAGE, 2, 64)
    op(host.bf(5, 8 * 64 + 3)[:1], host.i32(1), host.i32(1), cache, cache)
    a = host.calls[-1][1]
    assert a.T == 1 and a.q_stride % 8 == a.k_stride % 8 == a.v_stride % 8 == 0
    op(host.bf(5, 8 * 64 + 16)[:2], host.i32(2), host.i32(2), cache, cache)
    assert a.T == 2 and a.q_stride == a.k_stride == a.v_stride == 8 * 64 + 16


@pytest.mark.parametrize("D", [0, 32, 96, 256, 512])
def test_norm_rope_refuses_other_head_sizes(host, D):
    with pytest.raises(H.HpdError) as e:
        host.rope(D=D)
    assert e.value.status == 2


def test_norm_rope_output_grows_on_the_stream_of_the_call(host, monkeypatch):
    # memory of the current stream may still be written there by what was enqueued
    # before; the call's kernel does not wait for that
    made, cache = [], host.bf(2, PAGE, 2, 64)
    new_empty = host.torch.Tensor.new_empty

    def note(self, *a, **kw):
        made.append(host.stream)
        return new_empty(self, *a, **kw)

    monkeypatch.setattr(host.torch.Tensor, "new_empty", note)
    for stream in (None, "side"):
        made.clear()
        op = host.rope()
        for T in (3, 2, 9):
            op(host.bf(T, 8 * 64), host.i32(T), host.i32(T), cache, cache, stream=stream)
            assert host.calls[-1][2] == (stream or "current")
        assert set(made) == {stream or "current"}


# ---------------------------------------------------------------- attention --

def _attn_op(host, **kw):
    return H.ChunkAttn(4, host.bf(8, PAGE, 2, 64), host.bf(8, PAGE, 2, 64), host.i32(2, 4), max_tokens=8, **kw)


def test_attn_refuses_rows_that_share_storage(host):
    # one row expanded to eight has a stride of 0, which the C call takes as rows
    # side by side: eight rows from where there is one
    op, one, n = _attn_op(host), host.bf(1, 4, 64), len(host.calls)
    for bad in (one.expand(8, 4, 64), host.bf(16, 64).as_strided((8, 4, 64), (64, 64, 1))):
        with pytest.raises(H.HpdError) as e:
            op(bad, host.i32(3), host.i32(2))
        assert e.value.status == 1
    assert len(host.calls) == n
    op(one.expand(1, 4, 64), host.i32(3), host.i32(2))  # one row has no stride
    op(host.bf(8, 5, 64)[:, :4], host.i32(3), host.i32(2))
    assert [c[0] for c in host.calls[n:]] == ["hpd_chunk_attn"] * 2 and host.calls[-1][1].q_stride == 5 * 64


def test_attn_workspace_is_cleared_on_the_stream_that_allocated_it(host):
    # what the current stream still has to write there comes before the clearing
    for kw in ({}, dict(stream="side")):
        host.calls.clear()
        op = _attn_op(host, **kw)
        assert host.calls == [("clear", op.workspace.data_ptr(), op.workspace.numel(), "current"), ("synchronize",)]


def test_no_loads_past_the_coherent_cache():
    # kernels start while the one before them still writes what they read, and
    # non-coherent loads are only for what nothing writes while a kernel runs
    for path in B.sources() + [os.path.join(B.CSRC, f) for f in os.listdir(B.CSRC) if f.endswith(".cuh")]:
        with open(path) as f:
            text = f.read()
        assert not re.search(r"__ldg\b|ld\.global\.(\w+\.)*nc\b", text), path


def test_no_promise_that_inputs_are_not_written():
    # const and __restrict__ together let the compiler choose such loads by itself
    for path in B.sources():
        with open(path) as f:
            assert not re.search(r"\bconst\s+\w+\s*\*\s*__restrict__", f.read()), path


def _mark(c, s, j, head, col, value):
    c["vc"][int(c["table"][s, j // PAGE]), j % PAGE, head, col] = value


def _check_not_finite(torch, c, marks, op=None):
    """A call with values that are not finite: sequence, key, KV head, column and
    value of each.  A sum with a NaN or with infinities of both signs in it is NaN,
    with those of one sign that infinity, whatever the (positive) weights."""
    for m in marks:
        _mark(c, *m)
    hq, hkv = c["q"].shape[1], c["kc"].shape[2]
    op = op or H.ChunkAttn(hq, c["kc"], c["vc"], c["table"], max_tokens=c["q"].shape[0])
    full = None if c["full"] is None else c["full"]
    out, lse = op(c["q"], c["cu"], c["total"], full)
    torch.cuda.synchronize()
    assert op.errors() == 0
    out, lse = K._np(out), lse.cpu().numpy()
    cu, total = c["cu"].cpu().numpy(), c["total"].cpu().numpy()
    want = np.zeros(out.shape)
    for s, j, g, col, value in marks:
        n = cu[s + 1] - cu[s]
        lim = total[s] - n + np.arange(n) + 1
        if full is not None:
            lim = np.minimum(np.maximum(lim, int(full[s])), total[s])
        rows = cu[s] + np.flatnonzero(lim > j)
        G = hq // hkv
        with np.errstate(invalid="ignore"):
            want[rows, g * G: (g + 1) * G, col] += value
    off = ~np.isfinite(want)
    assert np.array_equal(~np.isfinite(out), off) and np.isfinite(lse).all()
    assert np.array_equal(out[off], want[off], equal_nan=True)
    K._near_oracle(c, ~off.any(-1), out, lse)
    return off


INF, NAN = float("inf"), float("nan")


@gpu
@pytest.mark.parametrize("new,total,full,hq,hkv,D", [
    ([100, 3], [300, 90], None, 16, 2, 128), ([100, 3], [300, 90], None, 16, 2, 64), ([128], [150], None, 1, 1, 128),
    ([128, 5], [250, 5], None, 4, 4, 64), ([60], [3000], None, 40, 8, 128), ([90, 1], [200, 77], [150, 0], 10, 2, 128),
    ([300], [300], [290], 8, 8, 64), ([33], [161], None, 6, 2, 128)])
def test_gpu_attn_several_values_not_finite(torch, new, total, full, hq, hkv, D):
    # among a tile's own keys, NaN and both infinities in one column at several
    # keys; one before them that all see; the last key of all
    c = K._attn_case(torch, new, total, hq, hkv, D, seed=30, full=full)
    L, n = total[0], new[0]
    at = lambda f: L - n + int(f * (n - 1))  # noqa: E731
    g = hkv - 1
    marks = [(0, at(.2), g, 5, INF), (0, at(.5), g, 5, INF), (0, at(.7), g, 5, -INF), (0, at(.4), g, 6, -INF),
             (0, at(.3), g, 63, INF), (0, at(.6), g, 63, NAN), (0, 0, g, 9, INF), (0, at(.8), g, 9, -INF),
             (0, L - 1, 0, 0, NAN), (0, at(.1), 0, D - 1, INF)]
    off = _check_not_finite(torch, c, marks)
    assert off.any() and (full or not off.all(-1).any())
    # whole rows of values, keys whose scores they leave alone
    for j in (at(.25), at(.55)):
        c["vc"][int(c["table"][0, j // PAGE]), j % PAGE] = NAN
    out, lse = H.ChunkAttn(hq, c["kc"], c["vc"], c["table"], max_tokens=sum(new))(c["q"], c["cu"], c["total"], c["full"])
    torch.cuda.synchronize()
    lim = L - n + np.arange(n) + 1
    if full:
        lim = np.minimum(np.maximum(lim, full[0]), L)
    assert np.array_equal(np.isnan(K._np(out)[:n]).all((1, 2)), lim > at(.25)) and bool(torch.isfinite(lse).all())


@gpu
def test_gpu_attn_values_not_finite_behind_a_long_context(torch):
    # more sequences than are split, so that one CTA has all of the long one, and
    # units of others behind it: no wait runs out, every row is written
    S, L, n = 700, 200_000, 40
    new, total = [n] + [1] * (S - 1), [L] + [1 + i % 40 for i in range(S - 1)]
    c = K._attn_case(torch, new, total, 4, 1, 64, seed=31)
    op = H.ChunkAttn(4, c["kc"], c["vc"], c["table"], max_tokens=sum(new), max_seq_len=L)
    op.out.fill_(7.0)
    _check_not_finite(torch, c, [(0, L - 25, 0, 5, INF), (0, L - 9, 0, 5, NAN), (0, L - 12, 0, 40, -INF)], op)


@gpu
def test_gpu_attn_values_not_finite_cost_passes_and_no_more(torch):
    # a unit with such values is run again, its maxima first: three times its blocks.
    # Far from that lies what depends on one row at a time (hundreds of times).
    S, L, n = 300, 8192, 40
    new, total = [n] + [0] * (S - 1), [L] + [0] * (S - 1)
    c = K._attn_case(torch, new, total, 4, 1, 128, seed=32)
    op = H.ChunkAttn(4, c["kc"], c["vc"], c["table"], max_tokens=n, max_seq_len=L)

    def us():
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        best = 1e9
        for _ in range(5):
            ev[0].record()
            op(c["q"], c["cu"], c["total"])
            ev[1].record()
            torch.cuda.synchronize()
            best = min(best, 1e3 * ev[0].elapsed_time(ev[1]))
        return best

    plain = us()
    _mark(c, 0, L - 3, 0, 7, INF)
    again = us()
    print(f"{plain:.0f} us, with an infinity among the last keys {again:.0f}")
    assert op.errors() == 0 and again <= 10 * plain


@gpu
@pytest.mark.parametrize("value", [NAN, INF])
def test_gpu_attn_values_not_finite_in_a_split_of_no_weight(torch, value):
    # the keys of the first splits weigh e^-424 of the others: no weight in 32 bits, but
    # a value among them that is not finite is in every row's sum
    c = K._attn_case(torch, [1], [3000], 16, 8, 128, seed=33)
    c["q"][..., 0] = 16.0
    slot = torch.arange(3000, device="cuda")
    at = c["table"][0][slot // PAGE].long() * PAGE + slot % PAGE
    c["kc"].view(-1, 8, 128)[at[:1500], :, 0] = -300.0
    c["kc"].view(-1, 8, 128)[at[1500:], :, 0] = 0.0
    _mark(c, 0, 5, 1, 3, value)
    op = H.ChunkAttn(16, c["kc"], c["vc"], c["table"], max_tokens=1)
    out, lse = op(c["q"], c["cu"], c["total"])
    torch.cuda.synchronize()
    assert op.errors() == 0 and bool(torch.isfinite(lse).all())
    off = ~np.isfinite(K._np(out)[0])
    want = np.zeros((16, 128), bool)
    want[2:4, 3] = True
    assert np.array_equal(off, want)


# --------------------------------------------------------------- branch step --

@gpu
def test_gpu_branch_units_ordered_where_shared_memory_passes_its_default(torch):
    # 4,096 buckets, 240 pages and 3,470 branches of one row: what the ordering holds
    # ends within 144 bytes of the default size
    n_docs, B, hkv, D = 240, 3470, 64, 64
    words = 4096 + 4 * n_docs + 1 + 2 * B + -(-B // 128) + n_docs
    assert 48 * 1024 - 144 < 4 * words <= 48 * 1024
    rng = np.random.default_rng(40)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    kc, vc = K._bf(torch, rng, 8, PAGE, hkv, D), K._bf(torch, rng, 8, PAGE, hkv, D)
    pk, pv = K._bf(torch, rng, n_docs, hkv, D), K._bf(torch, rng, n_docs, hkv, D)
    q = torch.randn(B, hkv, D, device="cuda", dtype=torch.bfloat16)
    cu = np.minimum(np.arange(n_docs + 1) * 15, B)
    cu[-1] = B
    length, table = rng.integers(1, 129, B), rng.integers(0, 8, (B, 8))
    d = H.DeviceInputs(q=q, prefix_k=pk, prefix_v=pv, prefix_cu=t(np.arange(n_docs + 1)), branch_cu=t(cu),
                       branch_prefix_len=t(np.ones(B)), k_cache=kc, v_cache=vc, page_table=t(table), branch_len=t(length),
                       n_docs=n_docs, B=B, m=1, H_q=hkv, H_kv=hkv, D=D, num_pages=8, max_pages=8, prefix_tokens=n_docs,
                       max_prefix_len=1, scale=0.0)
    op = H.BranchAttn(d)
    assert H.hpd_branch_attn_kernel_name(op.args, 0) == "unit_order"
    out, lse = op()
    torch.cuda.synchronize()
    assert op.errors() == 0
    for b in rng.integers(0, B, 40):
        page = int(np.searchsorted(cu, b, side="right")) - 1
        n = int(length[b])
        at = t(table[b]).long()
        k = torch.cat((pk[page: page + 1], kc[at].flatten(0, 1)[:n])).double()
        v = torch.cat((pv[page: page + 1], vc[at].flatten(0, 1)[:n])).double()
        x = torch.einsum("hd,lhd->hl", q[b].double(), k) / 8.0
        assert float((lse[b] - x.logsumexp(-1)).abs().max()) <= 1e-4
        ref = torch.einsum("hl,lhd->hd", x.softmax(-1), v)
        # one rounding to bf16 of each weight and of the result
        assert float((out[b] - ref).abs().max()) <= 2.0 ** -7 * float(v.abs().max())


# -------------------------------------------------------- prefill in chunks --

def test_prefill_takes_text_in_pieces_that_fit(host):
    # text behind the vision tokens goes in whatever pieces a step has room for;
    # vision tokens in one piece
    path = os.path.join(ROOT, "examples", "prefill_then_decode.py")
    spec = importlib.util.spec_from_file_location("prefill_example", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    pages, steps = object.__new__(mod.Pages), []
    pages.vision, pages.total, pages.room = [30, 0, 12], [230, 300, 13], 100
    pages.check = lambda: None

    def step(chunk):
        assert 0 < sum(chunk) <= pages.room and min(chunk) >= 0
        steps.append(chunk)
        return host.torch.zeros(sum(chunk), 1)

    pages.step = step
    got = pages.prefill(per_step=256)
    assert [len(x) for x in got] == pages.total
    first = [next(s[d] for s in steps if s[d]) for d in range(3)]
    assert first[0] >= 30 and first[2] >= 12
