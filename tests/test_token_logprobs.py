"""Log probabilities of given tokens with entropies and alternatives against the
64-bit oracle (GPU), and what the call refuses (no GPU: nothing is launched)."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import logprobs as O
from paper_2607_18839_gb300 import build as B
from paper_2607_18839_gb300 import hpd as H

gpu = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


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


def args(**kw):
    a = H.hpd_token_logprobs_args()
    for p in ("logits", "tokens", "logprob", "entropy", "top_tokens", "top_logprobs"):
        setattr(a, p, 4096)
    for k, v in {**dict(R=4, V=100, top=5, fp32=0, scale=0.0), **kw}.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("bad,status", [
    (dict(R=-1), 1), (dict(V=0), 1), (dict(top=-1), 1), (dict(top=33), 2), (dict(V=3, top=4), 1), (dict(fp32=2), 1),
    (dict(V=2 ** 30 + 1), 2), (dict(scale=2.0 ** -121), 1), (dict(scale=2.0 ** 121), 1),
    (dict(scale=-1.0), 1), (dict(scale=INF), 1), (dict(scale=NAN), 1), (dict(row_stride=99), 1), (dict(row_stride=-5), 1),
    (dict(logits=None), 1), (dict(tokens=None), 1), (dict(logprob=None), 1), (dict(top_tokens=None), 1),
    (dict(top_logprobs=None), 1), (dict(logits=4097), 1), (dict(logits=4098, fp32=1), 1), (dict(tokens=4098), 1),
    (dict(logprob=4098), 1), (dict(entropy=4098), 1), (dict(top_tokens=4098), 1), (dict(top_logprobs=4098), 1)])
def test_refuses(lib, bad, status):
    with pytest.raises(H.HpdError) as e:
        H.hpd_token_logprobs(args(**bad), None)
    assert e.value.status == status


def test_no_rows_need_no_device(lib):
    H.hpd_token_logprobs(args(R=0, logits=None, tokens=None, logprob=None), None)


@pytest.mark.parametrize("R,V", [(1, 2 ** 32 + 100), (2, 2 ** 31), (3, 2 ** 30 + 1), (2 ** 32 + 5, 1), (2 ** 31, 1)])
def test_sizes_that_do_not_fit_the_call_are_refused(lib, monkeypatch, R, V):
    torch = pytest.importorskip("torch")
    made = []

    class OnDevice(torch.Tensor):
        is_cuda = property(lambda self: True)

    monkeypatch.setattr(H, "_need_current", lambda *a: None)
    monkeypatch.setattr(H, "_stream_handle", lambda s: None)
    monkeypatch.setattr(H, "hpd_token_logprobs", lambda a, s: made.append((a.R, a.V)))
    on = lambda *n, **kw: torch.empty(n, device="meta", **kw).as_subclass(OnDevice)  # noqa: E731
    with pytest.raises(H.HpdError) as e:
        H.token_logprobs(on(R, V, dtype=torch.bfloat16), on(R, dtype=torch.int32))
    assert e.value.status == 2 and not made
    H.token_logprobs(on(7, 2 ** 30, dtype=torch.bfloat16), on(7, dtype=torch.int32))
    assert made == [(7, 2 ** 30)]


def test_struct_layout_matches_the_header(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    k = H.hpd_token_logprobs_args
    body = "".join(f'  printf(" %zu", offsetof(hpd_token_logprobs_args, {f}));\n' for f, _ in k._fields_)
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "hpd.h"\nint main(void) {\n'
                   '  printf("%zu", sizeof(hpd_token_logprobs_args));\n' + body + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in got] == [ctypes.sizeof(k)] + [getattr(k, f).offset for f, _ in k._fields_]


@gpu
def test_tensors_of_the_wrong_kind_are_refused(torch):
    bf = torch.zeros(4, 100, dtype=torch.bfloat16, device="cuda")
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: H.token_logprobs(bf.half(), tok), lambda: H.token_logprobs(bf.cpu(), tok),
                lambda: H.token_logprobs(bf, tok.long()), lambda: H.token_logprobs(bf, tok[:3]),
                lambda: H.token_logprobs(bf, tok.cpu()), lambda: H.token_logprobs(bf[:, ::2], tok),
                lambda: H.token_logprobs(bf[:1].expand(4, 100), tok), lambda: H.token_logprobs(bf, tok, top=-1),
                lambda: H.token_logprobs(bf[:, :5], tok, top=6), lambda: H.token_logprobs(bf, tok, temperature=0.0),
                lambda: H.token_logprobs(bf, tok, temperature=-1.0), lambda: H.token_logprobs(bf, tok, temperature=2e36),
                lambda: H.token_logprobs(bf, tok, temperature=1e-37), lambda: H.token_logprobs(bf, tok, temperature=NAN),
                lambda: H.token_logprobs(bf.T, tok), lambda: H.token_logprobs(bf.view(2, 2, 100)[:, :, :50], tok.view(2, 2))):
        with pytest.raises(H.HpdError) as e:
            bad()
        assert e.value.status == 1
    with pytest.raises(H.HpdError) as e:
        H.token_logprobs(bf, tok, top=33)
    assert e.value.status == 2


def _check(torch, x, tokens, top=0, temperature=1.0, got=None):
    """x: the logits as a device tensor [R, V]."""
    r = got or H.token_logprobs(x, torch.from_numpy(np.asarray(tokens, np.int32)).cuda(), top=top, temperature=temperature)
    torch.cuda.synchronize()
    lp, ent, ids, alt = O.logprobs(x.float().cpu().numpy(), tokens, top, temperature)
    # (what lies beyond the largest number of 32 bits, 2^128 (1 - 2^-24), by half a step and more rounds to -inf)
    lp, alt = (np.where(a <= -2.0 ** 128 * (1 - 2.0 ** -25), -INF, a) for a in (lp, alt))
    # Z: exponentials to 2^-22 of each, whose arguments d (a difference, a factor, log2 e
    # and its product: 2^-24 of it each, four times) are off by 2^-22 |d|; terms with
    # |d| above 88 are no numbers of 32 bits.  Sums in 32 bits of V / 512 terms in a thread at most
    # and a tree: below 2^-19 with all these V.  A log probability is off by that much of
    # log Z and by 2^-22 of itself; the entropy by as much of its two positive terms.
    V = x.shape[1]
    z = 2.0 ** -21 + 88 * 2.0 ** -22 + 2.0 ** -24 * (V / 512 + 12)
    near = lambda a, b: (np.isnan(a) & np.isnan(b)) | (a == b) | (np.abs(a - b) <= z * np.minimum(-b, 30.0) + 2.0 ** -21 * np.abs(b) + 1e-36)  # noqa: E731
    got_lp, got_ent = r.logprob.cpu().numpy().reshape(-1), r.entropy.cpu().numpy().reshape(-1)
    assert near(got_lp, lp).all(), np.abs(got_lp - lp).max()
    same = (np.isnan(got_ent) & np.isnan(ent)) | (np.abs(got_ent - ent) <= 2 * z * np.abs(ent) + 1e-36)
    assert same.all(), (got_ent, ent)
    if top:
        assert np.array_equal(r.top_tokens.cpu().numpy().reshape(ids.shape), ids)
        got_alt = r.top_logprobs.cpu().numpy().reshape(alt.shape)
        assert near(got_alt, alt).all()
    else:
        assert r.top_tokens is None and r.top_logprobs is None
    return r


def _logits(torch, rng, R, V, wide, std=3.0, sure=0.0):
    x = rng.standard_normal((R, V)).astype(np.float32) * std
    x[np.arange(R), rng.integers(0, V, R)] += sure
    x = torch.from_numpy(x).cuda()
    return x if wide else x.to(torch.bfloat16)


@gpu
@pytest.mark.parametrize("R,V,top,wide", [
    (1, 1, 1, False), (1, 1, 0, True), (3, 2, 2, False), (2, 31, 31, True), (5, 33, 32, False), (4, 100, 5, True),
    (7, 4095, 20, False), (7, 4097, 32, True), (1, 32000, 8, False), (64, 32000, 0, False), (200, 1009, 20, True),
    (2, 100003, 20, False), (1, 151936, 32, True), (300, 32001, 5, False), (9, 65536, 1, True), (4, 260000, 32, False)])
@pytest.mark.parametrize("sure", [0.0, 25.0])
def test_gpu_logprobs(torch, R, V, top, wide, sure):
    rng = np.random.default_rng(R * 1000003 + V)
    x = _logits(torch, rng, R, V, wide, sure=sure)
    tokens = np.where(rng.random(R) < 0.6, x.float().argmax(1).cpu().numpy(), rng.integers(0, V, R))
    _check(torch, x, tokens, top, temperature=[1.0, 0.7, 2.5][R % 3])


@gpu
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("V,top", [(40, 32), (1000, 20), (32000, 32), (70001, 5)])
def test_gpu_rows_out_of_the_ordinary(torch, wide, V, top):
    rng = np.random.default_rng(V)
    x = np.zeros((14, V), np.float32)
    x[1:] = rng.standard_normal((13, V)) * 2
    x[1, 2:] = -INF                              # two that may be chosen
    x[2] = -INF                                  # none
    x[3, V // 2] = NAN
    x[4, V - 1] = INF
    x[5] = NAN
    x[6, 1:] = NAN                               # one that is a number
    x[7] = np.arange(V) * 0.125                  # the largest last
    x[8] = -np.arange(V) * 0.125
    x[9] = np.where(np.arange(V) % 7 == 3, 5.0, 4.0)      # many equal ones
    x[10] = np.where(rng.random(V) < 0.9, -INF, x[10])
    x[11] = np.where(np.arange(V) % 2, 0.0, -0.0)         # equal, whatever their sign
    x[12] = 1.5e38 * np.where(np.arange(V) == V // 3, 1, -1)
    x[13] = -3e38
    tokens = [0, 1, 0, 1, V - 1, 3, 0, V - 1, 0, 3, 5, 1, V // 3, 2]
    x = torch.from_numpy(x).cuda()
    _check(torch, x if wide else x.to(torch.bfloat16), tokens, top)


@gpu
@pytest.mark.parametrize("temperature", [1e36, 1e30, 1e-30, 1e-36])
@pytest.mark.parametrize("wide", [False, True])
def test_gpu_temperatures_out_of_the_ordinary(torch, wide, temperature):
    rng = np.random.default_rng(9)
    x = _logits(torch, rng, 6, 9001, wide)
    x[1, 5000:] = -INF
    x[2, 1:] = -INF
    x[3] = -3e38
    x[3, 77] = 3e38
    x[4] *= 2.0 ** 110
    x[5] *= 2.0 ** -100
    _check(torch, x, [3, 4, 5, 77, 6, 7], 5, temperature)


@gpu
def test_gpu_values_a_step_above_a_threads_first_ones(torch):
    # a step of the values is more than 60 powers of two at this temperature, and a thread
    # has some 2,900 values a step above its first ones: 2^117.6 each, were those its base
    x = torch.full((8, 750000), 1.0 + 2.0 ** -23, device="cuda")
    x[:, :4096] = 1.0
    _check(torch, x.view(1, -1), [5000000], 0, temperature=0.51 * 2.0 ** -23 / 60 / np.log(2.0))


def _check_lost(torch, x, tokens, top, temperature):
    """_check where many terms of a row are below 2^-126 and count as 0: the entropy loses up to
    (1 + |d|) 2^-126 of each, |d| at most 126 log 2 = 87.4 there (what is smaller loses less)."""
    r = H.token_logprobs(x, torch.from_numpy(np.asarray(tokens, np.int32)).cuda(), top=top, temperature=temperature)
    ent = torch.from_numpy(O.logprobs(x.float().cpu().numpy(), tokens, 0, temperature)[1]).cuda()
    lost = (r.entropy - ent).abs() <= x.shape[1] * 88.4 * 2.0 ** -126
    _check(torch, x, tokens, top, temperature, got=r._replace(entropy=torch.where(lost, ent, r.entropy)))


@gpu
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("R,V,top", [(300, 32000, 8), (5, 32000, 0), (6, 151936, 20), (1, 70001, 32)])
def test_gpu_values_far_below_zero_behind_those_that_have_none(torch, wide, R, V, top):
    # a thread's first values are -inf, and those that follow are small: e^x is no number of 32 bits
    rng = np.random.default_rng(R + V)
    at = np.arange(V)
    few = [rng.choice(V, V // 100, replace=False) for _ in range(R)]
    some = np.zeros((R, V), bool)
    for r, i in enumerate(few):
        some[r, i] = True
    for allowed, mean, std, temperature in (
            (at >= 10000, -100.0, 2.0, 1.0), (at >= 10000, -12.0, 2.0, 0.1), (at >= V - 300, -82.0, 1.0, 1.0),
            (some, 0.0, 4.0, 0.1), (some, -1.0, 3.0, 0.02), (some | (at < 3), -3e4, 1.0, 1.0)):
        x = rng.standard_normal((R, V)).astype(np.float32) * std + np.float32(mean)
        x = torch.from_numpy(np.where(allowed, x, -INF).astype(np.float32)).cuda()
        tokens = np.where(rng.random(R) < 0.7, x.argmax(1).cpu().numpy(), rng.integers(0, V, R))
        _check_lost(torch, x if wide else x.to(torch.bfloat16), tokens, top, temperature)


@gpu
@pytest.mark.parametrize("wide", [False, True])
def test_gpu_a_few_values_far_below_zero(torch, wide):
    # rows without a piece of 16 bytes, and with a value or more on either side of the pieces
    rng = np.random.default_rng(11)
    for V in list(range(1, 20)) + [2049, 8195]:
        for shift in range(4):
            whole = torch.from_numpy(rng.standard_normal((4, V + 9)).astype(np.float32) - 100).cuda()
            x = (whole if wide else whole.to(torch.bfloat16))[:, shift: shift + V]
            _check(torch, x, rng.integers(0, V, 4), min(V, 5))


@gpu
def test_gpu_tokens_that_are_none(torch):
    x = _logits(torch, np.random.default_rng(1), 6, 500, False)
    x[5, 7] = NAN
    r = _check(torch, x, [-1, 500, 499, -(1 << 31), (1 << 31) - 1, -1])
    assert torch.isneginf(r.logprob).tolist() == [True, True, False, True, True, False]


@gpu
@pytest.mark.parametrize("wide", [False, True])
def test_gpu_strided_rows_at_odd_addresses(torch, wide):
    rng = np.random.default_rng(4)
    for V, extra, shift in ((1000, 24, 0), (1001, 6, 1), (999, 1, 3), (4000, 1, 5), (37, 40, 7)):
        whole = _logits(torch, rng, 8, V + extra + 8, wide)
        x = whole[:, shift: shift + V]
        keep = whole.clone()
        _check(torch, x, rng.integers(0, V, 8), top=10)
        assert torch.equal(whole, keep)


@gpu
def test_gpu_leading_extents(torch):
    rng = np.random.default_rng(5)
    x = _logits(torch, rng, 12, 3000, False)
    tok = rng.integers(0, 3000, 12)
    t = torch.from_numpy(tok.astype(np.int32)).cuda()
    r = H.token_logprobs(x.view(3, 4, 3000), t.view(3, 4), top=5)
    assert r.logprob.shape == r.entropy.shape == (3, 4) and r.top_tokens.shape == r.top_logprobs.shape == (3, 4, 5)
    _check(torch, x, tok, 5, got=r)
    one = H.token_logprobs(x[0], t[0], top=2)
    assert one.logprob.shape == () and one.top_tokens.shape == (2,)
    assert torch.equal(one.logprob, r.logprob[0, 0]) and torch.equal(one.top_tokens, r.top_tokens[0, 0, :2])
    empty = H.token_logprobs(x[:0], t[:0], top=2)
    assert empty.logprob.shape == (0,) and empty.top_logprobs.shape == (0, 2)


@gpu
def test_gpu_a_calls_bits_stay_and_the_number_of_rows_is_large(torch):
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(70001, 130, generator=gen, device="cuda").to(torch.bfloat16)
    t = torch.randint(0, 130, (70001,), generator=gen, device="cuda", dtype=torch.int32)
    a, b = (H.token_logprobs(x, t, top=3) for _ in range(2))
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    pick = torch.tensor([0, 1, 65535, 65536, 70000], device="cuda")
    _check(torch, x[pick], t[pick].tolist(), 3, got=H.TokenLogprobs(*(p[pick] for p in a)))


@gpu
def test_gpu_rows_beyond_32_bits(torch):
    # the last rows lie past 2^32 bytes and 2^31 values
    V, R = 262144, 8300
    x = torch.zeros(R, V, dtype=torch.bfloat16, device="cuda")
    x[-2:] = _logits(torch, np.random.default_rng(8), 2, V, False)
    t = torch.full((R,), 5, dtype=torch.int32, device="cuda")
    r = H.token_logprobs(x, t, top=4)
    _check(torch, x[-2:], [5, 5], 4, got=H.TokenLogprobs(*(p[-2:] for p in r)))
    assert torch.equal(r.top_tokens[0].cpu(), torch.arange(4, dtype=torch.int32))


@gpu
def test_gpu_on_another_stream_and_in_a_graph(torch):
    rng = np.random.default_rng(6)
    x = _logits(torch, rng, 20, 20000, False)
    t = torch.from_numpy(rng.integers(0, 20000, 20).astype(np.int32)).cuda()
    want = H.token_logprobs(x, t, top=7)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = H.token_logprobs(x, t, top=7, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = H.token_logprobs(x, t, top=7)
    x2 = _logits(torch, rng, 20, 20000, False)
    x.copy_(x2)
    g.replay()
    torch.cuda.synchronize()
    _check(torch, x2, t.cpu().numpy(), 7, got=held)


@gpu
def test_gpu_after_the_acceptance(torch):
    # the tokens that the verification of a step returns, with its logits
    rng = np.random.default_rng(7)
    B, m, V = 5, 4, 8000
    x = _logits(torch, rng, B * m, V, False).view(B, m, V)
    drafts = torch.from_numpy(rng.integers(0, V, (B, m)).astype(np.int32)).cuda()
    tokens, _ = H.pmtp_accept(x, drafts)
    r = H.token_logprobs(x, tokens, top=1)
    _check(torch, x.view(-1, V), tokens.view(-1).tolist(), 1, got=r)
    assert torch.equal(r.top_tokens[..., 0], tokens) and torch.equal(r.top_logprobs[..., 0], r.logprob)
