"""Chunks of new tokens over the paged cache at their edges: sizes at a limit,
calls of no rows and of one, tensors that share their storage, streams, values
that are not finite among long contexts."""
import contextlib
import os
import re

import pytest

from paper_2607_18839_gb300 import build as B
from paper_2607_18839_gb300 import hpd as H

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


# --------------------------------------------------- norms, rotation, write --

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
