"""What is measured of the operators that write a chunk of new tokens into the
paged KV cache and attend from it: their cases, inputs, work and definitions.

A page's prefix (vision tokens, then layout tokens) has to be in the paged
cache before its branches decode.  A program that puts it there makes three
calls: ``ChunkSlots`` (pages and slots of the new tokens of every sequence,
from the lengths alone, once a step), ``QkNormRope`` (per-head RMS norms of
queries and keys with the rotation by their positions, keys and values
written to their slots, once a layer) and ``ChunkAttn`` (the chunk's attention
over the paged cache, once a layer).  Sequences of one new token, the form of
ordinary decoding, go through the same calls.

Lengths come from the case alone (``len_seed``), so that the work does not
depend on the seed of the inputs; values, positions' offsets and the physical
order of the pages come from that seed.  Sizes are those of the presets of
``workloads.py`` and of the test suite, or generic.
"""
import functools
import json
import math

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1e-6
#: no drawn case costs more than the largest listed ones, or has larger padded scores or keys (bytes, 32 bits) in its
#: plain form
MAX_FLOPS, MAX_BYTES, MAX_SCORES, MAX_KEYS = 5.1e11, 1.2e9, 4.4e9, 2.2e9


# ---------------------------------------------------------------- the cases --

def _slots(name, **kw):
    case = dict(name=name, kind="slots", seqs=4, new_lo=1, new_hi=32, ctx_lo=0, ctx_hi=100, single=0.0,
                max_pages=64, len_seed=1)
    case.update(kw)
    return case


def _rope(name, **kw):
    case = dict(name=name, kind="rope", tokens=64, hq=16, hkv=2, d=128, axes=1, pad=0, max_pos=8192)
    case.update(kw)
    return case


def _attn(name, **kw):
    case = dict(name=name, kind="attn", seqs=1, new_lo=1, new_hi=1, ctx_lo=255, ctx_hi=255, single=0.0, hq=16,
                hkv=2, d=128, prefix_mask=False, len_seed=1)
    case.update(kw)
    return case


def _step(name, **kw):
    case = dict(name=name, kind="step", layers=4, seqs=4, new_lo=1152, new_hi=1152, ctx_lo=0, ctx_hi=0, single=0.0,
                hq=16, hkv=2, d=128, axes=3, max_pos=8192, len_seed=1)
    case.update(kw)
    return case


def listed():
    return [
        # the pages of a few short requests: latency alone
        _slots("slots_few"),
        # the pages of a large serving batch: prompts of all lengths among
        # requests that decode one token
        _slots("slots_batch", seqs=512, new_lo=0, new_hi=500, ctx_lo=0, ctx_hi=7000, single=0.5, max_pages=512,
               len_seed=2),
        # the tokens of one decode step of one page: 16 branches of 4
        _rope("rope_decode_step"),
        # vision tokens of three pages with rows of a wider projection, whose
        # positions have a time, a height and a width
        _rope("rope_vision_pages", tokens=3 * 1024 + 129, hq=32, hkv=8, axes=3, pad=64),
        # a large prefill, an odd number of tokens
        _rope("rope_long_prefill", tokens=32749, hq=16, hkv=2, max_pos=32768),
        # one new token of one short sequence: the smallest call
        _attn("attn_one_token", hq=8, hkv=2, d=64),
        # a batch that decodes one token a sequence, contexts of all lengths
        # (bound by the memory of keys and values)
        _attn("attn_token_batch", seqs=64, ctx_lo=100, ctx_hi=8191, hq=32, hkv=8, len_seed=3),
        # one page: 1,024 vision tokens that see one another, 128 layout
        # tokens that see what is before them
        _attn("attn_one_page", new_lo=1152, new_hi=1152, ctx_lo=0, ctx_hi=0, prefix_mask=True),
        # a chunk of a very long document (the largest case by operations)
        _attn("attn_long_chunk", new_lo=2048, new_hi=2048, ctx_lo=14336, ctx_hi=14336, hq=32, hkv=8),
        # a serving batch whose chunks are ragged, half of them single tokens
        # and some empty, with a head ratio that does not divide a tile
        _attn("attn_mixed_batch", seqs=24, new_lo=0, new_hi=300, ctx_lo=0, ctx_hi=3000, single=0.5, hq=40, hkv=8,
              len_seed=4),
        # short heads, several pages at once
        _attn("attn_head_64", seqs=6, new_lo=500, new_hi=1200, ctx_lo=0, ctx_hi=1000, hq=16, hkv=4, d=64,
              len_seed=5),
        # four pages read in through four layers: the three operators as they
        # are used together
        _step("step_prefill"),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    kind = rng.choice(["slots", "rope", "rope", "attn", "attn", "attn", "attn", "step"])
    seed = rng.randrange(1 << 20)
    heads = rng.choice([(8, 2), (16, 2), (32, 8), (16, 4), (40, 8), (6, 2), (16, 16), (14, 2), (32, 2)])
    d = rng.choice([64, 128, 128])
    while True:
        if kind == "slots":
            pages = rng.choice([64, 130, 512])
            hi = log(1, 500)
            case = _slots("", seqs=log(1, 512), new_lo=rng.choice([0, 1]), new_hi=hi, ctx_hi=pages * PAGE - hi,
                          single=rng.choice([0.0, 0.5, 1.0]), max_pages=pages, len_seed=seed)
        elif kind == "rope":
            case = _rope("", tokens=log(1, 20000), hq=heads[0], hkv=heads[1], d=d, axes=rng.choice([1, 3]),
                         pad=rng.choice([0, 8, 64]), max_pos=32768)
        elif kind == "attn":
            ctx, new = log(1, 12000), log(1, 2048)
            case = _attn("", seqs=log(1, 64), new_lo=rng.choice([0, 1, new]), new_hi=new, ctx_lo=rng.choice([0, ctx]),
                         ctx_hi=ctx, single=rng.choice([0.0, 0.0, 0.5, 1.0]), hq=heads[0], hkv=heads[1], d=d,
                         prefix_mask=rng.random() < 0.3, len_seed=seed)
        else:
            case = _step("", layers=rng.choice([1, 2, 4]), seqs=log(1, 8), new_lo=1, new_hi=log(16, 1200),
                         ctx_hi=log(1, 1500), single=rng.choice([0.0, 0.5]), hq=heads[0], hkv=heads[1], d=d,
                         axes=rng.choice([1, 3]), len_seed=seed)
        del case["name"]
        if case["kind"] == "rope":
            return case
        new, ctx = _lengths(case)
        if new.sum() < 1:
            seed += 1
            continue
        if case["kind"] == "slots" or (
                4 * len(new) * case["hq"] * int(new.max()) * int((new + ctx).max()) <= MAX_SCORES
                and 4 * len(new) * int((new + ctx).max()) * case["hkv"] * case["d"] <= MAX_KEYS
                and work(case)["flops"] <= MAX_FLOPS and work(case)["bytes"] <= MAX_BYTES):
            return case


@functools.lru_cache(maxsize=None)
def _lengths_of(text):
    case = json.loads(text)
    rng = np.random.default_rng(7919 + case["len_seed"])
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, case["seqs"])
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, case["seqs"])
    return np.where(rng.random(case["seqs"]) < case["single"], 1, new), ctx


def _lengths(case):
    """New tokens and tokens already cached of every sequence."""
    keys = ("len_seed", "new_lo", "new_hi", "ctx_lo", "ctx_hi", "seqs", "single")
    return _lengths_of(json.dumps({k: case[k] for k in keys}))


def _full(case, seqs, total):
    """Keys that every query of a sequence sees (its vision tokens)."""
    if case["seqs"] == 1:
        return np.minimum(total, 1024)
    return np.random.default_rng(104729 + case["len_seed"]).integers(0, total + 1)


# --------------------------------------------------------------- the inputs --

class _Maker:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(int(seed))

    def normal(self, *shape, std=0.5, mean=0.0):
        x = torch.empty(shape, dtype=torch.bfloat16, device=self.dev)
        return x.normal_(mean, std, generator=self.gen)

    def perm(self, n):
        return torch.randperm(n, generator=self.gen, device=self.dev, dtype=torch.int32)

    def ints(self, a):
        return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=self.dev)


def _table(mk, pages_of, max_pages, ids):
    """[seqs][max_pages] page ids, -1 past a sequence's pages."""
    count = mk.ints(pages_of)
    first = torch.cumsum(count, 0, dtype=torch.int32) - count
    j = torch.arange(max_pages, device=mk.dev, dtype=torch.int32)
    at = (first[:, None] + j).clamp(max=ids.numel() - 1)
    return torch.where(j < count[:, None], ids[at.long()], -1).to(torch.int32).contiguous()


def _rotation(max_pos, d, dev):
    """cos and sin of position * 1e6^(-2 i / d), [max_pos][d / 2][2], 32 bits."""
    i = torch.arange(d // 2, device=dev, dtype=torch.float64)
    a = torch.arange(max_pos, device=dev, dtype=torch.float64)[:, None] * 1e6 ** (-2.0 * i / d)
    return torch.stack((a.cos(), a.sin()), -1).float().contiguous()


def _sections(axes, d):
    """Frequencies of each axis: all, or a quarter for time and the rest for height and width."""
    h = d // 2
    return (h,) if axes == 1 else (h // 4, (h - h // 4) // 2, h - h // 4 - (h - h // 4) // 2)


def _positions(mk, axes, pos, max_pos):
    """Text positions as they are; images in grids of 32 x 32 with a time, a height and a width."""
    if axes == 1:
        return pos[None].contiguous()
    t = pos // 1024
    return torch.stack((t, t + (pos % 1024) // 32, t + pos % 32)).clamp(max=max_pos - 1).to(torch.int32).contiguous()


def _seq_state(mk, case, max_pages):
    """Sequences with their cached pages and a stack of free ones."""
    new, ctx = _lengths(case)
    held = (ctx + PAGE - 1) // PAGE
    need = (ctx + new + PAGE - 1) // PAGE - held
    num_pages = int(held.sum() + need.sum()) + 13
    ids = mk.perm(num_pages)
    n_held = int(held.sum())
    return dict(new_len=mk.ints(new), seq_len=mk.ints(ctx), page_table=_table(mk, held, max_pages, ids[:max(n_held, 1)]),
                free_pages=torch.nn.functional.pad(ids[n_held:], (0, n_held)).contiguous(),
                free_top=mk.ints([num_pages - n_held]), num_pages=num_pages, tokens=int(new.sum()))


def prepare(case, seed):
    mk = _Maker(seed)
    kind = case["kind"]
    if kind == "slots":
        return dict(case=case, **_seq_state(mk, case, case["max_pages"]))
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    st = dict(case=case)
    if kind in ("rope", "step"):
        st.update(q_weight=mk.normal(d, std=0.1, mean=1.0), k_weight=mk.normal(d, std=0.1, mean=1.0),
                  table=_rotation(case["max_pos"], d, mk.dev), sections=_sections(case["axes"], d),
                  axis=mk.ints(np.repeat(np.arange(case["axes"]), _sections(case["axes"], d))))
    if kind == "rope":
        T = case["tokens"]
        num_pages = -(-T // PAGE) + 5
        at = torch.arange(T, device=mk.dev, dtype=torch.int32)
        slot = mk.perm(num_pages)[(at // PAGE).long()] * PAGE + at % PAGE
        shift = int(torch.randint(0, max(1, case["max_pos"] - T), (1,), generator=mk.gen, device=mk.dev))
        st.update(qkv=mk.normal(T, (hq + 2 * hkv) * d + case["pad"], std=1.0), slot=slot.to(torch.int32),
                  pos=_positions(mk, case["axes"], at + shift, case["max_pos"]),
                  k_cache=mk.normal(num_pages, PAGE, hkv, d), v_cache=mk.normal(num_pages, PAGE, hkv, d))
        return st
    new, ctx = _lengths(case)
    total = new + ctx
    max_pages = max(1, -(-int(total.max()) // PAGE))
    st.update(max_new=int(new.max()), max_len=int(total.max()))
    if kind == "attn":
        pages = (total + PAGE - 1) // PAGE
        num_pages = int(pages.sum()) + 3
        # (queries and keys have the size that their norms leave them)
        st.update(q=mk.normal(int(new.sum()), hq, d, std=1.0), k_cache=mk.normal(num_pages, PAGE, hkv, d, std=1.0),
                  v_cache=mk.normal(num_pages, PAGE, hkv, d),
                  page_table=_table(mk, pages, max_pages, mk.perm(num_pages)), seq_len=mk.ints(total),
                  chunk_cu=mk.ints(np.concatenate(([0], np.cumsum(new)))),
                  full_len=mk.ints(_full(case, len(new), total)) if case["prefix_mask"] else None)
        return st
    st.update(_seq_state(mk, case, max_pages))
    T, at = st["tokens"], torch.arange(st["tokens"], device=mk.dev, dtype=torch.int32)
    at = at - torch.repeat_interleave(mk.ints(np.cumsum(new) - new), mk.ints(new), output_size=T)
    st["pos"] = _positions(mk, case["axes"], at + torch.repeat_interleave(mk.ints(ctx), mk.ints(new), output_size=T),
                           case["max_pos"])
    st["layers"] = [dict(qkv=mk.normal(T, (hq + 2 * hkv) * d, std=1.0),
                         k_cache=mk.normal(st["num_pages"], PAGE, hkv, d, std=1.0),
                         v_cache=mk.normal(st["num_pages"], PAGE, hkv, d)) for _ in range(case["layers"])]
    return st


# ------------------------------------------------------- the plain operators --

def _plain_slots(new_len, seq_len, page_table, free_pages, free_top, tokens):
    n, L = new_len.long(), seq_len.long()
    cu = torch.cat((n.new_zeros(1), torch.cumsum(n, 0)))
    held, need = (L + PAGE - 1) // PAGE, (L + n + PAGE - 1) // PAGE
    taken = torch.cumsum(need - held, 0)
    first = free_top.long() - taken[-1] + taken - (need - held)  # place of a sequence's first page on the stack
    j = torch.arange(page_table.shape[1], device=n.device)
    ids = free_pages[(first[:, None] + j - held[:, None]).clamp(0, free_pages.numel() - 1)]
    table = torch.where((j >= held[:, None]) & (j < need[:, None]), ids, page_table)
    t = torch.arange(tokens, device=n.device)
    s = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    pos = L[s] + t - cu[s]
    slot = table[s, pos // PAGE].long() * PAGE + pos % PAGE
    i32 = torch.int32
    return dict(chunk_cu=cu.to(i32), slot=slot.to(i32), pos=pos.to(i32), seq_len=(L + n).to(i32),
                free_top=(free_top.long() - taken[-1]).to(i32), page_table=table)


def _plain_norm_rope(x, weight, cos, sin):
    """x [T][H][D] normed over D, then rotated in pairs (i, i + D / 2)."""
    x = x.float()
    x = x * torch.rsqrt(torch.mean(x * x, -1, keepdim=True) + EPS) * weight.float()
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(torch.bfloat16)


def _plain_rope(case, qkv, q_weight, k_weight, table, axis, pos, slot, k_cache, v_cache):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = qkv[:, : (hq + 2 * hkv) * d].reshape(qkv.shape[0], hq + 2 * hkv, d)
    rot = table[pos.long()[axis.long()].T, torch.arange(d // 2, device=qkv.device)]  # [T][D / 2][2]
    cos, sin = rot[:, None, :, 0], rot[:, None, :, 1]
    k_cache.view(-1, hkv, d)[slot.long()] = _plain_norm_rope(x[:, hq: hq + hkv], k_weight, cos, sin)
    v_cache.view(-1, hkv, d)[slot.long()] = x[:, hq + hkv:]
    return _plain_norm_rope(x[:, :hq], q_weight, cos, sin)


def _plain_attn(case, q, k_cache, v_cache, page_table, seq_len, chunk_cu, full_len, max_new, max_len):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    dev, T = q.device, q.shape[0]
    cu, L = chunk_cu.long(), seq_len.long()
    n = cu[1:] - cu[:-1]
    i, j = torch.arange(max_new, device=dev), torch.arange(max_len, device=dev)
    x = q[(cu[:-1, None] + i).clamp(max=T - 1)].float()  # [S][n][Hq][D], padded
    x = x.view(-1, max_new, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(len(n), hkv, -1, d)
    at = (page_table[:, j // PAGE].long().clamp(min=0) * PAGE + j % PAGE)
    k = k_cache.view(-1, hkv, d)[at].float().permute(0, 2, 3, 1)
    v = v_cache.view(-1, hkv, d)[at].float().permute(0, 2, 1, 3)
    seen = (L - n)[:, None] + i + 1
    if full_len is not None:
        seen = torch.maximum(seen, full_len.long()[:, None])
    seen = torch.minimum(seen, L[:, None])
    mask = j < seen[:, :, None]  # [S][n][L]
    s = torch.matmul(x, k).view(len(n), hkv, hq // hkv, max_new, max_len) * (1.0 / math.sqrt(d))
    s = s.masked_fill_(~mask[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    o = torch.matmul(p.view(len(n), hkv, -1, max_len), v).view(len(n), hkv, hq // hkv, max_new, d)
    o = torch.where(total > 0, o / total, 0.0)
    t = torch.arange(T, device=dev)
    sq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    o = o.permute(0, 3, 1, 2, 4)[sq, t - cu[sq]].reshape(T, hq, d)
    return o.to(torch.bfloat16), lse.permute(0, 3, 1, 2)[sq, t - cu[sq]].reshape(T, hq)


def _plain(st):
    case = st["case"]
    rope = ("q_weight", "k_weight", "table", "axis")
    if case["kind"] == "slots":
        return _plain_slots(*(st[k] for k in ("new_len", "seq_len", "page_table", "free_pages", "free_top", "tokens")))
    if case["kind"] == "rope":
        q = _plain_rope(case, st["qkv"], *(st[k] for k in rope + ("pos", "slot", "k_cache", "v_cache")))
        return dict(q=q, k_cache=st["k_cache"], v_cache=st["v_cache"])
    if case["kind"] == "attn":
        out, lse = _plain_attn(case, *(st[k] for k in ("q", "k_cache", "v_cache", "page_table", "seq_len", "chunk_cu",
                                                       "full_len", "max_new", "max_len")))
        return dict(out=out, lse=lse)
    sl = _plain_slots(*(st[k] for k in ("new_len", "seq_len", "page_table", "free_pages", "free_top", "tokens")))
    got = dict(sl)
    for k, la in enumerate(st["layers"]):
        q = _plain_rope(case, la["qkv"], *(st[k] for k in rope + ("pos",)), sl["slot"], la["k_cache"], la["v_cache"])
        got["out%d" % k], got["lse%d" % k] = _plain_attn(
            case, q, la["k_cache"], la["v_cache"], sl["page_table"], sl["seq_len"], sl["chunk_cu"], None,
            st["max_new"], st["max_len"])
        got["k_cache%d" % k], got["v_cache%d" % k] = la["k_cache"], la["v_cache"]
    return got


# --------------------------------------------------- the framework's operators --

def _handles(st):
    """The call objects with their outputs and workspaces, which a program makes once."""
    from paper_2607_18839_gb300 import hpd
    case, ops = st["case"], {}
    if case["kind"] in ("slots", "step"):
        # (the lengths and the stack's top of the next step go to buffers of
        # their own, so that a pass can be made again)
        ops["slots"] = hpd.ChunkSlots(st["page_table"], st["seq_len"], st["free_pages"], st["free_top"],
                                      max_tokens=st["tokens"], in_place=False)
    if case["kind"] in ("rope", "step"):
        ops["rope"] = hpd.QkNormRope(case["hq"], case["hkv"], case["d"], st["q_weight"], st["k_weight"], st["table"],
                                     sections=st["sections"], eps=EPS)
    if case["kind"] in ("attn", "step"):
        new, ctx = _lengths(case)
        ops["attn"] = [hpd.ChunkAttn(case["hq"], la["k_cache"], la["v_cache"], st["page_table"],
                                     max_tokens=int(new.sum()), max_seq_len=st["max_len"])
                       for la in st.get("layers", [st])]
    return ops


def _call(st):
    case = st["case"]
    if "ops" not in st:
        st["ops"] = _handles(st)
    ops = st["ops"]
    if case["kind"] == "rope":
        q = ops["rope"](st["qkv"], st["pos"], st["slot"], st["k_cache"], st["v_cache"])
        return dict(q=q, k_cache=st["k_cache"], v_cache=st["v_cache"])
    if case["kind"] == "attn":
        out, lse = ops["attn"][0](st["q"], st["chunk_cu"], st["seq_len"], st["full_len"])
        return dict(out=out, lse=lse)
    c = ops["slots"](st["new_len"])
    got = dict(chunk_cu=c.chunk_cu, slot=c.slot, pos=c.pos, seq_len=c.seq_len, free_top=c.free_top,
               page_table=c.page_table)
    for k, la in enumerate(st.get("layers", ())):
        q = ops["rope"](la["qkv"], st["pos"], c.slot, la["k_cache"], la["v_cache"])
        got["out%d" % k], got["lse%d" % k] = ops["attn"][k](q, c.chunk_cu, c.seq_len)
        got["k_cache%d" % k], got["v_cache%d" % k] = la["k_cache"], la["v_cache"]
    return got


def run(state):
    return _call(state) if own else _plain(state)


# ----------------------------------------------------------------- the work --

def _work_slots(new, ctx):
    need = (ctx + new + PAGE - 1) // PAGE - (ctx + PAGE - 1) // PAGE
    open_page = np.count_nonzero((ctx % PAGE > 0) & (new > 0))
    # lengths twice in, offsets and lengths out, a page's id read and written, a slot and a position a token
    return 4 * (4 * len(new) + 2 * int(need.sum()) + open_page + 2 * int(new.sum()) + 3), 0


def _work_rope(case, T):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    rows = 2 * 2 * T * (hq + 2 * hkv) * d
    # a norm is 3 operations a value, its weight 1, the rotation 3
    return rows + 4 * T * (case["axes"] + 1) + 4 * d * min(T, case["max_pos"]) + 4 * d, 7 * T * (hq + hkv) * d


def _work_attn(case, new, ctx, full):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    keys = np.where(new > 0, new + ctx, 0)
    pairs = 0
    for n, c, f in zip(new.tolist(), ctx.tolist(), full.tolist()):
        low = max(0, min(n, f - c))  # queries that the prefix mask gives more than their own past
        pairs += low * f + (n - low) * c + (n * (n + 1) - low * (low + 1)) // 2
    T = int(new.sum())
    nbytes = 2 * 2 * int(keys.sum()) * hkv * d + 2 * 2 * T * hq * d + 4 * T * hq + 4 * int(((keys + 15) // 16).sum())
    return nbytes + 12 * len(new), 4 * pairs * hq * d


def work(case):
    if case["kind"] == "rope":
        b, f = _work_rope(case, case["tokens"])
    else:
        new, ctx = _lengths(case)
        if case["kind"] == "slots":
            b, f = _work_slots(new, ctx)
        elif case["kind"] == "attn":
            full = _full(case, len(new), new + ctx) if case["prefix_mask"] else np.zeros_like(new)
            b, f = _work_attn(case, new, ctx, full)
        else:
            b, f = _work_slots(new, ctx)
            rb, rf = _work_rope(case, int(new.sum()))
            ab, af = _work_attn(case, new, ctx, np.zeros_like(new))
            b, f = b + case["layers"] * (rb + ab), f + case["layers"] * (rf + af)
    return {"bytes": int(b), "flops": int(f)}


# ------------------------------------------------------ the results in 64 bits --

def _exact_rope(case, st, qkv, pos, slot, k_cache, v_cache):
    """Rotated queries, and the caches as they are after the call, 64 bits."""
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    axis = sum(([a] * c for a, c in enumerate(st["sections"])), [])
    table, pos = st["table"].double(), pos.long()
    cos = torch.stack([table[pos[axis[i]], i, 0] for i in range(d // 2)], 1)
    sin = torch.stack([table[pos[axis[i]], i, 1] for i in range(d // 2)], 1)

    def turn(x, w):
        x = x.double() / (x.double().pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
        z = torch.complex(x[..., : d // 2], x[..., d // 2:]) * torch.complex(cos, sin)[:, None]
        return torch.cat((z.real, z.imag), -1)

    heads = [qkv[:, h * d: (h + 1) * d] for h in range(hq + 2 * hkv)]
    q = turn(torch.stack(heads[:hq], 1), st["q_weight"])
    k, v = k_cache.double().reshape(-1, hkv, d), v_cache.double().reshape(-1, hkv, d)
    k.index_copy_(0, slot.long(), turn(torch.stack(heads[hq: hq + hkv], 1), st["k_weight"]))
    v.index_copy_(0, slot.long(), torch.stack(heads[hq + hkv:], 1).double())
    return q, k.view(k_cache.shape), v.view(v_cache.shape)


def _exact_attn(case, q, k_cache, v_cache, table, new, ctx, full):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    g = hq // hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    t = 0
    for s, (n, c) in enumerate(zip(new.tolist(), ctx.tolist())):
        if n == 0:
            continue
        pages = table[s, : -(-(n + c) // PAGE)].long()
        last = torch.arange(c, c + n, device=q.device).clamp(min=int(full[s]) - 1)
        hidden = torch.arange(n + c, device=q.device)[None] > last[:, None]
        for h in range(hq):
            if h % g == 0:
                k = k_cache[pages, :, h // g].reshape(-1, d)[: n + c].double()
                v = v_cache[pages, :, h // g].reshape(-1, d)[: n + c].double()
            x = (q[t: t + n, h].double() @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[t: t + n, h] = torch.logsumexp(x, -1)
            out[t: t + n, h] = torch.softmax(x, -1) @ v
        t += n
    return out, lse


def exact(case, seed):
    if case["kind"] == "slots":
        return None
    st = prepare(case, seed)
    if case["kind"] == "rope":
        q, k, v = _exact_rope(case, st, st["qkv"], st["pos"], st["slot"], st["k_cache"], st["v_cache"])
        return dict(q=q, k_cache=k, v_cache=v)
    new, ctx = _lengths(case)
    if case["kind"] == "attn":
        full = _full(case, len(new), new + ctx) if case["prefix_mask"] else np.zeros_like(new)
        out, lse = _exact_attn(case, st["q"], st["k_cache"], st["v_cache"], st["page_table"], new, ctx, full)
        return dict(out=out, lse=lse)
    # the pages that the sequences get, one after another
    got = dict.fromkeys(("chunk_cu", "slot", "pos", "seq_len", "free_top", "page_table"))
    table, free = st["page_table"].cpu().numpy().copy(), st["free_pages"].cpu().numpy()
    held, need = -(-ctx // PAGE), -(-(ctx + new) // PAGE)
    at = int(st["free_top"].item()) - int((need - held).sum())
    slot = []
    for s in range(len(new)):
        for j in range(held[s], need[s]):
            table[s, j] = free[at]
            at += 1
        slot += [int(table[s, p // PAGE]) * PAGE + p % PAGE for p in range(ctx[s], ctx[s] + new[s])]
    slot, table = torch.tensor(slot, device="cuda"), torch.as_tensor(table, device="cuda")
    for i, la in enumerate(st["layers"]):
        q, k, v = _exact_rope(case, st, la["qkv"], st["pos"], slot, la["k_cache"], la["v_cache"])
        got["k_cache%d" % i], got["v_cache%d" % i] = k, v
        # the attention is of the rounded queries and keys, as the cache holds them
        got["out%d" % i], got["lse%d" % i] = _exact_attn(
            case, q.bfloat16(), k.bfloat16(), v.bfloat16(), table, new, ctx, np.zeros_like(new))
    return got
