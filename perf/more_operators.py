"""What is measured of the paged cache held in 8 bits (its writing and the
attention that reads it) and of the log probabilities that a step reports:
their cases, inputs, work and definitions.

A cache of 8-bit codes (e4m3) with a scale for each page of 16 tokens and each
head takes half the memory of a bf16 one, and half the reading that bounds
decoding.  A program that keeps one makes, in every layer, two calls:
``QkNormRope`` with ``k_scale`` and ``v_scale`` (per-head RMS norms, rotation,
keys and values to the cache as codes) and ``ChunkAttn`` with the same two
(the new tokens' attention over it).  At the step's end ``token_logprobs``
gives the log probability of every token that was chosen, the entropy of its
distribution and the likeliest alternatives, which tell a reader of the parsed
page how far to trust it.

A page's scale is set when its first row is written, to the largest value
written by that call over 448; a later call that brings a larger value doubles
the scale as often as needed, so that the codes already there are halved that
often and (but for the smallest) not rounded again.

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
CODE_MAX = 448.0           # the largest e4m3 value
LEAST_SCALE = 2.0 ** -100  # of a page of zeros
#: no drawn case costs more than the largest listed ones, or has larger padded scores or keys (bytes, 32 bits) in its
#: plain form
MAX_FLOPS, MAX_BYTES, MAX_SCORES, MAX_KEYS = 5.1e11, 1.2e9, 4.4e9, 2.2e9


# ---------------------------------------------------------------- the cases --

def _write(name, **kw):
    case = dict(name=name, kind="write", seqs=16, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=40, single=0.0, hq=16, hkv=2,
                d=128, axes=1, pad=0, max_pos=8192, len_seed=1)
    case.update(kw)
    return case


def _attn(name, **kw):
    case = dict(name=name, kind="attn", seqs=1, new_lo=1, new_hi=1, ctx_lo=255, ctx_hi=255, single=0.0, hq=16,
                hkv=2, d=128, prefix_mask=False, len_seed=1)
    case.update(kw)
    return case


def _logp(name, **kw):
    case = dict(name=name, kind="logp", rows=64, vocab=32000, wide=False, top=0, banned=0.0, temperature=1.0)
    case.update(kw)
    return case


def _step(name, **kw):
    case = dict(name=name, kind="step", layers=4, seqs=24, new_lo=1, new_hi=1, ctx_lo=100, ctx_hi=4000, single=0.0,
                hq=16, hkv=2, d=128, axes=1, max_pos=8192, vocab=32000, top=5, len_seed=1)
    case.update(kw)
    return case


def listed():
    return [
        # one token of each of a few sequences into short heads: latency alone
        _write("write_few_tokens", hq=8, hkv=2, d=64),
        # a large batch that decodes: each token joins a page that has rows,
        # whose codes are halved where the token's values are larger
        _write("write_decode_batch", seqs=256, hq=32, hkv=8, len_seed=2),
        # vision tokens of three pages with rows of a wider projection, whose
        # positions have a time, a height and a width
        _write("write_vision_pages", seqs=3, new_lo=1024, new_hi=1153, hq=32, hkv=8, axes=3, pad=64, len_seed=3),
        # a large prefill, an odd number of tokens
        _write("write_long_prefill", seqs=1, new_lo=32749, new_hi=32749, ctx_lo=5, ctx_hi=5, max_pos=65536),
        # one new token of one short sequence: the smallest attention
        _attn("attn_one_token", hq=8, hkv=2, d=64),
        # a batch that decodes one token a sequence, contexts of all lengths
        # (bound by the memory of keys and values)
        _attn("attn_token_batch", seqs=64, ctx_lo=100, ctx_hi=8191, hq=32, hkv=8, len_seed=3),
        # a chunk of a very long document (the largest case by operations)
        _attn("attn_long_chunk", new_lo=2048, new_hi=2048, ctx_lo=14336, ctx_hi=14336, hq=32, hkv=8),
        # a serving batch whose chunks are ragged, half of them single tokens
        # and some empty, with a head ratio that does not divide a tile and
        # prefixes that all of a sequence's tokens see
        _attn("attn_mixed_batch", seqs=24, new_lo=0, new_hi=300, ctx_lo=0, ctx_hi=3000, single=0.5, hq=40, hkv=8,
              prefix_mask=True, len_seed=4),
        # the tokens of one decode step of one page, 16 branches of 4, and
        # nothing but their own log probabilities and entropies
        _logp("logp_one_page"),
        # the whole step of 32 pages (6,144 query tokens) with alternatives
        # (the largest by memory)
        _logp("logp_many_pages", rows=6144, top=8),
        # a large odd vocabulary in 32 bits, a third of it banned, sampled at
        # a temperature, many alternatives
        _logp("logp_wide_vocabulary", rows=160, vocab=100003, wide=True, top=20, banned=0.33, temperature=0.7),
        # a decode step of 24 sequences through four layers, then the log
        # probabilities of its tokens: the three operators as they are used
        # together
        _step("step_decode"),
    ]


def draw(rng):
    """Batches of 1 to 256 sequences and chunks of 1 to 2,048 tokens behind contexts of up to 12,000; 1 to 4,000 rows
    of 100 to 160,000 logits."""
    def log(lo, hi):
        return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    kind = rng.choice(["write", "write", "attn", "attn", "attn", "logp", "logp", "step"])
    seed = rng.randrange(1 << 20)
    heads = rng.choice([(8, 2), (16, 2), (32, 8), (16, 4), (40, 8), (6, 2), (16, 16), (14, 2), (32, 2)])
    d = rng.choice([64, 128, 128])
    if kind == "logp":
        vocab, wide = log(100, 160000), rng.random() < 0.4
        case = _logp("", rows=log(1, min(4000, int(MAX_BYTES / 3 / (vocab * (4 if wide else 2))))), vocab=vocab,
                     wide=wide, top=rng.choice([0, 1, 5, 20, 32]), banned=rng.choice([0.0, 0.0, 0.3, 0.99]),
                     temperature=rng.choice([1.0, 1.0, 0.6, 1.3]))
        del case["name"]
        return case
    while True:
        if kind == "write":
            seqs = log(1, 256)
            case = _write("", seqs=seqs, new_lo=rng.choice([0, 1]), new_hi=log(1, max(1, 16000 // seqs)),
                          single=rng.choice([0.0, 0.5, 1.0]), hq=heads[0], hkv=heads[1], d=d, axes=rng.choice([1, 3]),
                          pad=rng.choice([0, 8, 64]), max_pos=32768, len_seed=seed)
        elif kind == "attn":
            ctx, new = log(1, 12000), log(1, 2048)
            case = _attn("", seqs=log(1, 64), new_lo=rng.choice([0, 1, new]), new_hi=new, ctx_lo=rng.choice([0, ctx]),
                         ctx_hi=ctx, single=rng.choice([0.0, 0.0, 0.5, 1.0]), hq=heads[0], hkv=heads[1], d=d,
                         prefix_mask=rng.random() < 0.3, len_seed=seed)
        else:
            case = _step("", layers=rng.choice([1, 2, 4]), seqs=log(1, 32), new_lo=1, new_hi=log(1, 400),
                         ctx_lo=0, ctx_hi=log(1, 4000), single=rng.choice([0.5, 1.0]), hq=heads[0], hkv=heads[1], d=d,
                         axes=rng.choice([1, 3]), vocab=log(1000, 50000), top=rng.choice([0, 5]), len_seed=seed)
        del case["name"]
        new, ctx = _lengths(case)
        if new.sum() < 1:
            seed += 1
            continue
        w = work(case)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and (case["kind"] == "write" or (
                4 * len(new) * case["hq"] * int(new.max()) * int((new + ctx).max()) <= MAX_SCORES
                and 4 * len(new) * int((new + ctx).max()) * case["hkv"] * case["d"] <= MAX_KEYS)):
            return case
        seed += 1


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


def _full(case, total):
    """Keys that every query of a sequence sees (its vision tokens)."""
    if not case.get("prefix_mask"):
        return np.zeros_like(total)
    return np.random.default_rng(104729 + case["len_seed"]).integers(0, total + 1)


# --------------------------------------------------------------- the inputs --

class _Maker:
    def __init__(self, seed):
        self.dev = torch.device("cuda")
        self.gen = torch.Generator(device=self.dev)
        self.gen.manual_seed(int(seed))

    def normal(self, *shape, std=0.5, mean=0.0, dtype=torch.bfloat16):
        x = torch.empty(shape, dtype=dtype, device=self.dev)
        return x.normal_(mean, std, generator=self.gen)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.gen, device=self.dev)

    def perm(self, n):
        return torch.randperm(n, generator=self.gen, device=self.dev, dtype=torch.int32)

    def ints(self, a):
        return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device=self.dev)

    def cache(self, pages, hkv, d, std):
        """Codes and scales of pages that were written a row at a time: the largest value's scale, some a doubling
        above it."""
        x = self.normal(pages, PAGE, hkv, d, std=std)
        scale = x.abs().amax((1, 3)).float() / CODE_MAX * torch.exp2(torch.floor(2 * self.uniform(pages, hkv)))
        return (x / scale[:, None, :, None]).to(torch.float8_e4m3fn), scale


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


def _positions(axes, pos, max_pos):
    """Text positions as they are; images in grids of 32 x 32 with a time, a height and a width."""
    if axes == 1:
        return pos[None].contiguous()
    t = pos // 1024
    return torch.stack((t, t + (pos % 1024) // 32, t + pos % 32)).clamp(max=max_pos - 1).to(torch.int32).contiguous()


def _layer(mk, case, T, num_pages):
    k, k_scale = mk.cache(num_pages, case["hkv"], case["d"], 1.0)
    v, v_scale = mk.cache(num_pages, case["hkv"], case["d"], 0.5)
    la = dict(k_cache=k, k_scale=k_scale, v_cache=v, v_scale=v_scale)
    if case["kind"] != "attn":
        la["qkv"] = mk.normal(T, (case["hq"] + 2 * case["hkv"]) * case["d"] + case.get("pad", 0), std=1.0)
        # (values have half the size of queries and keys)
        la["qkv"][:, (case["hq"] + case["hkv"]) * case["d"]:] *= 0.5
    return la


def _logits(mk, rows, vocab, wide, banned):
    """Logits and chosen tokens: nine of ten distributions are sure of a token, seven of ten tokens are the likeliest."""
    x = mk.normal(rows, vocab, std=2.0, dtype=torch.float32)
    sure = torch.randint(0, vocab, (rows, 1), generator=mk.gen, device=mk.dev)
    x.scatter_add_(1, sure, 14.0 * (mk.uniform(rows, 1) < 0.9))
    if banned:
        x.masked_fill_(mk.uniform(rows, vocab) < banned, -math.inf)
    x = x if wide else x.to(torch.bfloat16)
    other = torch.randint(0, vocab, (rows,), generator=mk.gen, device=mk.dev)
    return x, torch.where(mk.uniform(rows) < 0.7, x.argmax(1), other).to(torch.int32)


def prepare(case, seed):
    mk = _Maker(seed)
    st = dict(case=case)
    if case["kind"] == "logp":
        st["logits"], st["tokens"] = _logits(mk, case["rows"], case["vocab"], case["wide"], case["banned"])
        return st
    hq, d = case["hq"], case["d"]
    new, ctx = _lengths(case)
    total, T = new + ctx, int(new.sum())
    pages = (total + PAGE - 1) // PAGE
    max_pages, num_pages = max(1, int(pages.max())), int(pages.sum()) + 3
    cu = np.concatenate(([0], np.cumsum(new)))
    st.update(max_new=int(new.max()), max_len=int(total.max()), tokens=T,
              page_table=_table(mk, pages, max_pages, mk.perm(num_pages)), seq_len=mk.ints(total), chunk_cu=mk.ints(cu))
    if case["kind"] == "attn":
        # (queries and keys have the size that their norms leave them)
        st.update(q=mk.normal(T, hq, d, std=1.0), full_len=mk.ints(_full(case, total)) if case["prefix_mask"] else None,
                  layers=[_layer(mk, case, T, num_pages)])
        return st
    seq = torch.repeat_interleave(torch.arange(len(new), device=mk.dev), mk.ints(new), output_size=T)
    pos = torch.arange(T, device=mk.dev, dtype=torch.int32) + mk.ints(ctx - cu[:-1])[seq]
    slot = st["page_table"][seq, (pos // PAGE).long()] * PAGE + pos % PAGE
    shift = int(torch.randint(0, max(1, case["max_pos"] - int(total.max())), (1,), generator=mk.gen, device=mk.dev))
    st.update(slot=slot.to(torch.int32).contiguous(), pos=_positions(case["axes"], pos + shift, case["max_pos"]),
              full_len=None, q_weight=mk.normal(d, std=0.1, mean=1.0), k_weight=mk.normal(d, std=0.1, mean=1.0),
              table=_rotation(case["max_pos"], d, mk.dev), sections=_sections(case["axes"], d),
              axis=mk.ints(np.repeat(np.arange(case["axes"]), _sections(case["axes"], d))),
              layers=[_layer(mk, case, T, num_pages) for _ in range(case.get("layers", 1))])
    if case["kind"] == "step":
        st["logits"], st["tokens_out"] = _logits(mk, T, case["vocab"], False, 0.0)
    return st


# ------------------------------------------------------- the plain operators --

def _plain_norm_rope(x, weight, cos, sin):
    """x [T][H][D] normed over D, then rotated in pairs (i, i + D / 2), 32 bits."""
    x = x.float()
    x = x * torch.rsqrt(torch.mean(x * x, -1, keepdim=True) + EPS) * weight.float()
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)


def _plain_put(x, slot, code, scale):
    """x [T][H][D] into the rows `slot` of the coded cache, in place."""
    page, row = torch.unique(slot // PAGE, return_inverse=True)
    x, page, off = x.float(), page.long(), (slot % PAGE).long()
    n, h = page.numel(), x.shape[1]
    top = x.new_zeros(n, h).index_reduce_(0, row, x.abs().amax(-1), "amax") / CODE_MAX
    first = torch.full((n,), PAGE, device=x.device).index_reduce_(0, row, off, "amin")
    had = scale[page]
    k = torch.ceil(torch.log2(top.double() / had.double())).clamp(min=0).float()  # doublings of a scale that is there
    now = torch.where((first > 0)[:, None], had * torch.exp2(k), top.clamp(min=LEAST_SCALE))
    scale[page] = now
    old = code[page].float()
    at = torch.arange(PAGE, device=x.device)
    kept = old * torch.exp2(-k)[:, None, :, None]
    old = torch.where((at < first[:, None])[:, :, None, None], kept, old)
    old[row, off] = (x / now[row][:, :, None]).clamp(-CODE_MAX, CODE_MAX)
    code[page] = old.to(code.dtype)


def _plain_write(case, qkv, q_weight, k_weight, table, axis, pos, slot, k_cache, k_scale, v_cache, v_scale):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    x = qkv[:, : (hq + 2 * hkv) * d].reshape(qkv.shape[0], hq + 2 * hkv, d)
    rot = table[pos.long()[axis.long()].T, torch.arange(d // 2, device=qkv.device)]  # [T][D / 2][2]
    cos, sin = rot[:, None, :, 0], rot[:, None, :, 1]
    _plain_put(_plain_norm_rope(x[:, hq: hq + hkv], k_weight, cos, sin), slot, k_cache, k_scale)
    _plain_put(x[:, hq + hkv:], slot, v_cache, v_scale)
    return _plain_norm_rope(x[:, :hq], q_weight, cos, sin).to(torch.bfloat16)


def _plain_attn(case, q, k_cache, k_scale, v_cache, v_scale, page_table, seq_len, chunk_cu, full_len, max_new, max_len):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    dev, T = q.device, q.shape[0]
    cu, L = chunk_cu.long(), seq_len.long()
    n = cu[1:] - cu[:-1]
    i, j = torch.arange(max_new, device=dev), torch.arange(max_len, device=dev)
    x = q[(cu[:-1, None] + i).clamp(max=T - 1)].float()  # [S][n][Hq][D], padded
    x = x.view(-1, max_new, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(len(n), hkv, -1, d)
    page = page_table.long().clamp(min=0)

    def values(code, scale):  # [S][L][Hkv][D]
        y = code[page].float() * scale[page][:, :, None, :, None]
        return y.view(len(n), -1, hkv, d)[:, :max_len]

    k, v = values(k_cache, k_scale).permute(0, 2, 3, 1), values(v_cache, v_scale).permute(0, 2, 1, 3)
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


def _plain_logp(logits, tokens, top, temperature):
    # in 64 bits: of a token that is nearly sure, 32 leave few digits of what its probability lacks to 1
    x = logits.double() * (1.0 / temperature)
    most = x.amax(-1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(-1, keepdim=True)
    rest = torch.log(total)
    mean = torch.where(e > 0, e * (x - most), 0.0).sum(-1) / total.squeeze(-1)
    got = dict(logprob=(x.gather(1, tokens.long()[:, None]) - most - rest).squeeze(1).float(),
               entropy=(rest.squeeze(1) - mean).float())
    if top:
        # the largest logits, the lowest of equal ones first: their order as whole numbers, then the place
        bits, last = (logits.float() + 0.0).view(torch.int32).long(), x.shape[1] - 1
        key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) + (last - torch.arange(last + 1, device=x.device))
        at = last - (torch.topk(key, top, dim=1).values & 0xFFFFFFFF)
        got.update(top_tokens=at.to(torch.int32), top_logprobs=(x.gather(1, at) - most - rest).float())
    return got


ROPE = ("q_weight", "k_weight", "table", "axis", "pos", "slot")
CACHE = ("k_cache", "k_scale", "v_cache", "v_scale")
LENGTHS = ("page_table", "seq_len", "chunk_cu", "full_len", "max_new", "max_len")


def _plain(st):
    case = st["case"]
    if case["kind"] == "logp":
        return _plain_logp(st["logits"], st["tokens"], case["top"], case["temperature"])
    got = {}
    for i, la in enumerate(st["layers"]):
        q = st.get("q")
        if q is None:
            q = _plain_write(case, la["qkv"], *(st[k] for k in ROPE), *(la[k] for k in CACHE))
            got.update({"q%d" % i: q}, **{k + str(i): la[k] for k in CACHE})
        if case["kind"] != "write":
            got["out%d" % i], got["lse%d" % i] = _plain_attn(case, q, *(la[k] for k in CACHE), *(st[k] for k in LENGTHS))
    if case["kind"] == "step":
        got.update(_plain_logp(st["logits"], st["tokens_out"], case["top"], 1.0))
    return got


# --------------------------------------------------- the framework's operators --

def _handles(st):
    """The call objects with their outputs and workspaces, which a program makes once."""
    from paper_2607_18839_gb300 import hpd
    case, ops = st["case"], {"hpd": hpd}
    if case["kind"] in ("write", "step"):
        ops["rope"] = hpd.QkNormRope(case["hq"], case["hkv"], case["d"], st["q_weight"], st["k_weight"], st["table"],
                                     sections=st["sections"], eps=EPS)
        # (every layer's queries are returned)
        ops["q"] = [torch.empty(st["tokens"], case["hq"], case["d"], dtype=torch.bfloat16, device="cuda")
                    for _ in st["layers"]]
    if case["kind"] in ("attn", "step"):
        ops["attn"] = [hpd.ChunkAttn(case["hq"], la["k_cache"], la["v_cache"], st["page_table"],
                                     max_tokens=st["tokens"], max_seq_len=st["max_len"], k_scale=la["k_scale"],
                                     v_scale=la["v_scale"]) for la in st["layers"]]
    return ops


def _call(st):
    case = st["case"]
    if "ops" not in st:
        st["ops"] = _handles(st)
    ops, got = st["ops"], {}
    for i, la in enumerate(st.get("layers", ())):
        q = st.get("q")
        if q is None:
            q = ops["rope"](la["qkv"], st["pos"], st["slot"], la["k_cache"], la["v_cache"], q_out=ops["q"][i],
                            k_scale=la["k_scale"], v_scale=la["v_scale"])
            got.update({"q%d" % i: q}, **{k + str(i): la[k] for k in CACHE})
        if case["kind"] != "write":
            got["out%d" % i], got["lse%d" % i] = ops["attn"][i](q, st["chunk_cu"], st["seq_len"], st["full_len"])
    if case["kind"] in ("write", "attn"):
        return got
    logits, tokens = st["logits"], st["tokens_out" if case["kind"] == "step" else "tokens"]
    r = ops["hpd"].token_logprobs(logits, tokens, top=case["top"], temperature=case.get("temperature", 1.0))
    got.update(logprob=r.logprob, entropy=r.entropy)
    if case["top"]:
        got.update(top_tokens=r.top_tokens, top_logprobs=r.top_logprobs)
    return got


def run(state):
    return _call(state) if own else _plain(state)


# ----------------------------------------------------------------- the work --

def _work_write(case, new, ctx):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    T = int(new.sum())
    pages = np.where(new > 0, (ctx + new + PAGE - 1) // PAGE - ctx // PAGE, 0).sum()
    # rows in bf16 in, queries in bf16 and codes out, positions and slots, the table's rows, a scale a page and head
    nbytes = 2 * T * (hq + 2 * hkv) * d + 2 * T * hq * d + 2 * T * hkv * d + 4 * T * (case["axes"] + 1)
    nbytes += 4 * d * min(T, case["max_pos"]) + 4 * d + 8 * int(pages) * hkv
    # a norm is 3 operations a value, its weight 1, the rotation 3, a code 2
    return nbytes, 7 * T * (hq + hkv) * d + 4 * T * hkv * d


def _work_attn(case, new, ctx, full):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    keys = np.where(new > 0, new + ctx, 0)
    pages = int(((keys + PAGE - 1) // PAGE).sum())
    pairs = 0
    for n, c, f in zip(new.tolist(), ctx.tolist(), full.tolist()):
        low = max(0, min(n, f - c))  # queries that the prefix mask gives more than their own past
        pairs += low * f + (n - low) * c + (n * (n + 1) - low * (low + 1)) // 2
    T = int(new.sum())
    nbytes = 2 * int(keys.sum()) * hkv * d + 8 * pages * hkv + 2 * 2 * T * hq * d + 4 * T * hq + 4 * pages
    return nbytes + 12 * len(new), 4 * pairs * hq * d


def _work_logp(rows, vocab, size, top):
    # an exponential, two sums and two products a value
    return rows * (vocab * size + 12 + 8 * top), 5 * rows * vocab


def work(case):
    if case["kind"] == "logp":
        b, f = _work_logp(case["rows"], case["vocab"], 4 if case["wide"] else 2, case["top"])
        return {"bytes": int(b), "flops": int(f)}
    new, ctx = _lengths(case)
    b = f = 0
    if case["kind"] != "attn":
        b, f = _work_write(case, new, ctx)
    if case["kind"] != "write":
        ab, af = _work_attn(case, new, ctx, _full(case, new + ctx))
        b, f = b + ab, f + af
    b, f = b * case.get("layers", 1), f * case.get("layers", 1)
    if case["kind"] == "step":
        lb, lf = _work_logp(int(new.sum()), case["vocab"], 2, case["top"])
        b, f = b + lb, f + lf
    return {"bytes": int(b), "flops": int(f)}


# ------------------------------------------------------ the results in 64 bits --

def _exact_put(x, slots, code, scale):
    """Codes (not rounded) and scales after rows x [T][H][D] went to `slots` (a list), page by page."""
    code, scale = code.double(), scale.double()
    t = 0
    while t < len(slots):
        page, first = divmod(slots[t], PAGE)
        n = 1
        while t + n < len(slots) and slots[t + n] == slots[t] + n and first + n < PAGE:
            n += 1
        rows = x[t: t + n]
        need = rows.abs().amax((0, 2)) / CODE_MAX
        if first == 0:
            scale[page] = need.clamp(min=LEAST_SCALE)
        else:
            doubled = torch.ceil(torch.log2(need / scale[page])).clamp(min=0)
            code[page, :first] /= torch.exp2(doubled)[None, :, None]
            scale[page] *= torch.exp2(doubled)
        code[page, first: first + n] = rows / scale[page][None, :, None]
        t += n
    return code, scale


def _exact_write(case, st, la):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    axis = sum(([a] * c for a, c in enumerate(st["sections"])), [])
    table, pos = st["table"].double(), st["pos"].long()
    cos = torch.stack([table[pos[axis[i]], i, 0] for i in range(d // 2)], 1)
    sin = torch.stack([table[pos[axis[i]], i, 1] for i in range(d // 2)], 1)

    def turn(x, w):
        x = x.double() / (x.double().pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
        z = torch.complex(x[..., : d // 2], x[..., d // 2:]) * torch.complex(cos, sin)[:, None]
        return torch.cat((z.real, z.imag), -1)

    heads = [la["qkv"][:, h * d: (h + 1) * d] for h in range(hq + 2 * hkv)]
    slots = st["slot"].tolist()
    k, ks = _exact_put(turn(torch.stack(heads[hq: hq + hkv], 1), st["k_weight"]), slots, la["k_cache"], la["k_scale"])
    v, vs = _exact_put(torch.stack(heads[hq + hkv:], 1).double(), slots, la["v_cache"], la["v_scale"])
    return turn(torch.stack(heads[:hq], 1), st["q_weight"]), k, ks, v, vs


def _exact_attn(case, q, k_code, k_scale, v_code, v_scale, table, new, ctx, full):
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
                of = lambda code, scale: (code[pages][:, :, h // g].double() * scale[pages, h // g].double()[:, None, None])  # noqa: E731
                k = of(k_code, k_scale).reshape(-1, d)[: n + c]
                v = of(v_code, v_scale).reshape(-1, d)[: n + c]
            x = (q[t: t + n, h].double() @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[t: t + n, h] = torch.logsumexp(x, -1)
            out[t: t + n, h] = torch.softmax(x, -1) @ v
        t += n
    return out, lse


def _exact_logp(logits, tokens, top, temperature):
    names = ("logprob", "entropy") + (("top_logprobs",) if top else ())
    parts = {k: [] for k in names}
    for x, t in zip(logits.split(256), tokens.split(256)):
        p = torch.log_softmax(x.double() / temperature, -1)
        parts["logprob"].append(p[torch.arange(len(t), device=t.device), t.long()])
        parts["entropy"].append(-torch.special.xlogy(p.exp(), p.exp()).sum(-1))
        if top:
            parts["top_logprobs"].append(torch.sort(p, -1, descending=True).values[:, :top])
    got = {k: torch.cat(v) for k, v in parts.items()}
    return dict(got, top_tokens=None) if top else got


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "logp":
        return _exact_logp(st["logits"], st["tokens"], case["top"], case["temperature"])
    new, ctx = _lengths(case)
    got = {}
    for i, la in enumerate(st["layers"]):
        q, cache = st.get("q"), [la[k] for k in CACHE]
        if q is None:
            q, *cache = _exact_write(case, st, la)
            got.update({"q%d" % i: q}, **{k + str(i): x for k, x in zip(CACHE, cache)})
            # the attention is of the rounded queries and codes, as the cache holds them
            q, cache = q.bfloat16(), [x.float().to(y.dtype) for x, y in zip(cache, (la[k] for k in CACHE))]
        if case["kind"] != "write":
            got["out%d" % i], got["lse%d" % i] = _exact_attn(case, q, *cache, st["page_table"], new, ctx,
                                                             _full(case, new + ctx))
    if case["kind"] == "step":
        got.update(_exact_logp(st["logits"], st["tokens_out"], case["top"], 1.0))
    return got
