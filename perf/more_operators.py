"""The operators of a layer with rotary positions on several axes and a paged
key/value cache, as plain cases: inputs from a seed, one pass, the work of a
pass, and the answer in 64 bits.

  rope    rotary embedding of query and key rows whose tokens have a position
          on each of several axes (time, height, width of images and video)
  store   new key and value rows written into the pages of a cache, quantized
          per token and head, and the same rows read back out of it
  attend  attention of the newest tokens of every sequence over its pages: one
          token each in a decode step, a chunk of a prompt, or both in a batch

Where ``own`` is false a pass is elementary torch operations; where it is true
it is the library's calls.
"""
import functools
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}

# Head layouts: those of this repository's workloads (4/4 of 64, 32/32, 28/4 and
# 40/40 of 128), in `draw` also generic grouped ones.  A case's lengths follow
# from its numbers alone: see _lengths.


def listed():
    return [
        # One text token of the smallest layer: nothing but launches and latency.
        dict(name="rope_tiny_one", kind="rope", m=1, hq=4, hkv=4, dh=64, dtype="f16", axes=3, theta=1e4),
        # Prompts of video frames and text through a grouped bf16 layer, 8192 tokens in all.
        dict(name="rope_qwen2vl7b_video", kind="rope", m=8192, hq=28, hkv=4, dh=128, dtype="bf16", axes=3, theta=1e6),
        # A decode step of 32 sequences into an int8 cache.
        dict(name="store_qwen2vl7b_step", kind="store", batch=32, ctx=8192, ragged=20, new=1, mixed=False, hkv=4, dh=128,
             dtype="bf16", fmt="i8", page=64),
        # Four prompts of 576 image and 64 text tokens.
        dict(name="store_llava7b", kind="store", batch=4, ctx=640, ragged=0, new=640, mixed=False, hkv=32, dh=128,
             dtype="f16", fmt="i8", page=64),
        # Eight prompts of odd lengths into an int4 cache of small pages.
        dict(name="store_llava13b", kind="store", batch=8, ctx=703, ragged=30, new=703, mixed=False, hkv=40, dh=128,
             dtype="f16", fmt="i4", page=16),
        # One token over 65 of the smallest layer.
        dict(name="attend_tiny_one", kind="attend", batch=1, ctx=65, ragged=0, new=1, mixed=False, hq=4, hkv=4, dh=64,
             dtype="f16", fmt="f16", page=16),
        # One long conversation, a cache as the projections leave it.
        dict(name="attend_qwen2vl7b_one", kind="attend", batch=1, ctx=30001, ragged=0, new=1, mixed=False, hq=28, hkv=4,
             dh=128, dtype="bf16", fmt="f16", page=64),
        # The decode batch of the grouped workload, int8 cache.
        dict(name="attend_qwen2vl7b_step", kind="attend", batch=32, ctx=8192, ragged=20, new=1, mixed=False, hq=28,
             hkv=4, dh=128, dtype="bf16", fmt="i8", page=64),
        # The decode batch of a layer whose heads each have keys of their own.
        dict(name="attend_llava7b_step", kind="attend", batch=16, ctx=4096, ragged=0, new=1, mixed=False, hq=32, hkv=32,
             dh=128, dtype="f16", fmt="f16", page=64),
        # The same with an int4 cache and lengths that differ.
        dict(name="attend_llava13b_step", kind="attend", batch=8, ctx=4096, ragged=20, new=1, mixed=False, hq=40,
             hkv=40, dh=128, dtype="f16", fmt="i4", page=16),
        # Chunks of 512 tokens of four long prompts.
        dict(name="attend_qwen2vl7b_chunk", kind="attend", batch=4, ctx=8192, ragged=10, new=512, mixed=False, hq=28,
             hkv=4, dh=128, dtype="bf16", fmt="i8", page=64),
        # A batch in which every fourth sequence brings a chunk of its prompt and the others one token.
        dict(name="attend_llava7b_mixed", kind="attend", batch=8, ctx=2501, ragged=40, new=333, mixed=True, hq=32,
             hkv=32, dh=128, dtype="f16", fmt="f16", page=32),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(("rope", "store", "attend", "attend"))
        hq, hkv, dh = rng.choice(((4, 4, 64), (32, 32, 128), (28, 4, 128), (40, 40, 128), (8, 2, 64), (16, 8, 128),
                                  (12, 1, 128)))
        dtype = rng.choice(("f16", "bf16"))
        if kind == "rope":
            c = dict(kind=kind, m=_log(rng, 1, 16384), hq=hq, hkv=hkv, dh=dh, dtype=dtype, axes=rng.choice((1, 2, 3, 3)),
                     theta=rng.choice((1e4, 1e6)))
        else:
            c = dict(kind=kind, batch=_log(rng, 1, 64), ctx=_log(rng, 1, 32768), ragged=rng.choice((0, 10, 50, 90)),
                     hkv=hkv, dh=dh, dtype=dtype, fmt=rng.choice(("f16", "i8", "i4")),
                     page=rng.choice((16, 32, 64, 128, 256)))
            if kind == "attend":
                c["hq"] = hq
            c["new"] = rng.choice((1, 1, _log(rng, 1, 1024))) if kind == "attend" else _log(rng, 1, 4096)
            c["new"] = min(c["new"], c["ctx"])
            c["mixed"] = rng.random() < 0.3
        if _cost(c) <= most and _space(c) <= 6e9:
            return c


def _lengths(case):
    """Tokens of every sequence, and how many of them are new: lengths spread
    over the last `ragged` percent below `ctx`; new tokens `new` each, or 1 but
    for every fourth sequence."""
    spread = case["ctx"] * case["ragged"] // 100
    lens = [case["ctx"] - (b * 7919) % (spread + 1) for b in range(case["batch"])]
    news = [min(n, 1 if case["mixed"] and b % 4 else case["new"]) for b, n in enumerate(lens)]
    return lens, news


def _sections(case):
    """Frequency pairs of each axis: a fourth of them for time, the rest in halves for height and width."""
    half = case["dh"] // 2
    return {1: [half], 2: [half // 2, half // 2], 3: [half // 4, half * 3 // 8, half * 3 // 8]}[case["axes"]]


# ---------------------------------------------------------------- inputs

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rows(gen, m, heads, dh):
    """N(0, 1) heads with one channel in sixteen four times larger, and row magnitudes that differ."""
    x = _randn(gen, m, heads, dh) * torch.exp(0.3 * _randn(gen, m, heads, 1))
    x[:, :, torch.randperm(dh, generator=gen, device="cuda")[:dh // 16]] *= 4.0
    return x


def _positions(case, gen):
    """Video of 14 x 14 patches a frame with text after every fourth frame: a
    patch has its frame, row and column, a text token the same position on all
    axes."""
    m = case["m"]
    t = torch.arange(m, device="cuda")
    block = 4 * 196 + 60
    at, first = t % block, t // block * 120 + torch.randint(0, 20000, (1,), generator=gen, device="cuda")
    text = at >= 4 * 196
    grid = torch.stack((at // 196, at % 196 // 14, at % 14))[3 - case["axes"]:]
    pos = torch.where(text, (at - 4 * 196 + 14).expand(case["axes"], m), grid) + first
    return pos.to(torch.int32).contiguous()


def _bits(case):
    return {"f16": 16, "i8": 8, "i4": 4}[case["fmt"]]


def _pack(codes):
    """int8 codes of [-7, 7] two to a byte, the even element in the low nibble."""
    return (codes[..., ::2] & 15) | (codes[..., 1::2] << 4)


def _unpack(packed):
    return torch.stack(((packed << 4) >> 4, packed >> 4), dim=-1).flatten(-2)


def _quantize(x, bits):
    """Codes and scales of fp32 rows, per row of the last axis: the quotients
    in 64 bits, where one half way between two codes is met exactly."""
    qm = 2.0 ** (bits - 1) - 1
    a = x.abs().amax(-1, keepdim=True)
    a = torch.where(a < 2.0 ** -119, torch.full_like(a, math.inf), a)      # such a row: codes 0, scale 1
    s = torch.where(a == math.inf, torch.ones_like(a), a / qm)
    return torch.round(x.double() * qm / a.double()).to(torch.int8), s[..., 0]


def _pool(case, gen, n_pages, filled):
    """Pages [n_pages][heads][page][dh] of keys or values (and scales), rows of earlier use in them."""
    shape = (n_pages, case["hkv"], case["page"], case["dh"])
    if not filled:
        x = torch.zeros(shape, device="cuda")
    else:
        x = _rows(gen, n_pages * case["page"], case["hkv"], case["dh"])
        x = x.view(n_pages, case["page"], case["hkv"], case["dh"]).transpose(1, 2)
    if case["fmt"] == "f16":
        return x.to(DTYPES[case["dtype"]]).contiguous(), None
    codes, scale = _quantize(x, _bits(case))
    return (codes if case["fmt"] == "i8" else _pack(codes)).contiguous(), scale.contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, dh = DTYPES[case["dtype"]], case["dh"]
    if case["kind"] == "rope":
        return dict(q=_rows(gen, case["m"], case["hq"], dh).to(dt), k=_rows(gen, case["m"], case["hkv"], dh).to(dt),
                    pos=_positions(case, gen))
    lens, news = _lengths(case)
    first = [sum(news[:b]) for b in range(len(news) + 1)]
    page = case["page"]
    if case["kind"] == "store":      # only the pages that new tokens meet are in the pool
        cols = [[c for c in range(-(-n // page)) if (c + 1) * page > n - k] for n, k in zip(lens, news)]
    else:
        cols = [list(range(-(-n // page))) for n in lens]
    used = sum(len(c) for c in cols)
    order = torch.randperm(used + 2, generator=gen, device="cuda")
    table = torch.zeros((len(lens), max(-(-n // page) for n in lens)), dtype=torch.int32)
    order_host, at = order.cpu(), 0
    for b, c in enumerate(cols):
        table[b, c[0]:c[0] + len(c)] = order_host[at:at + len(c)]
        at += len(c)
    filled = case["kind"] == "attend"
    k, ks = _pool(case, gen, used + 2, filled)
    v, vs = _pool(case, gen, used + 2, filled)
    st = dict(k=k, ks=ks, v=v, vs=vs, table=table.cuda(),
              lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
              first=torch.tensor(first, dtype=torch.int32, device="cuda"))
    if filled:
        # queries a little longer than keys: a softmax that prefers some tokens
        st["q"] = (1.5 * _rows(gen, first[-1], case["hq"], dh)).to(dt)
    else:
        st["k_new"] = _rows(gen, first[-1], case["hkv"], dh).to(dt)
        st["v_new"] = _rows(gen, first[-1], case["hkv"], dh).to(dt)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"] == "rope":
        st["q_out"], st["k_out"] = torch.empty_like(st["q"]), torch.empty_like(st["k"])
    elif case["kind"] == "store":
        st["k_back"], st["v_back"] = torch.empty_like(st["k_new"]), torch.empty_like(st["v_new"])
    else:
        st["out"] = torch.empty_like(st["q"])
    if case["kind"] != "rope":
        st["max_len"], st["max_new"] = (max(x) for x in _lengths(case))
    return st


# ---------------------------------------------------------------- one pass, plain

def _turned(x, cos, sin):
    a, b = x.float().chunk(2, dim=-1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1).to(x.dtype)


def _run_rope(st, c):
    # angles in 64 bits: positions reach tens of thousands
    half = c["dh"] // 2
    freq = c["theta"] ** (torch.arange(half, dtype=torch.float64, device="cuda") * (-2.0 / c["dh"]))
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"),
                                   torch.tensor(_sections(c), device="cuda"), output_size=half)
    angle = st["pos"].double().t()[:, axis] * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    return dict(q=_turned(st["q"], cos, sin), k=_turned(st["k"], cos, sin))


def _slots(st, c):
    """Page and row in it of every new token."""
    n_rows = st["k_new"].shape[0]
    row = torch.arange(n_rows, device="cuda")
    seq = torch.bucketize(row, st["first"][1:].long(), right=True)
    pos = st["lens"].long()[seq] - st["first"].long()[seq + 1] + row
    return st["table"].long()[seq, pos // c["page"]], pos % c["page"]


def _run_store(st, c):
    page, slot = _slots(st, c)
    out = {}
    for name, pool, scales in (("k", st["k"], st["ks"]), ("v", st["v"], st["vs"])):
        x = st[name + "_new"]
        if c["fmt"] == "f16":
            pool[page, :, slot] = x
            out[name] = pool[page, :, slot]
            continue
        codes, s = _quantize(x.float(), _bits(c))
        pool[page, :, slot] = codes if c["fmt"] == "i8" else _pack(codes)
        scales[page, :, slot] = s
        back = pool[page, :, slot]
        back = back if c["fmt"] == "i8" else _unpack(back)
        out[name] = (back.float() * scales[page, :, slot][..., None]).to(x.dtype)
    return out


def _gathered(pool, scales, table, c):
    """A sequence's pages as fp32 rows [batch][heads][tokens][dh]."""
    x = pool[table]                                     # [batch][cols][heads][page][..]
    if c["fmt"] == "i4":
        x = _unpack(x)
    x = x.float()
    if scales is not None:
        x = x * scales[table][..., None]
    return x.transpose(1, 2).flatten(2, 3)


def _run_attend(st, c):
    table, lens, first = st["table"].long(), st["lens"].long(), st["first"].long()
    batch, tokens = table.shape[0], table.shape[1] * c["page"]
    n_rows, group, dh = st["q"].shape[0], c["hq"] // c["hkv"], c["dh"]
    k, v = _gathered(st["k"], st["ks"], table, c), _gathered(st["v"], st["vs"], table, c)
    i = torch.arange(st["max_new"], device="cuda")
    new = first[1:] - first[:-1]
    row = (first[:-1, None] + i).clamp(max=n_rows - 1)
    q = st["q"][row].float().view(batch, -1, c["hkv"], group, dh).permute(0, 2, 1, 3, 4).flatten(2, 3)
    score = (q @ k.transpose(2, 3).contiguous()) * dh ** -0.5
    pos = (lens - new)[:, None] + i
    seen = torch.arange(tokens, device="cuda") <= pos[..., None]
    score = score.view(batch, c["hkv"], -1, group, tokens).masked_fill(~seen[:, None, :, None], -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    # rows of a page behind the last token are no values
    v = v * (torch.arange(tokens, device="cuda") < lens[:, None])[:, None, :, None]
    o = (p.flatten(2, 3) @ v).view(batch, c["hkv"], -1, group, dh).permute(0, 2, 1, 3, 4).flatten(2, 3)
    at = torch.bucketize(torch.arange(n_rows, device="cuda"), first[1:], right=True)
    return o[at, torch.arange(n_rows, device="cuda") - first[at]].to(st["q"].dtype)


# ---------------------------------------------------------------- one pass, the library

@functools.lru_cache(maxsize=None)
def _library():
    from paper_2510_16292_amd import binding
    return binding


def _dtype(c):
    return _library().QSVD_BF16 if c["dtype"] == "bf16" else _library().QSVD_F16


def _handles(st, c):
    """What a program keeps from call to call: the pool's and the batch's descriptions, and the workspace."""
    if "pool" not in st:
        B = _library()
        fmt = {"f16": B.QSVD_CACHE_F16, "i8": B.QSVD_CACHE_I8, "i4": B.QSVD_CACHE_I4}[c["fmt"]]
        st["pool"] = B.QsvdPages(fmt, _dtype(c), c["hkv"], c["dh"], c["page"], st["k"].shape[0], B.ptr(st["k"]),
                                 B.ptr(st["v"]), B.ptr(st["ks"]), B.ptr(st["vs"]))
        rows = st["q"] if c["kind"] == "attend" else st["k_new"]
        st["batch"] = B.QsvdPageBatch(st["table"].shape[0], st["table"].shape[1], B.ptr(st["table"]), B.ptr(st["lens"]),
                                      B.ptr(st["first"]), st["max_len"], st["max_new"], rows.shape[0])
        if c["kind"] == "attend":
            size = B.qsvd_paged_attention_workspace_size(st["pool"], st["batch"], c["hq"])
            st["ws"] = torch.empty((size,), dtype=torch.uint8, device="cuda")
    return st["pool"], st["batch"]


def _own_rope(st, c):
    B = _library()
    if "rope" not in st:
        st["rope"] = B.rope(c["dh"], _sections(c), c["theta"])
    wq, wk = c["hq"] * c["dh"], c["hkv"] * c["dh"]
    B.check(B.qsvd_rope_axes(st["rope"], B.ptr(st["pos"]), c["m"], c["m"], _dtype(c), B.ptr(st["q"]), wq, c["hq"],
                             B.ptr(st["q_out"]), wq, B.ptr(st["k"]), wk, c["hkv"], B.ptr(st["k_out"]), wk,
                             B.stream_handle()))
    return dict(q=st["q_out"], k=st["k_out"])


def _own_store(st, c):
    B = _library()
    pool, batch = _handles(st, c)
    w, s = c["hkv"] * c["dh"], B.stream_handle()
    B.check(B.qsvd_paged_append(pool, batch, B.ptr(st["k_new"]), w, B.ptr(st["v_new"]), w, 1.0, s))
    B.check(B.qsvd_paged_read(pool, batch, B.ptr(st["k_back"]), w, B.ptr(st["v_back"]), w, s))
    return dict(k=st["k_back"], v=st["v_back"])


def _own_attend(st, c):
    B = _library()
    pool, batch = _handles(st, c)
    w = c["hq"] * c["dh"]
    B.check(B.qsvd_paged_attention(pool, batch, B.ptr(st["q"]), w, c["hq"], 0.0, B.ptr(st["out"]), w, B.ptr(st["ws"]),
                                   st["ws"].numel(), B.stream_handle()))
    return st["out"]


def run(st):
    c = st["case"]
    if own:
        return {"rope": _own_rope, "store": _own_store, "attend": _own_attend}[c["kind"]](st, c)
    return {"rope": _run_rope, "store": _run_store, "attend": _run_attend}[c["kind"]](st, c)


# ---------------------------------------------------------------- work

def work(case):
    if case["kind"] == "rope":
        n = case["m"] * (case["hq"] + case["hkv"]) * case["dh"]
        return dict(bytes=4 * n + 4 * case["axes"] * case["m"], flops=3 * n)
    lens, news = _lengths(case)
    token = 2 * case["hkv"] * (case["dh"] * _bits(case) / 8 + (0 if case["fmt"] == "f16" else 4))   # bytes in the cache
    if case["kind"] == "store":
        n = 2 * sum(news) * case["hkv"] * case["dh"]
        return dict(bytes=4 * n + sum(news) * token, flops=(0 if case["fmt"] == "f16" else 6) * n)
    pairs = sum(k * n - k * (k - 1) // 2 for n, k in zip(lens, news))
    return dict(bytes=sum(lens) * token + 4 * sum(news) * case["hq"] * case["dh"],
                flops=4 * case["hq"] * case["dh"] * pairs)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 200)


def _space(case):
    """About the largest tensor of a plain pass, in bytes."""
    if case["kind"] == "rope":
        return 0
    rows = case["batch"] * case["ctx"] * case["hkv"] * case["dh"] * 4
    return max(rows, case["batch"] * case["ctx"] * case["new"] * case["hq"] * 4) if case["kind"] == "attend" else rows // 8


# ---------------------------------------------------------------- the answer in 64 bits

def _exact_rope(st, c):
    m, half = c["m"], c["dh"] // 2
    turns = torch.zeros((m, half), dtype=torch.float64, device="cuda")
    j = 0
    for axis, n in enumerate(_sections(c)):
        for _ in range(n):
            turns[:, j] = st["pos"][axis].double() / (2 * math.pi * c["theta"] ** (2 * j / c["dh"]))
            j += 1
    z = torch.polar(torch.ones_like(turns), 2 * math.pi * (turns - turns.floor()))[:, None]

    def turn(x):
        x = x.double()
        y = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * z
        return torch.cat((y.real, y.imag), dim=-1)

    return dict(q=turn(st["q"]), k=turn(st["k"]))


def _exact_store(st, c):
    out = {}
    for name in ("k", "v"):
        x = st[name + "_new"].double()
        if c["fmt"] != "f16":
            levels, top = 127 if c["fmt"] == "i8" else 7, x.abs().max(dim=-1, keepdim=True).values
            x = (levels * x / top).round() * top / levels
        out[name] = x
    return out


def _exact_attend(st, c):
    lens, news = _lengths(c)
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    group, at = c["hq"] // c["hkv"], 0
    for b, (n, new) in enumerate(zip(lens, news)):
        pages = st["table"][b, :-(-n // c["page"])].long()
        hidden = torch.ones((new, n), dtype=torch.bool, device="cuda").triu(n - new + 1)
        for h in range(c["hkv"]):
            rows = []
            for pool, scales in ((st["k"], st["ks"]), (st["v"], st["vs"])):
                x = pool[pages, h]
                if c["fmt"] == "i4":
                    x = torch.stack((x.int() << 28 >> 28, x.int() >> 4), dim=3).flatten(2)
                x = x.double()
                if scales is not None:
                    x = x * scales[pages, h].double().unsqueeze(-1)
                rows.append(x.reshape(-1, c["dh"])[:n])
            for g in range(h * group, (h + 1) * group):
                s = torch.matmul(st["q"][at:at + new, g].double(), rows[0].t()) / math.sqrt(c["dh"])
                out[at:at + new, g] = torch.softmax(s.masked_fill(hidden, -math.inf), dim=1) @ rows[1]
        at += new
    return out


def exact(case, seed):
    st = _inputs(case, seed)
    return {"rope": _exact_rope, "store": _exact_store, "attend": _exact_attend}[case["kind"]](st, case)
