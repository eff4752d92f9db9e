"""The operators around the attention path that complete a quantized decoder
layer, as plain cases: inputs from a seed, one pass, the work of a pass, and the
answer in 64 bits.

  norm    residual addition, root-mean-square norm and per-token quantization
          (or the normed rows themselves, for the fused decode projection)
  gate    silu(gate) * up of a gated MLP with per-token quantization
  linear  8-bit integer product with a scale per token and per output channel,
          bias and residual

Where ``own`` is false a pass is elementary torch operations; where it is true
it is the library's calls.  Quantized rows are returned as the values their
codes and scales stand for.
"""
import functools
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = float(torch.tensor(1e-6, dtype=torch.float32))

# Widths: the layers of this repository's workloads (256, 4096, 3584, 5120) and
# gated MLPs of 11/4 times the width (704, 11264, 9856, 14080).


def listed():
    return [
        # One token on the smallest layer: nothing but launches and latency.
        dict(name="norm_tiny_one", kind="norm", m=1, k=256, dtype="f16", residual=False, out="codes", bits=8, clip=1.0),
        # A decode batch; the fused decode projection takes the normed rows themselves.
        dict(name="norm_llava7b_step", kind="norm", m=16, k=4096, dtype="f16", residual=True, out="y", bits=8,
             clip=1.0),
        # One prompt of odd length through a bf16 layer, with activation clipping.
        dict(name="norm_qwen2vl7b", kind="norm", m=1337, k=3584, dtype="bf16", residual=True, out="codes", bits=8,
             clip=0.9),
        # Eight prompts of 576 image and 128 text tokens of the W4A4 stack.
        dict(name="norm_llava13b", kind="norm", m=5632, k=5120, dtype="f16", residual=True, out="codes", bits=4,
             clip=1.0),
        # A decode batch between the MLP's products.
        dict(name="gate_qwen2vl7b_step", kind="gate", m=32, k=9856, dtype="bf16", bits=8, clip=1.0),
        # Four prompts of 576 image and 64 text tokens.
        dict(name="gate_llava7b", kind="gate", m=2560, k=11264, dtype="f16", bits=8, clip=1.0),
        # One token on the smallest layer.
        dict(name="linear_tiny_one", kind="linear", m=1, n=256, k=256, dtype="f16", bias=False, residual=True),
        # Output projection of a decode batch, added to the residual stream.
        dict(name="linear_llava7b_step", kind="linear", m=16, n=4096, k=4096, dtype="f16", bias=False, residual=True),
        # Down projection of a decode batch.
        dict(name="linear_qwen2vl7b_down", kind="linear", m=32, n=3584, k=9856, dtype="bf16", bias=False,
             residual=True),
        # A projector of odd sizes with a bias.
        dict(name="linear_odd", kind="linear", m=333, n=1001, k=1008, dtype="bf16", bias=True, residual=False),
        # Output projection of four prompts.
        dict(name="linear_llava7b", kind="linear", m=2560, n=4096, k=4096, dtype="f16", bias=False, residual=True),
        # Gate and up projections of eight prompts in one product.
        dict(name="linear_llava13b_up", kind="linear", m=5632, n=28160, k=5120, dtype="f16", bias=False,
             residual=False),
    ]


def _log(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(("norm", "gate", "linear", "linear"))
        dtype = rng.choice(("f16", "bf16"))
        m = _log(rng, 1, 8192)
        if kind == "norm":
            c = dict(kind=kind, m=m, k=8 * _log(rng, 8, 2048), dtype=dtype, residual=rng.random() < 0.75,
                     out=rng.choice(("codes", "codes", "y")), bits=rng.choice((8, 8, 4)),
                     clip=rng.choice((1.0, 1.0, 0.9)))
        elif kind == "gate":
            c = dict(kind=kind, m=m, k=8 * _log(rng, 8, 4096), dtype=dtype, bits=8, clip=rng.choice((1.0, 1.0, 0.9)))
        else:
            c = dict(kind=kind, m=m, n=_log(rng, 48, 32768), k=16 * _log(rng, 8, 1024), dtype=dtype,
                     bias=rng.random() < 0.4, residual=rng.random() < 0.5)
        if _cost(c) <= most:
            return c


# ---------------------------------------------------------------- inputs

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _rows(gen, m, k):
    """N(0, 1) rows with one channel in a hundred 30 times larger, and row
    magnitudes that differ."""
    x = _randn(gen, m, k) * torch.exp(0.5 * _randn(gen, m, 1))
    x[:, torch.randperm(k, generator=gen, device="cuda")[:max(1, k // 100)]] *= 30.0
    return x


def _codes(x):
    """int8 codes and fp32 scales per row."""
    s = x.abs().amax(1, keepdim=True) / 127.0
    return torch.clamp(torch.round(x / s), -127, 127).to(torch.int8), s[:, 0].contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    m, k, dt = case["m"], case["k"], DTYPES[case["dtype"]]
    if case["kind"] == "norm":
        st = dict(x=_rows(gen, m, k).to(dt), gamma=(1.0 + 0.3 * _randn(gen, k)).to(dt))
        if case["residual"]:
            st["residual"] = (3.0 * _rows(gen, m, k)).to(dt)
        return st
    if case["kind"] == "gate":
        # gate and up side by side, as one product writes them
        return dict(gate_up=(1.2 * _randn(gen, m, 2 * k)).to(dt))
    n = case["n"]
    xq, sx = _codes(_rows(gen, m, k))
    wq, sw = _codes(0.02 * _randn(gen, n, k))
    st = dict(xq=xq, sx=sx, wq=wq, sw=sw)
    if case["bias"]:
        st["bias"] = _randn(gen, n).to(dt)
    if case["residual"]:
        st["residual"] = (3.0 * _randn(gen, m, n)).to(dt)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    m, k, dt = case["m"], case["k"], DTYPES[case["dtype"]]

    def buf(cols, dtype):
        return torch.empty((m, cols), dtype=dtype, device="cuda")

    if case["kind"] == "linear":
        st["y"] = buf(case["n"], dt)
        return st
    if case["kind"] == "norm":
        if case["residual"]:
            st["h"] = buf(k, dt)
        if case["out"] == "y":
            st["y"] = buf(k, dt)
            return st
    st["codes"] = buf(k * case["bits"] // 8, torch.int8)
    st["scale"] = buf(1, torch.float32)
    st["values"] = buf(k, dt)
    return st


# ---------------------------------------------------------------- one pass

def _quantized(y, bits, clip, dt):
    """The values of the codes of fp32 rows y."""
    qm = 2.0 ** (bits - 1) - 1
    a = clip * y.abs().amax(1, keepdim=True)
    zero = a == 0
    inv = torch.where(zero, torch.zeros_like(a), qm / a)
    s = torch.where(zero, torch.ones_like(a), a / qm)
    return (torch.clamp(torch.round(y * inv), -qm, qm) * s).to(dt), s


def _run_norm(st, c, dt):
    h = st["x"]
    if c["residual"]:
        h = (h.float() + st["residual"].float()).to(dt)
    # the mean square in 64 bits: codes lie next to rounding borders
    r = (1.0 / torch.sqrt(h.double().square().mean(1, keepdim=True) + EPS)).float()
    y = h.float() * r * st["gamma"].float()
    if c["out"] == "y":
        out = dict(y=y.to(dt))
    else:
        values, s = _quantized(y, c["bits"], c["clip"], dt)
        out = dict(values=values, scale=s)
    return dict(out, h=h) if c["residual"] else out


def _run_gate(st, c, dt):
    g, u = st["gate_up"][:, :c["k"]].float(), st["gate_up"][:, c["k"]:].float()
    values, s = _quantized(g / (1.0 + torch.exp(-g)) * u, c["bits"], c["clip"], dt)
    return dict(values=values, scale=s)


def _run_linear(st, c, dt):
    y = st["xq"].float() @ st["wq"].float().t()
    y = y * st["sx"][:, None] * st["sw"]
    if c["bias"]:
        y = y + st["bias"].float()
    if c["residual"]:
        y = y + st["residual"].float()
    return dict(y=y.to(dt))


@functools.lru_cache(maxsize=None)
def _library():
    from paper_2510_16292_amd import binding
    return binding


def _values(st, c):
    """Codes and scales of a library call as the values they stand for."""
    q = st["codes"]
    if c["bits"] == 4:
        q = torch.stack(((q << 4) >> 4, q >> 4), dim=-1).view(c["m"], c["k"])
    torch.mul(q, st["scale"], out=st["values"])
    return dict(values=st["values"], scale=st["scale"])


def _own_norm(st, c, dtype):
    B = _library()
    k, res, h = c["k"], st.get("residual"), st.get("h")
    B.check(B.qsvd_rmsnorm_quantize_act(
        B.ptr(st["x"]), k, B.ptr(res), k, B.ptr(st["gamma"]), c["m"], k, dtype, EPS, c["bits"], c["clip"], B.ptr(h),
        k, B.ptr(st.get("y")), k, B.ptr(st.get("codes")), B.ptr(st.get("scale")), B.stream_handle()))
    out = dict(y=st["y"]) if c["out"] == "y" else _values(st, c)
    return dict(out, h=h) if c["residual"] else out


def _own_gate(st, c, dtype):
    B = _library()
    k, gate = c["k"], B.ptr(st["gate_up"])
    B.check(B.qsvd_silu_mul_quantize_act(gate, 2 * k, gate + 2 * k, 2 * k, c["m"], k, dtype, c["bits"], c["clip"],
                                         B.ptr(st["codes"]), B.ptr(st["scale"]), B.stream_handle()))
    return _values(st, c)


def _own_linear(st, c, dtype):
    B = _library()
    B.check(B.qsvd_linear_i8(B.ptr(st["xq"]), c["k"], B.ptr(st["sx"]), B.ptr(st["wq"]), B.ptr(st["sw"]), c["m"],
                             c["n"], c["k"], B.ptr(st.get("bias")), B.ptr(st.get("residual")), c["n"], dtype,
                             B.ptr(st["y"]), c["n"], B.stream_handle()))
    return dict(y=st["y"])


def run(st):
    c = st["case"]
    if own:
        dtype = _library().QSVD_BF16 if c["dtype"] == "bf16" else _library().QSVD_F16
        return {"norm": _own_norm, "gate": _own_gate, "linear": _own_linear}[c["kind"]](st, c, dtype)
    return {"norm": _run_norm, "gate": _run_gate, "linear": _run_linear}[c["kind"]](st, c, DTYPES[c["dtype"]])


# ---------------------------------------------------------------- work

def work(case):
    m, k = case["m"], case["k"]
    if case["kind"] == "linear":
        n = case["n"]
        b = m * k + n * k + 4 * (m + n) + 2 * m * n * (2 if case["residual"] else 1) + (2 * n if case["bias"] else 0)
        return dict(bytes=b, flops=2 * m * n * k)
    codes = m * k * case["bits"] / 8 + 4 * m
    if case["kind"] == "gate":
        return dict(bytes=4 * m * k + codes, flops=12 * m * k)
    b = 2 * k + 2 * m * k * (3 if case["residual"] else 1)
    return dict(bytes=b + (2 * m * k if case["out"] == "y" else codes), flops=10 * m * k)


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


# ---------------------------------------------------------------- the answer in 64 bits

def _exact_quantized(y, bits, clip):
    qm = 2 ** (bits - 1) - 1
    step = clip * y.abs().max(dim=1, keepdim=True).values / qm
    step = torch.where(step > 0, step, torch.ones_like(step))
    return dict(values=(y / step).round().clamp(-qm, qm) * step, scale=step)


def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "linear":
        y = (st["xq"].double() * st["sx"].double()[:, None]) @ (st["wq"].double() * st["sw"].double()[:, None]).t()
        for name in ("bias", "residual"):
            if name in st:
                y = y + st[name].double()
        return dict(y=y)
    if case["kind"] == "gate":
        g, u = st["gate_up"].double().split(case["k"], dim=1)
        return _exact_quantized(torch.sigmoid(g) * g * u, case["bits"], case["clip"])
    # the sum is stored, and normed as stored
    h = st["x"].double()
    total = h + st["residual"].double() if "residual" in st else h
    h = total.to(DTYPES[case["dtype"]]).double()
    y = h * (h.pow(2).sum(dim=1, keepdim=True) / case["k"] + EPS).rsqrt() * st["gamma"].double()
    out = dict(y=y) if case["out"] == "y" else _exact_quantized(y, case["bits"], case["clip"])
    return dict(out, h=total) if "residual" in st else out
