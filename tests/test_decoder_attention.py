"""The attention's part of a quantized decoder layer (test_gpu_decoder_layer.py): the
output projection's rows by themselves, before the residual streams and the MLP
cover them, relative to their own size.  Mistakes planted in the 64-bit
reference have to be rejected by the same bound."""
import numpy as np
import pytest

import gpu_harness as H
import test_gpu_decoder_layer as D
from oracle import layer_oracle as L
from paper_2510_16292_amd import binding as B

LENS, STEPS = [37, 70], 4

# Relative rms error of 8-bit rows whose largest value is 4 standard deviations:
# e = 4 / 127 / sqrt(12) = 0.9%.  Queries, keys and values come from two quantized
# rows (normed and latent): sqrt(2) e = 1.3% each.  Values: that is the output's
# error.  Scores (of unit variance): sqrt(2) 1.3% = 1.8% from queries and keys, which
# is the weights' relative and so the output's error.  The output's own codes: 0.9%.
# Together sqrt(1.3^2 + 1.8^2 + 0.9^2) = 2.4% over the rows of a prompt, held to 3%;
# a single token has a few large score errors per head, so its row may have twice that.
PROMPT, TOKEN = 0.03, 0.05


def attention(layer, x, res, past, mistake=None):
    """Output projection rows (without the residual) and all latent rows of a
    sequence that has `past` latent rows, in 64 bits."""
    h = x + res
    c = h / np.sqrt((h ** 2).mean(1, keepdims=True) + D.EPS) * layer.gamma[0] @ layer.A
    rows = np.concatenate([past, c])
    q, k, v = np.split(rows @ layer.B, [D.HQ * D.DH, (D.HQ + D.HKV) * D.DH], axis=1)
    n, m = len(rows), len(c)
    at, key = np.arange(n - m, n)[:, None], np.arange(n)[None, :]
    hidden = key > at
    if mistake == "own token hidden":
        hidden |= (key == at) & (at > 0)
    if mistake == "next token seen":
        hidden = key > at + 1
    if mistake == "first row dropped":
        hidden |= (key == 0) & (at > 0)
    if mistake == "last token before this one dropped":
        hidden |= (key == at - 1) & (at > 1)
    scale = (0.9 if mistake == "scale" else 1.0) / np.sqrt(D.DH)
    out = np.empty((m, D.HQ * D.DH))
    for i in range(D.HQ):
        j = i * D.HKV // D.HQ
        if mistake == "key head":
            j = i % D.HKV
        s = np.where(hidden, -np.inf, q[n - m:, i * D.DH:(i + 1) * D.DH] @ k[:, j * D.DH:(j + 1) * D.DH].T * scale)
        p = np.exp(s - s.max(1, keepdims=True))
        out[:, i * D.DH:(i + 1) * D.DH] = p / p.sum(1, keepdims=True) @ v[:, j * D.DH:(j + 1) * D.DH]
    return out @ layer.w["o"], rows


def inputs():
    """Rows (x, residual) of the prompts and then of each step, the sequences side by side."""
    g = np.random.default_rng(1)
    rows = lambda m: L.round16(g.standard_normal((m, D.D)), False)      # noqa: E731
    return [(rows(m), rows(m)) for m in [sum(LENS)] + STEPS * [len(LENS)]]


def reference(layer, mistake=None):
    """Per prompt and then per token and sequence: the output projection's rows."""
    (x, res), *steps = inputs()
    out, past, at = [], [], 0
    for n in LENS:
        o, c = attention(layer, x[at:at + n].astype(np.float64), res[at:at + n].astype(np.float64),
                         np.empty((0, D.R)), mistake)
        out.append(o)
        past.append(c)
        at += n
    for x, res in steps:
        for b in range(len(LENS)):
            o, past[b] = attention(layer, x[b:b + 1].astype(np.float64), res[b:b + 1].astype(np.float64), past[b], mistake)
            out.append(o)
    return out


def errors(got, want):
    return [float(np.linalg.norm(a - b) / np.linalg.norm(b)) for a, b in zip(got, want)]


@pytest.fixture
def host_layer(monkeypatch):
    """The layer of the GPU test with its weights on the host only."""
    monkeypatch.setattr(B, "DeviceLayer", lambda pl: None)
    monkeypatch.setattr(H, "dev", lambda a: a)
    return D.Layer()


@pytest.mark.parametrize("mistake", ["own token hidden", "next token seen", "first row dropped",
                                     "last token before this one dropped", "scale", "key head"])
def test_planted_mistakes_pass_the_bound(host_layer, mistake):
    """Prompts and tokens each show the mistake by twice the bound (what quantization
    adds may point the other way).  A token has no next one."""
    err = errors(reference(host_layer, mistake), reference(host_layer))
    prompts, tokens = err[:len(LENS)], err[len(LENS):]
    H.say(f"{mistake}: prompts {min(prompts):.3f} to {max(prompts):.3f}, tokens {min(tokens):.3f} to {max(tokens):.3f}")
    assert max(prompts) > 2 * PROMPT
    assert max(tokens) > 2 * TOKEN or mistake == "next token seen"


def test_reference_is_that_of_the_layer(host_layer):
    """The projection's rows, put through the rest of the layer, are its 64-bit output."""
    (x, res), *_ = inputs()
    n = LENS[0]
    x, res = x[:n].astype(np.float64), res[:n].astype(np.float64)
    o, rows = attention(host_layer, x, res, np.empty((0, D.R)))
    want, c = host_layer.ref(x, res, np.empty((0, D.R)))
    h2 = o + x + res
    gu = h2 / np.sqrt((h2 ** 2).mean(1, keepdims=True) + D.EPS) * host_layer.gamma[1] @ host_layer.w["up"]
    got = L.silu_mul(gu[:, :D.F], gu[:, D.F:]) @ host_layer.w["down"] + h2
    assert np.allclose(got, want, rtol=1e-12, atol=1e-12) and np.array_equal(rows, c)


@pytest.mark.gpu
def test_attention_of_the_layer_prompts_then_tokens():
    t = H.torch()
    assert t.cuda.is_available(), "GPU tests need a GPU"
    outs = []

    class Seen(D.Layer):
        def linear(self, name, qs, res=None):
            y = super().linear(name, qs, res)
            if name == "o":
                outs.append(y.double().cpu().numpy())
            return y

    layer = Seen()
    cache = B.DeviceCache(B.QSVD_CACHE_F16, len(LENS), 80, D.R, LENS)
    up = lambda a: H.dev(a.astype(np.float16))                        # noqa: E731
    (x, res), *steps = inputs()
    layer.prompt(up(x), up(res), LENS, cache)
    for x, res in steps:
        layer.token(up(x), up(res), cache)
    t.cuda.synchronize()
    prompt, *tokens = outs
    got = np.split(prompt, np.cumsum(LENS)[:-1]) + [o[b:b + 1] for o in tokens for b in range(len(LENS))]
    err = errors(got, reference(layer))
    H.say("attention's part: prompts " + " ".join(f"{e:.4f}" for e in err[:len(LENS)]) + ", tokens " +
          " ".join(f"{e:.4f}" for e in err[len(LENS):]))
    assert max(err[:len(LENS)]) <= PROMPT and max(err[len(LENS):]) <= TOKEN
    assert H.host(cache.seq_len).tolist() == [n + STEPS for n in LENS]
