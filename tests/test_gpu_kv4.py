"""Decoders whose caches hold 4 bits a value, against the float64 oracle with the same
keys and values: rounded to MXFP4 in the encoder, LM module and next-byte decoder, to
float16 in the MB window."""
import ctypes

import numpy as np
import pytest

import oracle
import oracle.model as om
import paged_plain as plain
import synth
from gpu_harness import SELF_VERIFY, THRESHOLD, forced_run, new_decoder

pytestmark = pytest.mark.gpu

TINY = synth.WORKLOADS["tiny_f32"].model
# The library's keys are off by some 1e-6 of their size, so about one element in 10^5 goes
# to a neighbouring code.  One code is at most half of its block's largest value (5 to 6, 4 to 6): with
# keys near 0.25 (weights of 0.02, width 128) a score moves by 0.1 x 0.25 / sqrt(32) = 0.005,
# an output channel by that times one weight of some 1/50 times a value of 0.25, a logit by
# 2e-5 x 0.02 x sqrt(128) = 5e-6; a flipped value likewise.  A few of these, times the gain of
# the unembedding.
TOL = 5e-5


@pytest.fixture
def four_bits(monkeypatch):
    """The oracle with rounded keys and values."""
    real = om.stack

    def attention(name):
        def f(x, P, mask, pos, n_heads, rope_base, attn_scale):
            T, d = x.shape
            q, k, v = ((x @ P[w].T).reshape(T, n_heads, d // n_heads) for w in ("wq", "wk", "wv"))
            q, k = om.rope(q, pos, rope_base), om.rope(k, pos, rope_base)
            k, v = (plain.to_mxfp4(a) if name != "mb" else a.astype(np.float16).astype(np.float64) for a in (k, v))
            o = np.empty((T, n_heads, d // n_heads))
            for h in range(n_heads):
                s = np.where(mask, q[:, h] @ k[:, h].T * attn_scale / np.sqrt(d // n_heads), -np.inf)
                p = np.exp(s - s.max(-1, keepdims=True))
                o[:, h] = p / p.sum(-1, keepdims=True) @ v[:, h]
            return o.reshape(T, d) @ P["wo"].T

        return f

    def stack(u, W, name, *rest):
        monkeypatch.setattr(om, "attention", attention(name))
        return real(u, W, name, *rest)

    monkeypatch.setattr(om, "stack", stack)


def fp4_decoder(model, W, batch, max_ctx, **kw):
    from paper_2608_15454_amd import MXFP4

    return new_decoder(model, W, batch, max_ctx, kv_dtype=MXFP4, **kw)


@pytest.mark.parametrize("mode", [THRESHOLD, SELF_VERIFY])
def test_steps_of_a_batch(four_bits, mode):
    """Prompts of 1 to 150 bytes, which end inside pages; with verification the caches are
    rolled back and the dropped slots written again."""
    raw = synth.make_weights(TINY, seed=3, gain_jitter=0.2, logit_gain=20.0)
    W = oracle.to_float64(raw)
    dec = fp4_decoder(TINY, raw, 3, 260)
    prompts = [synth.make_prompt(i, n) for i, n in enumerate((1, 64, 150))]
    st = forced_run(dec, W, TINY, prompts, 6, [3, 5], 0.5, mode, tol=20 * TOL)
    assert st.max_err > 0


def test_four_bits_differ_from_float32_caches(four_bits):
    """The tolerance above tells the formats apart."""
    raw = synth.make_weights(TINY, seed=3, gain_jitter=0.2, logit_gain=20.0)
    out = []
    for kv in (0, 3):
        dec = new_decoder(TINY, raw, 1, 260, kv_dtype=kv)
        dec.prefill([synth.make_prompt(5, 150)])
        dec.decode_step(3, 0.5)
        out.append(dec.logits()[0].double().cpu().numpy())
    want = om.step_logits(oracle.to_float64(raw), TINY, synth.make_prompt(5, 150), 3)
    assert np.abs(out[1] - want).max() <= 20 * TOL < np.abs(out[0] - want).max() / 3


def test_learned_boundaries_mlp_head_and_chunks(four_bits):
    for kw, cfg in ((dict(boundary="learned"), {}), (dict(head="mlp", n_mb=3), dict(max_chunk=50)), (dict(window_mode=1), {})):
        model = TINY.replace(**kw)
        raw = synth.make_weights(model, seed=4, gain_jitter=0.2, logit_gain=20.0)
        dec = fp4_decoder(model, raw, 2, 200, **cfg)
        forced_run(dec, oracle.to_float64(raw), model, [synth.make_prompt(7, 90), synth.make_prompt(8, 33)], 3, 3, 0.5, tol=20 * TOL)


def test_full_sequence_forward(four_bits):
    raw = synth.make_weights(TINY, seed=3, gain_jitter=0.2, logit_gain=20.0)
    x = synth.make_prompt(2, 200)
    dec = fp4_decoder(TINY, raw, 1, 260)
    nll, loss = dec.forward(x)
    W = oracle.to_float64(raw)
    tr = om.trunk(W, TINY, x)
    rows = om.head_logits(tr["h1"], W["nt_norm"], W, TINY.rms_eps)[:-1]
    want = np.log(np.exp(rows - rows.max(1, keepdims=True)).sum(1)) + rows.max(1) - rows[np.arange(199), np.asarray(x[1:], int)]
    assert np.abs(nll[0, :199].double().cpu().numpy() - want).max() <= 40 * TOL


def test_split_row_passes_of_bfloat16_models():
    """Long passes of bfloat16 models take split rows; their attention output is split
    behind the 4-bit attention.  Passes of other lengths run on float32 rows: the same
    logits within the bfloat16 weights' tolerance of 4-bit flips."""
    model = synth.WORKLOADS["lca_d1024_b1"].model.replace(n_enc=1, n_lm=1, n_nb=1, n_mb=1)
    raw = synth.make_weights(model, seed=1)
    prompt = synth.make_prompt(3, 700)
    out = []
    for chunk in (0, 40):
        dec = fp4_decoder(model, raw, 1, 800, max_chunk=chunk)
        dec.prefill([prompt])
        dec.decode_step(3, 0.5)
        out.append(dec.logits()[0].double().cpu().numpy())
    assert np.isfinite(out[0]).all() and np.abs(out[0] - out[1]).max() <= 2e-2


def test_the_workspace_shrinks():
    import paper_2608_15454_amd as m

    model = synth.WORKLOADS["lca_d1024_b64"].model
    size = {kv: m.lib().mbp_workspace_bytes(ctypes.byref(m.make_config(model, max_batch=64, max_ctx=8192, max_n=5, kv_dtype=kv))) for kv in (m.F16, m.MXFP4)}
    # caches of 2 x (2 + 16 + 2) layers x 64 x 8192 x 1024 values: 40 GiB of float16, 10.6 of 4.25 bits
    assert size[m.F16] - size[m.MXFP4] > 20 << 30
