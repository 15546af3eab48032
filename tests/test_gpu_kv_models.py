"""GPU: a target whose KV cache is kept in 8 bits (SD_FLAG_KV_E4M3), through sd_prefill, sd_step and sd_step_baseline.

The oracle is the usual one with keys and values rounded as the cache rounds them.  A key or value that lies closer to the middle of two codes than the two
sides' arithmetic agrees is rounded the other way by one of them: one element then differs by a step, where every element's own rounding is off by up to half of one.
Of n elements that is a share of about 4 / sqrt(n) of what the rounding as a whole changes (n is 10^4 and more here, and few lie that close in fp32), so logits
are held to the model's usual tolerance plus a quarter of the distance between the oracle's models with and without rounding; a target that did not round
would be off by that whole distance."""
import numpy as np
import pytest
import torch

from oracle import transformer as T
from paper_2211_17192_amd import synth
from pairs import W_STD, row_rel_err as rel_err
from test_gpu_models import TOL, check_level_s, make_decoder
from test_gpu_kv import pow2, quantised

pytestmark = pytest.mark.gpu


class Rounded(T.Transformer):
    """Keys and values through the 8-bit cache (rounding twice is rounding once)."""

    def _attend(self, q, keys, vals, *args):
        def through(x):
            c, e = quantised(torch.from_numpy(x.reshape(len(x), -1, self.cfg.d_head)))
            return (c * pow2(e).unsqueeze(-1)).numpy().reshape(x.shape)
        return super()._attend(q, through(keys), through(vals), *args)


def pair(arch, dtype, d_head, seed=5, max_len=200, heads=4, kv_heads=2, d_model=128):
    kw = dict(dtype=dtype, logit_scale=4.0, d_head=d_head)
    if arch == T.GQA:
        kw["n_kv_heads"] = kv_heads
    cfg = synth.model_cfg(arch, 2, d_model, heads, 160, 512, max_len, **kw)
    w = synth.random_weights(cfg, seed, w_std=W_STD[dtype])
    cfg_q, w_q = synth.truncated_noisy_copy(cfg, w, 1, seed + 50, 0.02)
    return cfg, w, cfg_q, w_q


def scorers(cfg, w):
    n = synth.to_numpy_weights(w)
    return T.CachedScorer(Rounded(T.ModelConfig(**cfg), n)), T.CachedScorer(T.Transformer(T.ModelConfig(**cfg), n))


def check_logits(z, rounded, plain, dtype, where):
    assert np.isfinite(z).all()
    off, whole = rel_err(z, rounded), rel_err(plain, rounded)
    assert off <= TOL[dtype] + whole / 4, (where, off, whole)
    return off, whole


@pytest.mark.parametrize("arch,dtype,d_head,heads", [(T.GPT, "f32", 32, 4), (T.GQA, "f32", 32, 4), (T.GQA, "f32", 128, 8), (T.GPT, "bf16", 64, 4), (T.GQA, "bf16", 64, 8),
                                                     (T.GQA, "bf16", 128, 8), (T.GPT, "bf16", 32, 4)])
@pytest.mark.parametrize("temperature,flags", [(1.0, 1), (0.0, 0)])
def test_decoding_matches_the_oracle_with_a_rounded_cache(arch, dtype, d_head, heads, temperature, flags):
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(arch, dtype, d_head, heads=heads, kv_heads=2)
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=5, flags=flags | binding.SD_FLAG_KV_E4M3)
    rounded, plain = scorers(cfg, w)
    prefix = [int(t) for t in synth.random_tokens(3, 37, 512)]
    dec.prefill(prefix)
    u = synth.uniform_stream(4, 12 * 11).reshape(12, 11)
    gaps = []
    for it, gamma in enumerate((5, 3, 5, 1, 4, 5)):
        n, toks = dec.step(gamma, temperature, u[it, :2 * gamma + 1], prefix=prefix)
        zp, zq = dec.logits(0, gamma + 1).astype(np.float64), dec.logits(1, gamma).astype(np.float64)
        x = check_level_s(n, toks, zp, zq, u[it, :2 * gamma + 1], gamma, temperature, {"accept": 0, "draw": 0}, f"iteration {it}")
        gaps.append(check_logits(zp, rounded.score(prefix + x, gamma + 1), plain.score(prefix + x, gamma + 1), dtype, it)[1])
        prefix = prefix + toks
    assert max(gaps) > 1e-3                            # (the rounding shows)


@pytest.mark.parametrize("dtype,d_head", [("bf16", 128), ("f32", 64)])
def test_long_contexts_and_prompts(dtype, d_head):
    """Contexts of several key ranges; a prompt in passes of many rows (bf16) or 16, then plain steps."""
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(T.GQA, dtype, d_head, max_len=1400, heads=8, kv_heads=2)
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=4, flags=1 | binding.SD_FLAG_KV_E4M3)
    rounded, plain = scorers(cfg, w)
    prefix = [int(t) for t in synth.random_tokens(6, 1203, 512)]
    dec.prefill(prefix)
    n, toks = dec.step(4, 1.0, synth.uniform_stream(7, 9))
    zp, zq = dec.logits(0, 5).astype(np.float64), dec.logits(1, 4).astype(np.float64)
    x = check_level_s(n, toks, zp, zq, synth.uniform_stream(7, 9), 4, 1.0, {"accept": 0, "draw": 0})
    check_logits(zp, rounded.score(prefix + x, 5), plain.score(prefix + x, 5), dtype, "step")
    prefix = prefix + toks
    for it in range(2):
        tok = dec.step_baseline(0.0)
        z = dec.logits(2, 1).astype(np.float64)
        check_logits(z, rounded.score(prefix, 1), plain.score(prefix, 1), dtype, f"plain {it}")
        assert tok == int(z[0].argmax())
        prefix.append(tok)


def logits_of(dec, prompt, steps=3, gamma=4, temperature=1.0):
    dec.prefill(prompt)
    out, u = [], synth.uniform_stream(9, steps * 9).reshape(steps, 9)
    for i in range(steps):
        n, toks = dec.step(gamma, temperature, u[i])
        out.append((n, toks, dec.logits(0, gamma + 1).copy()))
    return out


def same(a, b):
    return all(x[:2] == y[:2] and np.array_equal(x[2], y[2]) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,d_head", [("bf16", 128), ("bf16", 64), ("f32", 32)])
def test_pages_workspaces_and_graphs_do_not_change_a_bit(dtype, d_head):
    """Scattered pages; prompt passes of fewer rows, down to 16; replayed graphs; the same context again after a reset."""
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(T.GQA, dtype, d_head, max_len=1100, heads=8, kv_heads=2)
    prompt = [int(t) for t in synth.random_tokens(8, 701, 512)]
    kv = binding.SD_FLAG_KV_E4M3
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=4, flags=kv)
    first = logits_of(dec, prompt)
    dec.reset()
    assert same(first, logits_of(dec, prompt))
    for flags in (kv | 1, kv | 1 | binding.SD_FLAG_SCATTER_PAGES):
        assert same(first, logits_of(make_decoder(cfg, w, cfg_q, w_q, max_gamma=4, flags=flags), prompt)), flags
    assert same(first, logits_of(make_decoder(cfg, w, cfg_q, w_q, max_gamma=4, flags=kv | 1, page_size=64), prompt))


@pytest.mark.parametrize("arch,dtype,d_head", [(T.GQA, "bf16", 128), (T.GPT, "bf16", 64), (T.GQA, "f32", 64)])
def test_argmax_decoding_is_plain_argmax_decoding(arch, dtype, d_head):
    """A row's sums do not depend on how many rows a forward has."""
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(arch, dtype, d_head, max_len=1000, heads=8, kv_heads=2)
    prompt = [int(t) for t in synth.random_tokens(10, 850, 512)]
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=3, flags=1 | binding.SD_FLAG_KV_E4M3)
    dec.prefill(prompt)
    spec = []
    while len(spec) < 24:
        spec += dec.step(3, 0.0)[1]
    dec.reset()
    dec.prefill(prompt)
    assert [dec.step_baseline(0.0) for _ in range(24)] == spec[:24]


@pytest.mark.parametrize("dtype,d_head,batch", [("bf16", 128, 5), ("bf16", 64, 40), ("f32", 32, 3)])
def test_several_sequences(dtype, d_head, batch):
    """Each sequence of a batch against its own oracle run."""
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(T.GQA, dtype, d_head, heads=4, kv_heads=2)
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=3, flags=1 | binding.SD_FLAG_KV_E4M3, batch=batch)
    prompts = [[int(t) for t in synth.random_tokens(20 + b, 5 + (37 * b) % 90, 512)] for b in range(batch)]
    for b in reversed(range(batch)):
        dec.prefill(prompts[b], row=b)
    u = synth.uniform_stream(11, 2 * batch * 7).reshape(2, batch, 7)
    checked = sorted({0, 1, batch // 2, batch - 1})
    models = {b: scorers(cfg, w) for b in checked}
    for it in range(2):
        res = dec.step(3, 1.0, u[it])
        zp, zq = dec.logits(0, 4 * batch).reshape(batch, 4, -1).astype(np.float64), dec.logits(1, 3 * batch).reshape(batch, 3, -1).astype(np.float64)
        for b in checked:
            n, toks = res[b]
            x = check_level_s(n, toks, zp[b], zq[b], u[it, b], 3, 1.0, {"accept": 0, "draw": 0}, f"sequence {b}")
            check_logits(zp[b], models[b][0].score(prompts[b] + x, 4), models[b][1].score(prompts[b] + x, 4), dtype, (it, b))
        for b in range(batch):
            prompts[b] = prompts[b] + res[b][1]


def test_measurements_and_flags():
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(T.GQA, "bf16", 64)
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=4, flags=1 | binding.SD_FLAG_KV_E4M3)
    dec.prefill([1, 2, 3, 4])
    a, b = dec.measure_cost(reps=3)
    assert a > 0 and b > 0
    assert dec.time_forward(0, 4, reps=3) > dec.time_forward(0, 4, skip_ops=511 & ~binding.SD_OP["head"], reps=3) > 0
    first = logits_of(dec, [5, 6, 7])
    dec.set_flags(1)                                   # (the cache stays as it was loaded)
    dec.reset()
    assert same(first, logits_of(dec, [5, 6, 7]))
    plain = make_decoder(cfg, w, cfg_q, w_q, max_gamma=4, flags=1)
    assert not same(first, logits_of(plain, [5, 6, 7]))
    plain.set_flags(1 | binding.SD_FLAG_KV_E4M3)       # (likewise)
    plain.reset()
    assert not same(first, logits_of(plain, [5, 6, 7]))


def test_drafts_without_mq():
    """A table draft and the copying draft over a target with an 8-bit cache."""
    from paper_2211_17192_amd import binding
    cfg, w, cfg_q, w_q = pair(T.GPT, "bf16", 64)
    dec = make_decoder(cfg, w, cfg_q, w_q, max_gamma=3, flags=1 | binding.SD_FLAG_KV_E4M3)
    rounded, plain = scorers(cfg, w)
    dec.set_copy_draft(2)
    prefix = [3, 9, 4, 3, 9, 4, 3, 9]
    dec.prefill(prefix)
    for it in range(3):
        n, toks = dec.step(3, 1.0, synth.uniform_stream(30 + it, 7))
        zp = dec.logits(0, 4).astype(np.float64)
        check_logits(zp[:n + 1], rounded.score(prefix + toks[:n], n + 1), plain.score(prefix + toks[:n], n + 1), "bf16", it)
        prefix = prefix + toks
