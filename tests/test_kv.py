"""The paged key-value cache's C entries without a GPU: what they refuse, and sizes.  (Addresses are made up: a refused call reads nothing.)"""
import ctypes as C

import pytest

from paper_2211_17192_amd import binding as b

AT = 1 << 40


def cache(**kw):
    c = b._KvCache(pool=AT, exps=AT + 4096, page_table=AT + 8192, dtype=b.SD_E4M3, n_pages=100, n_seq=4, table_stride=25, page_size=16, n_kv_heads=8, d_head=128)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    r = b._KvRows(k=AT, v=AT + 65536, k_row_stride=1024, k_head_stride=128, v_row_stride=1024, v_head_stride=128, dtype=b.SD_BF16)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def refused(status, word, st):
    assert st == status, (st, b.lib.sd_last_error(None))
    assert word in (b.lib.sd_last_error(None) or b"").decode()


BAD_CACHES = [(dict(pool=None), "null"), (dict(page_table=None), "null"), (dict(exps=None), "exps"), (dict(dtype=b.SD_F32), "SD_BF16 or SD_E4M3"), (dict(dtype=3), "SD_BF16 or SD_E4M3"),
              (dict(pool=AT + 8), "aligned"), (dict(exps=AT + 4), "aligned"), (dict(d_head=96), "d_head"), (dict(d_head=0), "d_head"), (dict(page_size=8), "page_size"),
              (dict(page_size=48), "page_size"), (dict(page_size=0), "page_size"), (dict(n_pages=0), "size"), (dict(n_seq=0), "size"), (dict(table_stride=0), "size"), (dict(n_kv_heads=0), "size"),
              (dict(n_kv_heads=70000), "kv heads"), (dict(page_size=1 << 29), "2^28")]


@pytest.mark.parametrize("kw,word", BAD_CACHES)
def test_bad_caches_are_refused(kw, word):
    c = C.byref(cache(**kw))
    for f in (b.lib.sd_kv_append, b.lib.sd_kv_read):
        refused(b.SD_EINVAL, word, f(c, C.byref(rows()), None, AT, 4, None))
    refused(b.SD_EINVAL, word, b.lib.sd_kv_attention(c, AT, 4096, 128, b.SD_BF16, AT, 32, 1, 100, 0.1, AT, None, AT, 1 << 30, None))
    assert b.lib.sd_kv_attention_scratch_bytes(c, 32, 1, 100) == 0


def test_a_bf16_cache_needs_no_exponents():
    assert b.lib.sd_kv_attention_scratch_bytes(C.byref(cache(dtype=b.SD_BF16, exps=None)), 32, 1, 100) > 0


@pytest.mark.parametrize("kw,word", [(dict(k=None), "null"), (dict(v=None), "null"), (dict(dtype=b.SD_E4M3), "SD_F32 or SD_BF16"), (dict(k=AT + 2), "aligned"), (dict(v=AT + 8), "aligned"),
                                     (dict(k_row_stride=1020), "strides"), (dict(v_head_stride=129), "strides")])
def test_bad_rows_are_refused(kw, word):
    for f in (b.lib.sd_kv_append, b.lib.sd_kv_read):
        refused(b.SD_EINVAL, word, f(C.byref(cache()), C.byref(rows(**kw)), None, AT, 4, None))


def test_bad_numbers_of_rows_are_refused_and_none_is_fine():
    for f in (b.lib.sd_kv_append, b.lib.sd_kv_read):
        refused(b.SD_EINVAL, "negative", f(C.byref(cache()), C.byref(rows()), None, AT, -1, None))
        refused(b.SD_ERANGE, "too many", f(C.byref(cache(n_kv_heads=64)), C.byref(rows()), None, AT, 0x7ffffffc, None))
        refused(b.SD_EINVAL, "same number", f(C.byref(cache()), C.byref(rows()), None, AT, 5, None))
        refused(b.SD_EINVAL, "null", f(C.byref(cache()), None, None, AT, 4, None))
        refused(b.SD_EINVAL, "null", f(None, C.byref(rows()), None, AT, 4, None))
        assert f(C.byref(cache()), C.byref(rows()), None, None, 0, None) == b.SD_OK


GOOD = dict(q=AT, row=4096, head=128, dtype=b.SD_BF16, pos=AT, n_heads=32, rows=1, max_len=400, scale=0.1, out=AT, scratch=AT, nbytes=1 << 30)


@pytest.mark.parametrize("kw,status,word", [
    (dict(q=None), b.SD_EINVAL, "null"), (dict(pos=None), b.SD_EINVAL, "null"), (dict(out=None), b.SD_EINVAL, "null"), (dict(scratch=None), b.SD_EINVAL, "null"),
    (dict(dtype=b.SD_E4M3), b.SD_EINVAL, "SD_F32 or SD_BF16"), (dict(q=AT + 4), b.SD_EINVAL, "aligned"), (dict(out=AT + 4), b.SD_EINVAL, "aligned"), (dict(scratch=AT + 4), b.SD_EINVAL, "aligned"),
    (dict(row=4097), b.SD_EINVAL, "strides"), (dict(head=4), b.SD_EINVAL, "strides"), (dict(n_heads=31), b.SD_EINVAL, "n_heads"), (dict(n_heads=0), b.SD_EINVAL, "n_heads"),
    (dict(rows=0), b.SD_EINVAL, "rows"), (dict(rows=-3), b.SD_EINVAL, "rows"), (dict(max_len=0), b.SD_ERANGE, "max_len"), (dict(max_len=b.SD_KV_MAX_LEN + 1), b.SD_ERANGE, "max_len"),
    (dict(scale=0.0), b.SD_EINVAL, "scale"), (dict(scale=-1.0), b.SD_EINVAL, "scale"), (dict(scale=float("nan")), b.SD_EINVAL, "scale"), (dict(scale=float("inf")), b.SD_EINVAL, "scale"),
    (dict(nbytes=1000), b.SD_ENOMEM, "scratch"), (dict(rows=1 << 20), b.SD_ERANGE, "rows")])
def test_bad_attention_calls_are_refused(kw, status, word):
    a = dict(GOOD, **kw)
    refused(status, word, b.lib.sd_kv_attention(C.byref(cache()), a["q"], a["row"], a["head"], a["dtype"], a["pos"], a["n_heads"], a["rows"], a["max_len"], a["scale"], a["out"],
                                                None, a["scratch"], a["nbytes"], None))


def test_sizes_out_of_range():
    refused(b.SD_ERANGE, "sequences", b.lib.sd_kv_attention(C.byref(cache(n_seq=70000)), AT, 4096, 128, b.SD_BF16, AT, 8, 1, 100, 0.1, AT, None, AT, 1 << 30, None))
    refused(b.SD_ERANGE, "SD_KV_MAX_GROUPS", b.lib.sd_kv_attention(C.byref(cache(n_seq=9000)), AT, 4096, 128, b.SD_BF16, AT, 8, 1, 100, 0.1, AT, None, AT, 1 << 30, None))


def test_the_largest_calls_are_told_from_those_beyond():
    """A launch has less than 2^32 threads: 2^24 workgroups of 4096 bytes of rows.  """
    for dtype, d, heads in ((b.SD_BF16, 128, 8), (b.SD_F32, 32, 64), (b.SD_F32, 128, 2)):
        row = d * (2 if dtype == b.SD_BF16 else 4)
        most = ((1 << 24) // heads - 1) * (4096 // row)
        c, r = cache(n_kv_heads=heads, d_head=d, n_seq=1), rows(dtype=dtype)
        refused(b.SD_ERANGE, "too many", b.lib.sd_kv_append(C.byref(c), C.byref(r), None, AT, most + 1, None))
        refused(b.SD_ERANGE, "too many", b.lib.sd_kv_read(C.byref(c), C.byref(r), None, AT, most + 1, None))
    refused(b.SD_EINVAL, "scale", b.lib.sd_kv_attention(C.byref(cache()), AT, 4096, 128, b.SD_BF16, AT, 32, 1, 400, 3e38, AT, None, AT, 1 << 30, None))
    # many groups of rows times many ranges of a long context
    assert b.lib.sd_kv_attention_scratch_bytes(C.byref(cache(n_seq=1, n_kv_heads=1)), 4, 4160, b.SD_KV_MAX_LEN) >= 520 * 128 * 32 * 130 * 4


@pytest.mark.parametrize("n_seq,H,Hkv,R,max_len", [(1, 8, 8, 1, 1), (1, 32, 8, 1, 131072), (1, 32, 8, 16, b.SD_KV_MAX_LEN), (64, 32, 8, 5, 8192), (300, 64, 64, 1, 5000), (3, 40, 1, 7, 257)])
def test_scratch_holds_what_the_ranges_leave(n_seq, H, Hkv, R, max_len):
    """Tickets, and per (sequence, group of up to 32 rows, kv head) and range of at most 4096 keys d_head + 2 floats a row."""
    n = b.lib.sd_kv_attention_scratch_bytes(C.byref(cache(n_seq=n_seq, n_kv_heads=Hkv)), H, R, max_len)
    assert n >= 4 * 65536
    per_range = 4 * n_seq * Hkv * R * (H // Hkv) * 130
    assert n - 4 * 65536 >= (-(-max_len // 4096) * per_range if max_len > 4096 else 0)
    assert n - 4 * 65536 <= 2 * min(128, -(-max_len // 128)) * per_range


# ------------------------------------------------------------------ a target with an 8-bit cache
from oracle import transformer as T                     # noqa: E402
from paper_2211_17192_amd import synth                  # noqa: E402
from test_launches import launches, pair, run           # noqa: E402, F401


def workspace(cfg_p, cfg_q, flags, batch=1):
    rt = b._RuntimeCfg(batch=batch, max_gamma=4, page_size=16, flags=flags)
    return b.lib.sd_workspace_bytes(C.byref(b._cfg_struct(cfg_p)), C.byref(b._cfg_struct(cfg_q)), C.byref(rt))


def test_an_8_bit_cache_takes_half_the_memory_and_one_layer():
    cfg = synth.model_cfg(T.GQA, 16, 256, 8, 512, 512, 4096, n_kv_heads=8, d_head=128, dtype="bf16")
    small = dict(cfg, n_layers=1)
    layer = 8 * 4096 * 2 * 8 * 128                      # rows of one layer's cache, 8 sequences
    saved = workspace(cfg, small, 0, 8) - workspace(cfg, small, b.SD_FLAG_KV_E4M3, 8)
    exps = layer // 128
    assert 16 * layer - 16 * exps - 2 * layer - (64 << 20) <= saved <= 16 * layer - 16 * exps - 2 * layer + (1 << 20)


def test_targets_with_a_position_bias_have_no_8_bit_cache():
    cfg, draft = pair(T.T5DEC, enc_len=61)
    gqa, _ = pair(T.GQA, n_kv_heads=2)
    assert workspace(cfg, draft, b.SD_FLAG_KV_E4M3) == 0 and workspace(cfg, draft, 0) > 0
    assert workspace(gqa, draft, b.SD_FLAG_KV_E4M3) > 0            # (a draft may have one: its cache stays as it is)


@pytest.mark.parametrize("arch,dtype,kw,batch", [(T.GPT, "f32", {}, 1), (T.GPT, "bf16", {}, 1), (T.GQA, "bf16", dict(n_kv_heads=2), 18)])
def test_what_a_target_with_an_8_bit_cache_launches(run, arch, dtype, kw, batch):       # noqa: F811
    """Each layer of a verify forward appends and attends over the 8-bit cache; a prompt's layers append and, but for the last, read back for the
    attention of the storage type.  The draft launches what it always does."""
    calls = [f"load {batch} 4 33 1 0", *(f"prefill {i} 100" for i in range(batch)), "time 0 4", "time 1 1"]
    out = run(*pair(arch, dtype=dtype, **kw), *calls)
    kinds = lambda lines: [next((k for k in ("kv_append", "kv_read", "kv_attention", "attn_mma", "attn_kernel") if k in n), None) for _, n, _, _ in launches(lines)]
    prompt, verify, draft = (([k for k in kinds(lines) if k]) for lines in (out[1], out[-2], out[-1]))
    assert verify == ["kv_append", "kv_attention"] * 2
    own = "attn_mma" if dtype == "bf16" else "attn_kernel"
    assert draft == [own]
    per_pass = ["kv_append", "kv_read", own, "kv_append"]
    assert prompt[:4] == per_pass and prompt.count("kv_append") == 2 * prompt.count("kv_read") and "kv_attention" not in prompt
    calls[0] = f"load {batch} 4 1 1 0"
    assert not any(k and k.startswith("kv_") for lines in run(*pair(arch, dtype=dtype, **kw), *calls) for k in kinds(lines))
