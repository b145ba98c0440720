"""Host checks of the paged-cache and log-probability entry points: every refusal comes before
the device is touched (these run without one), and sizes are what the header says."""

import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

from paper_2408_07802_amd import kraken as K

OK, INVALID, UNSUPPORTED = K.OK, K.ERR_INVALID_ARG, K.ERR_UNSUPPORTED
A = 4096                 # stands for a device address: no call here gets as far as using one


def cache(**kw):
    c = K._PagedCache(A, A, None, K.DTYPE_F16, 2, 2, 64, 10, 16, 3, 4, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(data=A, sub=4096, row=512):
    return K._Rows(data, sub, row)


BAD_CACHES = [
    (dict(dtype=4), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
    (dict(head_dim=0), UNSUPPORTED), (dict(n_sub=0), INVALID), (dict(n_sub=65536), INVALID),
    (dict(n_kv_heads=0), INVALID), (dict(num_pages=0), INVALID), (dict(page_size=0), INVALID),
    (dict(page_size=-16), INVALID), (dict(num_seqs=0), INVALID), (dict(num_seqs=257), INVALID),
    (dict(pages_per_seq=0), INVALID), (dict(table_ld=3), INVALID),
    (dict(pages_per_seq=1 << 27, table_ld=1 << 27), INVALID),
    (dict(n_sub=65535, n_kv_heads=65535, num_pages=2 ** 31 - 1), INVALID),
    (dict(page_size=1 << 24, pages_per_seq=1, table_ld=1), UNSUPPORTED),    # 2^32 bytes a page
]
BAD_POINTERS = [
    (dict(pages=None), INVALID), (dict(table=None), INVALID), (dict(pages=A + 8), INVALID),
    (dict(scales=A), INVALID), (dict(dtype=K.DTYPE_E4M3), INVALID),
]


def append(dtype=K.DTYPE_F16, q=True, k=True, v=True, q_out=True, k_out=None, T=3, heads=4,
           pos=A, seq=None, freq=None, rot=0, c=None, fault=None):
    pick = lambda r: rows() if r is True else r   # noqa: E731
    arr = None if freq is None else (ctypes.c_double * len(freq))(*freq)
    return K.lib().kraken_op_paged_append(
        dtype, pick(q), pick(k), pick(v), pick(q_out), pick(k_out), T, heads, pos, seq,
        ctypes.cast(arr, ctypes.c_void_p) if arr else None, rot, 0,
        cache() if c is None else c, fault, None)


def attention(dtype=K.DTYPE_F16, q=True, out=True, heads=4, lens=A, max_len=64, scale=0.0,
              work=A, floats=1 << 40, c=None):
    pick = lambda r: rows() if r is True else r   # noqa: E731
    return K.lib().kraken_op_paged_attention(dtype, pick(q), pick(out), heads,
                                             cache() if c is None else c, lens, max_len, scale,
                                             work, floats, None, None)


@pytest.mark.parametrize("kw,status", BAD_CACHES + BAD_POINTERS)
def test_bad_caches_are_refused(kw, status):
    assert append(c=cache(**kw)) == status and K.lib().kraken_last_error()
    assert attention(c=cache(**kw), max_len=0) == status
    if (kw, status) in BAD_CACHES:
        assert K.lib().kraken_paged_cache_bytes(cache(**kw)) == 0
        assert K.lib().kraken_paged_attention_work_floats(cache(**kw), 4, 1) < 0


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(dtype=K.DTYPE_BF16), UNSUPPORTED), (dict(T=-1), INVALID), (dict(T=4), INVALID),
    (dict(T=4194305, seq=A), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(pos=None), INVALID),
    (dict(q=None), INVALID), (dict(q_out=None), INVALID), (dict(heads=0), INVALID),
    (dict(heads=3), INVALID), (dict(rot=4), INVALID), (dict(rot=72), INVALID),
    (dict(rot=-8), INVALID), (dict(rot=8), INVALID),
    (dict(rot=8, freq=[1.0, 0.1, math.nan, 0.0]), INVALID),
    (dict(rot=8, freq=[1.0, 0.1, 0.2, math.inf]), INVALID),
    (dict(q=rows(A + 2)), INVALID), (dict(k=rows(None)), INVALID),
    (dict(v=rows(row=513)), INVALID), (dict(k=rows(sub=4097)), INVALID),
    (dict(k_out=rows(row=-512)), INVALID), (dict(q_out=rows(row=128)), INVALID),
    (dict(q_out=rows(sub=0)), INVALID), (dict(k_out=rows(row=0)), INVALID),
    (dict(dtype=K.DTYPE_F32, c=cache(dtype=K.DTYPE_E4M3, scales=A)), UNSUPPORTED),
    # strides of a row each, or that meet further on: sub-layer 1's rows are some of sub-layer 0's
    (dict(q_out=rows(sub=256, row=256)), INVALID), (dict(q_out=rows(sub=512, row=256)), INVALID),
    (dict(k_out=rows(sub=256, row=136)), INVALID),
])
def test_append_refuses(kw, status):
    assert append(**kw) == status and K.lib().kraken_last_error()


def test_append_of_nothing_is_nothing():
    assert append(T=0) == OK
    assert append(T=0, k=None, v=None, pos=None, q=None, q_out=None) == OK
    assert append(T=0, q=rows(None), q_out=rows(None)) == OK


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=K.DTYPE_F32), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(lens=None), INVALID),
    (dict(heads=5), INVALID), (dict(heads=0), INVALID), (dict(max_len=-1), INVALID),
    (dict(max_len=65), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
    (dict(q=rows(A + 4)), INVALID), (dict(out=rows(row=128)), INVALID),
    (dict(out=rows(sub=128)), INVALID), (dict(work=A + 4), INVALID), (dict(floats=-1), INVALID),
    (dict(dtype=K.DTYPE_F32, c=cache(dtype=K.DTYPE_E4M3, scales=A)), UNSUPPORTED),
    (dict(out=rows(sub=256, row=256)), INVALID), (dict(out=rows(sub=512, row=256)), INVALID),
])
def test_attention_refuses(kw, status):
    assert attention(**kw) == status and K.lib().kraken_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), UNSUPPORTED), (dict(logits=None), INVALID), (dict(logits=A + 2), INVALID),
    (dict(rows=-1), INVALID), (dict(vocab=0), INVALID), (dict(ld=99), INVALID),
    (dict(rows=4194305), UNSUPPORTED),
    (dict(top=-1), INVALID), (dict(top=65), INVALID), (dict(top=5, vocab=4, ld=4), INVALID),
    (dict(tokens=None), INVALID), (dict(logprob=None), INVALID), (dict(ids=None), INVALID),
    (dict(best=None), INVALID), (dict(top=0), INVALID), (dict(work=A + 4), INVALID),
    (dict(floats=-1), INVALID),
])
def test_logprobs_refuse(kw, status):
    a = dict(dtype=0, logits=A, ld=100, rows=2, vocab=100, tokens=A, logprob=A, entropy=A, top=5,
             ids=A, best=A, work=A, floats=1 << 40)
    a.update(kw)
    assert K.lib().kraken_op_token_logprobs(
        a["dtype"], a["logits"], a["ld"], a["rows"], a["vocab"], a["tokens"], a["logprob"],
        a["entropy"], a["top"], a["ids"], a["best"], a["work"], a["floats"], None) == status
    assert K.lib().kraken_last_error()


def test_attention_refuses_2_30_tiles():
    # 65535 sub-layers of 2 heads of 256 sequences of 2049 keys: 33 tiles of 64 keys each
    c = cache(n_sub=65535, num_seqs=256, pages_per_seq=257, table_ld=257)
    assert 65535 * 2 * 256 * 33 >= 2 ** 30
    assert attention(c=c, max_len=2049) == UNSUPPORTED
    assert b"tiles" in K.lib().kraken_last_error()
    # as many units without any key
    c = cache(n_sub=65535, n_kv_heads=65, num_seqs=256)
    assert attention(c=c, heads=65, max_len=0, q=rows(row=65536, sub=1 << 24),
                     out=rows(row=65536, sub=1 << 24)) == UNSUPPORTED


def test_sizes():
    assert K.lib().kraken_paged_cache_bytes(cache()) == 2 * 2 * 10 * 2 * 16 * 64 * 2
    assert K.lib().kraken_paged_cache_bytes(cache(dtype=0, page_size=7)) == 2 * 2 * 10 * 2 * 7 * 64 * 4
    big = cache(dtype=K.DTYPE_E4M3, n_sub=8, n_kv_heads=16, head_dim=128, num_pages=1 << 20)
    assert K.lib().kraken_paged_cache_bytes(big) == 8 * 2 * 16 * 128 * 16 << 20
    assert K.lib().kraken_paged_cache_bytes(None) == 0
    f = K.lib().kraken_paged_attention_work_floats
    assert f(cache(), 4, 0) >= 0 and f(cache(), 4, 64) >= 0
    assert f(cache(), 3, 64) < 0 and f(cache(), 4, 65) < 0 and f(cache(), 4, -1) < 0
    g = K.lib().kraken_token_logprobs_work_floats
    assert g(0, 10, 0) == 0 and g(1, 51200, 64) >= 0
    assert g(-1, 10, 0) < 0 and g(1, 0, 0) < 0 and g(1, 10, 65) < 0 and g(1, 10, 11) < 0


# --------------------------------------------------------------- the binding's own checks

class Fake:
    """A CPU tensor that says it is on a GPU (the binding reads no element)."""

    def __init__(self, t, index=0):
        self.t, self.is_cuda, self.device = t, True, torch.device("cuda", index)

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_binding_refuses_wrong_tensors(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    h = torch.float16
    pages = Fake(torch.zeros((2, 2, 10, 2, 16, 64), dtype=h))
    table = Fake(torch.zeros((3, 4), dtype=torch.int32))
    q, kv = Fake(torch.zeros((2, 3, 256), dtype=h)), Fake(torch.zeros((2, 3, 128), dtype=h))
    i3 = Fake(torch.zeros(3, dtype=torch.int32))
    freq = torch.ones(32, dtype=torch.float64)
    good = dict(q=q, k=kv, v=kv, pages=pages, table=table, pos=i3, q_out=q, inv_freq=freq)
    cases = [
        (dict(q=torch.zeros((2, 3, 256), dtype=h)), "GPU tensor"),
        (dict(q=Fake(torch.zeros((2, 3, 256)))), "dtype"),
        (dict(q=Fake(torch.zeros((2, 3, 250), dtype=h))), "head_dim"),
        (dict(k=Fake(torch.zeros((2, 4, 128), dtype=h))), "shape"),
        (dict(v=Fake(torch.zeros((2, 128, 3), dtype=h).transpose(1, 2))), "adjacent"),
        (dict(q_out=Fake(torch.zeros((2, 3, 256), dtype=h), index=1)), "is on"),
        (dict(q=None), "without q"), (dict(k_out=q), "shape"),
        (dict(pos=Fake(torch.zeros(3, dtype=torch.int64))), "int32"),
        (dict(seq=Fake(torch.zeros(2, dtype=torch.int32))), "int32"),
        (dict(table=Fake(torch.zeros((4, 3), dtype=torch.int32).t())), "adjacent"),
        (dict(pages=Fake(torch.zeros((2, 2, 10, 2, 64, 16), dtype=h).transpose(4, 5))),
         "contiguous"),
        (dict(pages=Fake(torch.zeros((2, 2, 10, 2, 16, 64), dtype=torch.float64))), "dtype"),
        (dict(inv_freq=Fake(freq)), "host"), (dict(inv_freq=freq.float()), "host"),
        (dict(scales=Fake(torch.zeros((2, 2, 3)))), "float32"),
        (dict(fault=Fake(torch.zeros(2, dtype=torch.int32))), "int32"),
    ]
    for kw, pat in cases:
        with pytest.raises(ValueError, match=pat):
            K.op_paged_append(**{**good, **kw})
    good = dict(q=q, pages=pages, table=table, lens=i3, max_len=64, out=q,
                work=Fake(torch.zeros(1 << 22)))
    cases = [
        (dict(q=Fake(torch.zeros((2, 2, 256), dtype=h))), "shape"),
        (dict(out=Fake(torch.zeros((2, 3, 256)))), "dtype"),
        (dict(lens=Fake(torch.zeros(4, dtype=torch.int32))), "int32"), (dict(lens=None), "lens"),
        (dict(work=Fake(torch.zeros(1 << 22, dtype=h))), "float32"),
        (dict(work=torch.zeros(1 << 22)), "GPU tensor"),
    ]
    for kw, pat in cases:
        with pytest.raises(ValueError, match=pat):
            K.op_paged_attention(**{**good, **kw})
    x = Fake(torch.zeros((3, 100)))
    for args, pat in [((torch.zeros((3, 100)),), "GPU tensor"),
                      ((Fake(torch.zeros((100, 3)).t()),), "adjacent"),
                      ((Fake(torch.zeros(3, 100, dtype=torch.float64)),), "dtype"),
                      ((x, Fake(torch.zeros(3, dtype=torch.int64))), "int32"),
                      ((x, Fake(torch.zeros(4, dtype=torch.int32))), "int32"),
                      ((x, i3, 65), "top"), ((x, i3, -1), "top")]:
        with pytest.raises(ValueError, match=pat):
            K.op_token_logprobs(*args)
    # another device than the current one
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        K.op_paged_append(q, kv, kv, pages, table, i3, q)


# -------------------------------------------------------- the kernels' index arithmetic, on the host

@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_index_arithmetic_under_the_sanitizers(tmp_path):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "paged_driver.cpp")
    exe = str(tmp_path / "driver")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined",
                          "-fno-sanitize-recover=all", src, "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120,
                         env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert res.returncode == 0 and "holds" in res.stdout, res.stdout + res.stderr[-3000:]
