"""The paged-cache operators on the GPU, against their formulas in 64 bits.

Bounds (u: half a step of the output type, 2^-24 of fp32 arithmetic):
  * a rotated value a cos - b sin: the fp32 angle is within pi 2^-24 of the exact one, cos and
    sin within 2 ulp (2^-23) more, two products and a sum round: 8 x 2^-24 (|a| + |b|) covers
    them; then one rounding to the output type, u |value| (and half the smallest subnormal);
  * an attention output: a score, scale sum_j q_j k_j, is off by ds <= (hd + 2) 2^-24 scale
    sum |q_j k_j|, its exponential by another 2^-22 + |s - max| 2^-23 relative, the weight in two
    16-bit terms by 2^-16, a sum over len keys by len 2^-24; with D the largest of the first two
    over the keys, the output is off by (2 D + 2^-16 + 2 len 2^-24) sum p |v|, plus u |out|.
"""

import math

import pytest
import torch

from paper_2408_07802_amd import kraken as K

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11,
             F8: 2.0 ** -4}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25,
        F8: 2.0 ** -10}


def say(msg):
    print(msg, flush=True)


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def normal(shape, dtype, g, std=1.0):
    return (torch.randn(shape, generator=g) * std).to(dtype).to(DEV)


def make_cache(n, heads, hd, page, lens, dtype, g, spare=2, width=0):
    """(pages full of random values, table with -1 behind each sequence's last page)."""
    need = [-(-max(v, 0) // page) for v in lens]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g).to(torch.int32)
    table = torch.full((len(lens), max([1, width] + need)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(need):
        table[b, :c] = order[at:at + c]
        at += c
    pages = normal((n, 2, total, heads, page, hd), torch.float32, g, 30.0 if dtype == F8 else 1.0)
    return pages.to(dtype), table.to(DEV)


def rotate64(x, pos, freq, rot, neighbours, hd):
    """x [n, T, heads * hd] in 64 bits, rotated; and |a| + |b| of every element's pair."""
    x = x.double().unflatten(-1, (-1, hd))
    ang = pos.double()[:, None] * freq.to(x.device)[None]
    c, s = ang.cos()[None, :, None], ang.sin()[None, :, None]
    y, mag = x.clone(), torch.zeros_like(x)
    if rot:
        ia = torch.arange(0, rot, 2) if neighbours else torch.arange(rot // 2)
        ib = ia + 1 if neighbours else ia + rot // 2
        a, b = x[..., ia], x[..., ib]
        y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
        mag[..., ia] = mag[..., ib] = a.abs() + b.abs()
    return y.flatten(-2), mag.flatten(-2)


def near(got, ref, slack, what):
    u, tiny = HALF_STEP[got.dtype], TINY[got.dtype]
    got = got.double()
    bound = u * (ref.abs() + slack) + slack + tiny
    over = (got - ref).abs() - bound
    assert bool((over <= 0).all()), (what, float(over.max()))


APPENDS = [  # n, H, Hkv, hd, dtype, cache dtype, page, rot, neighbours, keys out, queries
    (1, 1, 1, 32, torch.float32, None, 1, 32, False, True, True),
    (2, 4, 2, 64, torch.bfloat16, None, 16, 64, False, False, True),
    (3, 6, 3, 128, torch.float16, None, 48, 104, True, True, True),
    (2, 4, 4, 128, torch.bfloat16, F8, 7, 128, True, True, True),
    (2, 8, 1, 64, torch.float16, F8, 64, 8, False, False, True),
    (8, 16, 16, 128, torch.float16, None, 16, 128, False, False, True),
    (1, 4, 2, 32, torch.bfloat16, None, 33, 24, False, True, True),
    (2, 3, 3, 64, torch.float32, None, 128, 40, True, False, True),
    (2, 2, 2, 64, torch.bfloat16, F8, 16, 0, False, False, False),
    (1, 5, 5, 32, torch.float16, None, 8, 0, False, True, True),
]


@pytest.mark.parametrize("starts,news", [
    ([0], [1]), ([5, -1, 0, 30], [1, 1, 1, 1]), ([0, 3, -1, 1000000], [37, 1, 2, 130]),
    ([2 ** 30 - 5], [4]),
], ids=["first", "step", "ragged", "far"])
@pytest.mark.parametrize("case", APPENDS, ids=[str(k) for k in range(len(APPENDS))])
def test_append(case, starts, news):
    n, H, Hkv, hd, dtype, cdt, page, rot, neighbours, keys_out, queries = case
    cdt = cdt or dtype
    far = max(starts) > 10000
    if far:
        page = 4099                         # (few pages reach far positions; most stay unused)
        if n * Hkv * hd > 256:
            n, H, Hkv = 1, H // Hkv, 1
    say(f"[append] {case} starts={starts} news={news} page={page}")
    g = gen(len(news) + 7 * rot)
    lens = [a + b if a >= 0 else 0 for a, b in zip(starts, news)]
    T, B = sum(news), len(news)
    if far:                                 # only the pages that are written exist
        width = max(lens) // page + 1
        table = torch.full((B, width), -1, dtype=torch.int32)
        used = 0
        for b, (a, c) in enumerate(zip(starts, news)):
            for j in range(a // page, (a + c - 1) // page + 1) if a >= 0 else ():
                table[b, j] = used
                used += 1
        table = table.to(DEV)
        pages = normal((n, 2, used + 1, Hkv, page, hd), dtype, g).to(cdt)
    else:
        pages, table = make_cache(n, Hkv, hd, page, lens, cdt, g)
    dq, dkv = H * hd, Hkv * hd
    qkv = normal((n, T, dq + 2 * dkv + 16), dtype, g)      # a wider row than the three need
    q, k, v = qkv[..., :dq], qkv[..., dq:dq + dkv], qkv[..., dq + dkv:dq + 2 * dkv]
    seq = torch.repeat_interleave(torch.arange(B), torch.tensor(news)).to(torch.int32).to(DEV)
    pos = torch.cat([torch.arange(c, dtype=torch.int32) + a if a >= 0 else
                     torch.full((c,), -1 - c, dtype=torch.int32)
                     for a, c in zip(starts, news)]).to(DEV)
    freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1))
    scales = (0.02 + 0.01 * torch.rand((n, 2, Hkv), generator=g)).to(DEV) if cdt == F8 else None
    q_out = torch.full((n, T, dq), 7.0, dtype=dtype, device=DEV) if queries else None
    k_out = torch.full((n, T, dkv), 7.0, dtype=dtype, device=DEV) if keys_out else None
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    before = pages.clone()
    K.op_paged_append(q if queries else None, k, v, pages, table, pos, q_out, seq=seq,
                      k_out=k_out, inv_freq=freq if rot else None, neighbours=neighbours,
                      scales=scales, fault=fault)
    torch.cuda.synchronize()
    assert int(fault) == 0
    live = pos >= 0
    kr, kmag = rotate64(k, pos, freq, rot, neighbours, hd)
    if queries:
        qr, qmag = rotate64(q, pos, freq, rot, neighbours, hd)
        near(q_out[:, live], qr[:, live], 8 * 2.0 ** -24 * qmag[:, live], "q")
        assert bool((q_out[:, ~live] == 7).all())
    if keys_out:
        near(k_out[:, live], kr[:, live], 8 * 2.0 ** -24 * kmag[:, live], "k")
        assert bool((k_out[:, ~live] == 7).all())
    # the cache: the new places, and nothing else
    where = table[seq[live].long(), (pos[live] // page).long()].long()
    off = (pos[live] % page).long()
    wrote = torch.zeros(pages.shape[2], page, dtype=torch.bool, device=DEV)
    wrote[where, off] = True
    kept = ~wrote[None, None, :, None, :, None].expand(pages.shape)
    raw = torch.uint8 if cdt == F8 else torch.int16 if cdt != torch.float32 else torch.int32
    assert torch.equal(pages.view(raw)[kept], before.view(raw)[kept])
    for j, (ref, mag) in enumerate([(kr, kmag), (v.double(), torch.zeros_like(kmag))]):
        got = pages.view(raw)[:, j][:, where, :, off].view(cdt)       # [rows, n, heads, hd]
        ref = ref[:, live].unflatten(-1, (Hkv, hd)).transpose(0, 1)
        slack = 8 * 2.0 ** -24 * mag[:, live].unflatten(-1, (Hkv, hd)).transpose(0, 1)
        if scales is not None:
            sc = scales[:, j].double()[None, :, :, None]
            ref, slack = (ref / sc).clamp(-448, 448), slack / sc + 2.0 ** -23 * (ref / sc).abs()
        near(got, ref, slack, "KV"[j])


def test_append_8_bit_saturates_and_keeps_nan():
    x = torch.tensor([0.0, -0.0, 447.9, 448.0, 449.0, 1e4, -1e4, math.inf, -math.inf, math.nan,
                      2.0 ** -9, 2.0 ** -10, 2.0 ** -10 * 1.5, 17.0, 19.0, -21.0] * 2,
                     dtype=torch.float16, device=DEV)
    pages = torch.zeros((1, 2, 1, 1, 4, 32), dtype=F8, device=DEV)
    table = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    K.op_paged_append(None, x.view(1, 1, 32), x.view(1, 1, 32), pages, table,
                      torch.tensor([2], dtype=torch.int32, device=DEV),
                      scales=torch.ones((1, 2, 1), device=DEV))
    want = x.float().clamp(-448, 448).to(F8).float()      # (a NaN passes the clamp)
    got = pages.float()[0, :, 0, 0]
    for j in (0, 1):
        assert torch.equal(got[j, 2].nan_to_num(999.0), want.nan_to_num(999.0))
        assert bool((got[j, [0, 1, 3]] == 0).all())


def test_append_in_place_and_strided_rows():
    # queries and keys of one projection turned where they are; sub-layers behind rows
    n, T, H, hd, page = 2, 5, 2, 64, 16
    g = gen(5)
    x = normal((T, n, 3 * H * hd), torch.bfloat16, g).transpose(0, 1)
    pages, table = make_cache(n, H, hd, page, [40], torch.bfloat16, g)
    pos = torch.arange(11, 16, dtype=torch.int32, device=DEV)
    seq = torch.zeros(T, dtype=torch.int32, device=DEV)
    freq = 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    d = H * hd
    p2, q2, k2 = pages.clone(), torch.empty((n, T, d), dtype=torch.bfloat16, device=DEV), \
        torch.empty((n, T, d), dtype=torch.bfloat16, device=DEV)
    K.op_paged_append(x[..., :d], x[..., d:2 * d], x[..., 2 * d:], p2, table, pos, q2, seq=seq,
                      k_out=k2, inv_freq=freq)
    v = x[..., 2 * d:].clone()
    K.op_paged_append(x[..., :d], x[..., d:2 * d], x[..., 2 * d:], pages, table, pos, x[..., :d],
                      seq=seq, k_out=x[..., d:2 * d], inv_freq=freq)
    torch.cuda.synchronize()
    assert torch.equal(x[..., :d], q2) and torch.equal(x[..., d:2 * d], k2)
    assert torch.equal(x[..., 2 * d:], v) and torch.equal(pages, p2)


def test_append_leaves_out_bad_rows():
    n, hd, page, B = 2, 32, 8, 3
    g = gen(9)
    pages, table = make_cache(n, 1, hd, page, [16, 16, 16], torch.float32, g)
    table[1, 1] = pages.shape[2]                 # one past the last page
    table[2, 0] = -5
    k = normal((n, 6, hd), torch.float32, g)
    # good, bad page, bad page, position past the table, no such sequence, good
    pos = torch.tensor([3, 9, 0, 2 ** 31 - 1, 4, 12], dtype=torch.int32, device=DEV)
    seq = torch.tensor([0, 1, 2, 0, B, 0], dtype=torch.int32, device=DEV)
    before, q_out = pages.clone(), torch.full((n, 6, hd), 7.0, device=DEV)
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    K.op_paged_append(k, k, k, pages, table, pos, q_out, seq=seq, fault=fault)
    assert int(fault) == 1
    assert bool((q_out[:, 1:5] == 7).all())
    assert torch.equal(q_out[:, [0, 5]], k[:, [0, 5]])
    want = before.clone()
    want[:, :, table[0, 0].long(), 0, 3] = k[:, None, 0]
    want[:, :, table[0, 1].long(), 0, 4] = k[:, None, 5]
    assert torch.equal(pages, want)
    # without a fault word the same rows are left out
    K.op_paged_append(k, k, k, pages, table, pos, q_out, seq=seq)
    assert torch.equal(pages, want)


# --------------------------------------------------------------------------------- attention

def attention64(q, pages, table, lens, scales, scale, hd):
    """(out, bound without the output's rounding) in 64 bits."""
    n, B, dq = q.shape
    Hkv, page = pages.shape[3], pages.shape[4]
    group = dq // hd // Hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    slack = torch.zeros_like(out)
    for b, L in enumerate(lens):
        if L == 0:
            continue
        used = table[b, :-(-L // page)].long()
        for i in range(n):
            kv = []
            for j in (0, 1):
                raw = pages.view(torch.uint8)[i, j][used].view(pages.dtype) \
                    if pages.dtype == F8 else pages[i, j][used]
                x = raw.double().transpose(0, 1).reshape(Hkv, -1, hd)[:, :L]
                kv.append(x if scales is None else x * scales[i, j].double()[:, None, None])
            k, v = kv
            qq = q[i, b].double().view(Hkv, group, hd)
            s = torch.matmul(qq, k.transpose(1, 2).contiguous()) * scale
            ds = (hd + 2) * 2.0 ** -24 * abs(scale) * \
                torch.matmul(qq.abs(), k.abs().transpose(1, 2).contiguous())
            p = torch.softmax(s, -1)
            far = (s.amax(-1, keepdim=True) - s) * 2.0 ** -23
            D = (ds + torch.where(p > 2.0 ** -60, far, 0.0)).amax(-1, keepdim=True)
            out[i, b] = torch.matmul(p, v).flatten()
            slack[i, b] = ((2 * D + 2.0 ** -16 + 2.0 ** -22 + 2 * L * 2.0 ** -24) *
                           torch.matmul(p, v.abs())).flatten()
    return out, slack


ATTENTIONS = [  # n, H, Hkv, hd, dtype, cache dtype, page
    (1, 1, 1, 32, torch.float32, None, 1),
    (2, 4, 4, 64, torch.float32, None, 16),
    (2, 6, 2, 128, torch.float32, None, 33),
    (1, 4, 4, 32, torch.bfloat16, None, 16),
    (2, 4, 2, 64, torch.bfloat16, None, 7),
    (3, 3, 1, 128, torch.bfloat16, None, 64),
    (2, 16, 16, 128, torch.float16, None, 16),
    (1, 32, 1, 64, torch.float16, None, 48),
    (2, 20, 1, 128, torch.float16, None, 128),
    (1, 40, 2, 32, torch.float16, None, 200),
    (2, 4, 4, 128, torch.bfloat16, F8, 16),
    (1, 16, 1, 64, torch.bfloat16, F8, 5),
    (1, 32, 2, 128, torch.float16, F8, 128),
    (2, 6, 6, 32, torch.float16, F8, 32),
]
LENS = {"one": [1], "empty": [0], "zeros": [0, 5, 0, 0], "tile": [31, 32, 33, 64, 65, 128, 129],
        "ragged": [700, 1, 0, 1533, 256, 17], "long": [5003]}


@pytest.mark.parametrize("lens", LENS.values(), ids=LENS.keys())
@pytest.mark.parametrize("case", ATTENTIONS, ids=[str(k) for k in range(len(ATTENTIONS))])
def test_attention(case, lens):
    n, H, Hkv, hd, dtype, cdt, page = case
    cdt = cdt or dtype
    say(f"[paged attention] {case} lens={lens}")
    g = gen(sum(lens) + H)
    pages, table = make_cache(n, Hkv, hd, page, lens, cdt, g, width=3)
    raw = torch.uint8 if cdt == F8 else torch.int16 if cdt != torch.float32 else torch.int32
    # places that no sequence reads hold NaN
    need = torch.tensor([-(-v // page) for v in lens])
    there = torch.zeros(pages.shape[2], page, dtype=torch.bool)
    for b, v in enumerate(lens):
        for j in range(int(need[b])):
            there[table[b, j].item(), :min(page, v - j * page)] = True
    nan = torch.full((1,), math.nan, dtype=torch.float32).to(cdt).view(raw).to(DEV)
    bits = pages.view(raw)
    bits.copy_(torch.where(there.to(DEV)[None, None, :, None, :, None], bits, nan))
    scales = (0.02 + 0.02 * torch.rand((n, 2, Hkv), generator=g)).to(DEV) if cdt == F8 else None
    q = normal((n, len(lens), H * hd + 32), dtype, g, 2.0)[..., :H * hd]
    out = torch.full((n, len(lens), H * hd), 7.0, dtype=dtype, device=DEV)
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for max_len in {max(lens), min(max(lens) + 300, table.shape[1] * page)}:
        out.fill_(7.0)
        K.op_paged_attention(q, pages, table, lens_d, max_len, out, scales=scales, fault=fault)
        torch.cuda.synchronize()
        assert int(fault) == 0
        ref, slack = attention64(q, pages, table, lens, scales, hd ** -0.5, hd)
        near(out, ref, slack, f"max_len {max_len}")
        assert all(bool((out[:, b] == 0).all()) for b, v in enumerate(lens) if v == 0)
        again = torch.empty_like(out)
        K.op_paged_attention(q, pages, table, lens_d, max_len, again, scales=scales)
        assert torch.equal(again, out)


def test_attention_takes_a_scale_and_a_workspace():
    g = gen(3)
    lens = [300, 77]
    pages, table = make_cache(2, 2, 64, 16, lens, torch.float16, g)
    q = normal((2, 2, 256), torch.float16, g)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    need = K.paged_attention_work_floats(pages, table, 4, 300)
    work = torch.full((max(need, 4),), math.nan, device=DEV)
    out = K.op_paged_attention(q, pages, table, lens_d, 300, scale=0.31, work=work)
    ref, slack = attention64(q, pages, table, lens, None, 0.31, 64)
    near(out, ref, slack, "scale")


def test_attention_of_extreme_scores():
    # the smallest and largest finite queries, keys of -inf: weights of 0 and 1, no NaN
    hd, page = 64, 16
    g = gen(4)
    pages, table = make_cache(1, 1, hd, page, [50], torch.bfloat16, g)
    lens_d = torch.tensor([50], dtype=torch.int32, device=DEV)
    flat = pages[0, 0]                                   # [pages, heads, page, hd]
    rows = [(int(table[0, k // page]), k % page) for k in range(50)]
    q = torch.zeros((1, 1, hd), dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1.0
    for k, (pg, at) in enumerate(rows):
        flat[pg, 0, at, 0] = -math.inf if k < 33 else -3.0e38 if k < 49 else 5.0
    out = K.op_paged_attention(q, pages, table, lens_d, 50)
    assert torch.equal(out[0, 0], pages[0, 1, rows[49][0], 0, rows[49][1]])
    flat[rows[49][0], 0, rows[49][1], 0] = -math.inf
    out = K.op_paged_attention(q, pages, table, lens_d, 50)
    v = torch.stack([pages[0, 1, pg, 0, at] for pg, at in rows[33:49]]).double().mean(0)
    near(out[0, 0], v, v.abs() * 2.0 ** -16 + 2.0 ** -16, "lowest values")


def test_attention_marks_bad_rows():
    lens = [40, 40, 40, 40, 40]
    g = gen(6)
    pages, table = make_cache(2, 2, 32, 8, lens, torch.float16, g)
    q = normal((2, 5, 128), torch.float16, g)
    good = K.op_paged_attention(q, pages, table, torch.tensor(lens, dtype=torch.int32,
                                                              device=DEV), 40)
    table[1, 3] = pages.shape[2]
    table[3, 0] = -1
    lens_d = torch.tensor([40, 40, 41, 40, -1], dtype=torch.int32, device=DEV)
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = K.op_paged_attention(q, pages, table, lens_d, 40, fault=fault)
    assert int(fault) == 1
    assert bool(out[:, 1:].isnan().all()) and torch.equal(out[:, 0], good[:, 0])
    # a page that the length does not reach may be anything
    lens_d[1:] = torch.tensor([24, 0, 0, 8], dtype=torch.int32)
    fault.zero_()
    out = K.op_paged_attention(q, pages, table, lens_d, 40, fault=fault)
    assert int(fault) == 0 and bool(out.isfinite().all())


def test_attention_of_256_sequences():
    """More units than waves, and as many sequences as a call takes: runs that end in the middle
    of units, rows without keys in between, a row length out of range."""
    n, H, Hkv, hd, page, B = 3, 12, 6, 64, 24, 256
    g = gen(30)
    lens = [0 if b % 7 == 3 else (37 * b) % 300 for b in range(B)]
    lens[100], lens[255] = 2500, 1
    pages, table = make_cache(n, Hkv, hd, page, lens, torch.bfloat16, g)
    q = normal((B, n, H * hd), torch.bfloat16, g).transpose(0, 1)       # sub-layers behind rows
    out = torch.empty((B, n, H * hd), dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    lens_d[17] = 2501
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    K.op_paged_attention(q, pages, table, lens_d, 2500, out, fault=fault)
    assert int(fault) == 1
    lens[17] = 0
    ref, slack = attention64(q, pages, table, lens, None, 0.125, hd)
    assert bool(out[:, 17].isnan().all())
    keep = torch.arange(B, device=DEV) != 17
    near(out[:, keep], ref[:, keep], slack[:, keep], "256")


def test_a_table_of_wider_rows_and_a_cache_past_32_bit_offsets():
    """Pages at the far end of a cache of 6.4 GB (2^31.7 elements a sub-layer), named by the left
    part of a wider table: append there, attend there, and nothing else is touched."""
    n, H, hd, page, B = 2, 2, 128, 64, 3
    total = 24600
    pages = torch.empty((n, 2, total, H, page, hd), dtype=torch.float16, device=DEV)
    wide = torch.full((B, 40), -1, dtype=torch.int32, device=DEV)
    table = wide[:, :5]
    far = torch.arange(total - 15, total, dtype=torch.int32, device=DEV).flip(0).view(B, 5)
    table.copy_(far)
    g = gen(31)
    lens = [300, 1, 129]
    T = sum(lens)
    d = H * hd
    x = normal((n, T, 3 * d), torch.float16, g)
    seq = torch.repeat_interleave(torch.arange(B), torch.tensor(lens)).to(torch.int32).to(DEV)
    pos = torch.cat([torch.arange(v, dtype=torch.int32) for v in lens]).to(DEV)
    low = pages[:, :, :8].clone()
    fault = torch.zeros(1, dtype=torch.int32, device=DEV)
    K.op_paged_append(x[..., :d], x[..., d:2 * d], x[..., 2 * d:], pages, table, pos, seq=seq,
                      fault=fault)
    new = normal((n, B, d), torch.float16, g)
    out = K.op_paged_attention(new, pages, table, torch.tensor(lens, dtype=torch.int32,
                                                               device=DEV), 300, fault=fault)
    assert int(fault) == 0
    assert torch.equal(pages[:, :, :8].view(torch.int16), low.view(torch.int16))
    at = 0
    for b, L in enumerate(lens):
        rows = pages[:, :, table[b].long()].transpose(2, 3).reshape(n, 2, H, -1, hd)[:, :, :, :L]
        for j in (0, 1):
            want = x[:, at:at + L, (1 + j) * d:(2 + j) * d].unflatten(-1, (H, hd)).transpose(1, 2)
            assert torch.equal(rows[:, j], want)
        at += L
    small, ids = pages[:, :, total - 15:].contiguous(), (table - (total - 15)).contiguous()
    ref, slack = attention64(new, small, ids, lens, None, hd ** -0.5, hd)
    near(out, ref, slack, "far pages")


def test_sequences_share_pages():
    g = gen(8)
    pages, table = make_cache(1, 2, 64, 16, [100], torch.bfloat16, g)
    table = table.expand(3, -1).contiguous()
    q = normal((1, 1, 256), torch.bfloat16, g).expand(1, 3, 256).contiguous()
    lens_d = torch.tensor([100, 100, 60], dtype=torch.int32, device=DEV)
    out = K.op_paged_attention(q, pages, table, lens_d, 100)
    ref, slack = attention64(q, pages, table, [100, 100, 60], None, 0.125, 64)
    near(out, ref, slack, "shared")


# ------------------------------------------------------------------- the operators together

@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_prompt_then_steps_equal_attention_of_the_whole(dtype):
    """A prompt through append and kraken_op_attention, then single tokens through append and
    paged attention: every token's output is the row that causal attention over the whole
    sequence (rotated in 64 bits) gives it."""
    n, H, Hkv, hd, page, steps = 2, 4, 2, 64, 16, 5
    prompts = [37, 64, 3]
    g = gen(12)
    full = [p + steps for p in prompts]
    pages, table = make_cache(n, Hkv, hd, page, full, dtype, g)
    dq, dkv = H * hd, Hkv * hd
    xs = [normal((n, L, dq + 2 * dkv), dtype, g) for L in full]
    freq = 10000.0 ** (-torch.arange(hd // 2, dtype=torch.float64) * 2 / hd)
    cu = K.cu_from_lens(prompts)
    T = cu[-1]
    x = torch.cat([a[:, :p] for a, p in zip(xs, prompts)], 1).contiguous()
    pos = torch.cat([torch.arange(p, dtype=torch.int32) for p in prompts]).to(DEV)
    seq = torch.repeat_interleave(torch.arange(3), torch.tensor(prompts)).to(torch.int32).to(DEV)
    qk = torch.empty((n, T, dq + dkv), dtype=dtype, device=DEV)
    K.op_paged_append(x[..., :dq], x[..., dq:dq + dkv], x[..., dq + dkv:], pages, table, pos,
                      qk[..., :dq], seq=seq, k_out=qk[..., dq:], inv_freq=freq)
    vt = torch.zeros((n, dkv, K.vt_ld(T)), dtype=dtype, device=DEV)
    vt[..., :T] = x[..., dq + dkv:].transpose(1, 2)
    rows = torch.empty((n, T, dq), dtype=dtype, device=DEV)
    K.op_attention(qk, vt, rows, n, dq, H, cu, n_kv_heads=Hkv)
    got = [[rows[:, cu[b]:cu[b + 1]]] for b in range(3)]
    work = torch.empty(K.paged_attention_work_floats(pages, table, H, max(full)), device=DEV)
    for s in range(steps):
        new = torch.stack([a[:, p + s] for a, p in zip(xs, prompts)], 1)
        at = torch.tensor([p + s for p in prompts], dtype=torch.int32, device=DEV)
        q = K.op_paged_append(new[..., :dq], new[..., dq:dq + dkv], new[..., dq + dkv:], pages,
                              table, at, inv_freq=freq)
        o = K.op_paged_attention(q, pages, table, at + 1, max(full), work=work)
        for b in range(3):
            got[b].append(o[:, b:b + 1])
    u = HALF_STEP[dtype]
    for b, L in enumerate(full):
        p_ = torch.arange(L, device=DEV)
        q64, qm = rotate64(xs[b][..., :dq], p_, freq, hd, False, hd)
        k64, km = rotate64(xs[b][..., dq:dq + dkv], p_, freq, hd, False, hd)
        q64, k64 = (t.unflatten(-1, (-1, hd)).transpose(1, 2) for t in (q64, k64))
        v64 = xs[b][..., dq + dkv:].double().unflatten(-1, (-1, hd)).transpose(1, 2)
        k64, v64 = (t.repeat_interleave(H // Hkv, 1) for t in (k64, v64))
        s = torch.matmul(q64, k64.transpose(-1, -2).contiguous()) / 8
        s = s.masked_fill(torch.ones(L, L, device=DEV).triu(1).bool(), -math.inf)
        p = torch.softmax(s, -1)
        ref = torch.matmul(p, v64).transpose(1, 2).flatten(-2)
        # rotated queries and keys are rounded to the type (u each): a score moves by
        # 2.1 u scale sum |q k|; the prompt's kernel rounds its weights to 16 bits (u)
        D = 2.1 * u * torch.matmul(q64.abs(), k64.abs().transpose(-1, -2).contiguous()) / 8
        D = torch.where(p > 0, D, 0.0).amax(-1, keepdim=True)
        slack = (2 * D + u + 2.0 ** -12) * torch.matmul(p, v64.abs())
        near(torch.cat(got[b], 1), ref, slack.transpose(1, 2).flatten(-2), f"sequence {b}")


def test_captured_steps_follow_positions_lengths_and_pages():
    """One captured append + attention step, replayed over a growing conversation: positions,
    lengths and the table are read at every replay."""
    n, H, hd, page, B = 2, 4, 64, 8, 3
    g = gen(15)
    pages, table = make_cache(n, H, hd, page, [40] * B, torch.float16, g)
    d = H * hd
    steps = [normal((n, B, 3 * d), torch.float16, g) for _ in range(4)]
    freq = 10000.0 ** (-torch.arange(hd // 2, dtype=torch.float64) * 2 / hd)
    x, q, out = steps[0].clone(), torch.empty((n, B, d), dtype=torch.float16, device=DEV), \
        torch.empty((n, B, d), dtype=torch.float16, device=DEV)
    pos = torch.tensor([17, 0, -1], dtype=torch.int32, device=DEV)
    lens = pos + 1
    work = torch.empty(K.paged_attention_work_floats(pages, table, H, 40), device=DEV)

    def step(cache, q_out, o, w):
        K.op_paged_append(x[..., :d], x[..., d:2 * d], x[..., 2 * d:], cache, table, pos, q_out,
                          inv_freq=freq)
        K.op_paged_attention(q_out, cache, table, lens, 40, o, work=w)

    eager = pages.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(pages, q, out, work)
    q.zero_()
    for r, new in enumerate(steps):
        x.copy_(new)
        if r == 2:                                   # a sequence gets other pages
            table[1] = table[1].flip(0)
        want_q, want = torch.zeros_like(q), torch.empty_like(out)
        step(eager, want_q, want, None)
        torch.cuda.synchronize()
        out.fill_(7.0)
        work.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(q[:, :2], want_q[:, :2]), r
        assert torch.equal(pages, eager), r
        pos[:2] += 1
        lens[:2] += 1
    assert bool((out[:, 2] == 0).all())


def test_two_streams_at_one_time():
    """Calls on two streams, each with a workspace of its own, and outputs that the binding
    allocates for the stream they are written on."""
    g = gen(21)
    lens = [3000, 11, 900]
    sets = []
    for _ in range(2):
        pages, table = make_cache(2, 4, 64, 16, lens, torch.bfloat16, g)
        q = normal((2, 3, 512), torch.bfloat16, g)
        sets.append((q, pages, table))
    lens_d = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = [K.op_paged_attention(*s, lens_d, 3000) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [K.op_paged_attention(*s, lens_d, 3000, stream=st) for s, st in zip(sets, streams)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
