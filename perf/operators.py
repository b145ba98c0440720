"""The serving operators over a paged key/value cache, as cases that can be timed and compared.

One serving step of a Kraken layer's attention over pages, and the scoring of what it answers:

* ``append``: the new tokens' queries and keys are rotated by their positions (fp32, the angle in
  64 bits), and keys and values go to their places in a paged cache, as they are or in 8 bits with
  one scale per sub-layer and head;
* ``attention``: one new token per sequence attends over the pages of its sequence;
* ``logprobs``: log probabilities of given tokens, the entropy of every row and its most likely
  tokens, from rows of logits.

Each has a plain form in elementary torch operations (``own`` false) and the call a user makes of
the framework (``own`` true).  A paged cache holds ``[n_sub][2 (K, V)][num_pages][kv_heads]
[page_size][head_dim]``; row b of ``table`` lists the pages of sequence b in order.
"""

import math

import torch

own = False

DEVICE = "cuda"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "e4m3": torch.float8_e4m3fn}
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------ cases

def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def append(starts, news, n, heads, kv_heads, hd, dtype, page, cache="", rot=0, pairs="halves",
           keys_out=False, **more):
    """news[b] new tokens of sequence b behind the starts[b] it holds; a start of -1 is a padding
    row.  rot: rotated dimensions of a head (0: all).  keys_out: the rotated keys are wanted too,
    as rows for the attention of a prompt."""
    return dict(op="append", starts=_text(starts), news=_text(news), n=n, heads=heads,
                kv_heads=kv_heads, hd=hd, dtype=dtype, cache=cache or dtype, page=page,
                rot=rot or hd, pairs=pairs, keys_out=keys_out, **more)


def attention(lens, n, heads, kv_heads, hd, dtype, page, cache="", **more):
    """lens[b]: keys of sequence b, its new token's own among them (0: a padding row)."""
    return dict(op="attention", lens=_text(lens), n=n, heads=heads, kv_heads=kv_heads, hd=hd,
                dtype=dtype, cache=cache or dtype, page=page, **more)


def logprobs(rows, vocab, dtype, top, pad=0, **more):
    """rows of vocab logits, pad unused columns behind each."""
    return dict(op="logprobs", rows=rows, vocab=vocab, dtype=dtype, top=top, pad=pad, **more)


def listed():
    return [
        # one conversation's next token on the benchmark's layer: bound by one launch
        append([777], [1], 8, 16, 16, 128, "bf16", 16, name="append_d2048_b1"),
        # a serving batch's next tokens, four key/value heads, some rows of the batch unused
        append([-1 if b % 16 == 15 else 37 + (53 * b) % 900 for b in range(128)], [1] * 128, 4, 16,
               4, 64, "f16", 16, name="append_d1024_gqa4_b128"),
        # the benchmark's prompt of 8192 tokens entering the cache
        append([0], [8192], 8, 16, 16, 128, "f16", 64, keys_out=True, name="append_d2048_s8192"),
        # eight ragged prompts into a cache of 8 bits: neighbouring pairs, half of a head rotated
        append([0] * 8, [2755, 1653, 3903, 817, 2210, 3377, 512, 2001], 4, 20, 20, 64, "bf16", 48,
               cache="e4m3", rot=32, pairs="neighbours", keys_out=True,
               name="append_d1280_ragged8_e4m3"),
        # a small model's step over one short conversation, fp32: bound by launches
        attention([65], 2, 4, 4, 32, "f32", 16, name="attention_f32_d128_len65"),
        # one long conversation on the benchmark's layer
        attention([8192], 8, 16, 16, 128, "f16", 16, name="attention_d2048_b1_len8192"),
        # eight conversations of different lengths, four key/value heads
        attention([8001, 514, 4098, 2047, 7164, 1201, 5556, 3073], 8, 16, 4, 128, "bf16", 64,
                  name="attention_gqa4_d2048_b8"),
        # a large serving batch of short conversations, some rows of the batch unused
        attention([0 if b % 16 == 15 else 38 + (53 * b) % 900 for b in range(128)], 4, 16, 16, 64,
                  "bf16", 32, name="attention_d1024_b128"),
        # long documents in a cache of 8 bits, two key/value heads of 16 queries each
        attention([32768 - 1777 * b for b in range(16)], 1, 32, 2, 128, "f16", 128, cache="e4m3",
                  name="attention_gqa2_d4096_b16_e4m3"),
        # the next token of one conversation: its log probability and five alternatives
        logprobs(1, 51200, "f32", 5, name="logprobs_b1"),
        # a batch's next tokens from 16-bit logits of an odd vocabulary, twenty alternatives
        logprobs(61, 50257, "bf16", 20, pad=47, name="logprobs_b61_bf16"),
        # every token of a prompt scored: perplexity and the likeliest token of each position
        logprobs(2048, 51200, "f32", 1, name="logprobs_s2048"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _layer(rng):
    """Sub-layers, heads, key/value heads, head size, type, the cache's type and page size."""
    hd = rng.choice([32, 64, 64, 128, 128])
    n = rng.choice([1, 2, 4, 8])
    kv_heads = _log_int(rng, 1, 20)
    group = rng.choice([1, 1, 2, 3, 4, 8, 16, 20])
    while kv_heads * group > 40:
        group = max(1, group // 2)
    dtype = rng.choice(["f16", "bf16", "f32"])
    cache = "e4m3" if dtype != "f32" and rng.random() < 0.3 else dtype
    page = rng.choice([1, 8, 16, 16, 32, 48, 64, 128, 200, 256])
    return n, kv_heads * group, kv_heads, hd, dtype, page, cache


def draw(rng):
    """One more case of these ranges, no larger than the largest listed one of its operator."""
    op = rng.choice(["append", "attention", "logprobs"])
    limit = max(work(c)["bytes"] for c in listed() if c["op"] == op)
    while True:
        if op == "logprobs":
            vocab = _log_int(rng, 1000, 160000)
            c = logprobs(_log_int(rng, 1, 4096), vocab, rng.choice(["f32", "bf16", "f16"]),
                         rng.choice([0, 1, 5, 20, 64]), pad=rng.choice([0, 0, 1, -vocab % 64]))
        elif op == "attention":
            n, heads, kv_heads, hd, dtype, page, cache = _layer(rng)
            top = _log_int(rng, 1, 65536)
            seqs = _log_int(rng, 1, 256)
            c = attention([rng.choice([0, top, rng.randint(0, top), rng.randint(0, top)])
                           for _ in range(seqs - 1)] + [top], n, heads, kv_heads, hd, dtype, page,
                          cache=cache)
            if max(_ints(c["lens"])) * seqs * n * 2 * kv_heads * hd > 1 << 30:
                continue        # (the plain form gathers every sequence at the longest's length)
        else:
            n, heads, kv_heads, hd, dtype, page, cache = _layer(rng)
            if rng.random() < 0.5:
                top, seqs = _log_int(rng, 1, 8192), _log_int(rng, 1, 256)
                starts = [rng.choice([-1, top, rng.randint(0, top), rng.randint(0, top)])
                          for _ in range(seqs - 1)] + [top]
                news = [1] * seqs
            else:
                seqs = _log_int(rng, 1, 16)
                starts = [rng.choice([0, 0, rng.randint(0, 4096)]) for _ in range(seqs)]
                news = [_log_int(rng, 1, 8192) for _ in range(seqs)]
            c = append(starts, news, n, heads, kv_heads, hd, dtype, page, cache=cache,
                       rot=rng.choice([hd, hd, hd // 2, hd - 8]),
                       pairs=rng.choice(["halves", "neighbours"]),
                       keys_out=rng.choice([True, False]))
            if sum(a + b for a, b in zip(starts, news)) * n * 2 * kv_heads * hd > 1 << 29:
                continue
        if work(c)["bytes"] <= limit:
            return c


def work(case):
    if case["op"] == "logprobs":
        e = TORCH[case["dtype"]].itemsize
        rows, vocab, top = case["rows"], case["vocab"], case["top"]
        # the largest, the sums of exp and of exp times the logit: about five operations each
        return {"bytes": rows * (vocab * e + 12 + 8 * top), "flops": 5.0 * rows * vocab}
    n, hd, e = case["n"], case["hd"], TORCH[case["dtype"]].itemsize
    ec = TORCH[case["cache"]].itemsize
    dq, dkv = case["heads"] * hd, case["kv_heads"] * hd
    if case["op"] == "append":
        rows = sum(b for a, b in zip(_ints(case["starts"]), _ints(case["news"])) if a >= 0)
        moved = 2 * dq * e + 2 * dkv * (e + ec) + (dkv * e if case["keys_out"] else 0)
        turned = (dq + dkv) * case["rot"] / hd
        return {"bytes": rows * (n * moved + 8), "flops": 3.0 * rows * n * turned}
    lens = _ints(case["lens"])
    pages = sum(-(-v // case["page"]) for v in lens)
    return {"bytes": n * (sum(lens) * 2 * dkv * ec + 2 * len(lens) * dq * e) + 4 * pages,
            "flops": 4.0 * n * dq * sum(lens)}


# ------------------------------------------------------------------------------------ inputs

def _table(lens, page, g):
    """Pages of a cache that holds lens[b] tokens of sequence b, in no order, with some unused
    ones: (number of pages, table [B][pages of the longest], -1 behind a sequence's last)."""
    need = [-(-max(v, 0) // page) for v in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    width = max(1, max(need))
    counts = torch.tensor(need, device=DEVICE)
    at = torch.arange(width, device=DEVICE)[None]
    first = (counts.cumsum(0) - counts)[:, None]
    return pages, torch.where(at < counts[:, None], order[(first + at).clamp(max=pages - 1)], -1)


def _normal(shape, dtype, g):
    if dtype == torch.float8_e4m3fn:      # keys and values that fill the type's range
        return (torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float16) * 40).to(dtype)
    return torch.randn(shape, generator=g, device=DEVICE, dtype=dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    s = dict(case)
    dtype = TORCH[case["dtype"]]
    if case["op"] == "logprobs":
        rows, vocab = case["rows"], case["vocab"]
        # logits of a trained model: wide, an offset per row, a few tokens far above the others
        x = torch.randn((rows, vocab + case["pad"]), generator=g, device=DEVICE) * 2.5
        peaks = torch.randint(vocab, (rows, 24), generator=g, device=DEVICE)
        x.scatter_add_(1, peaks, 8 * torch.rand((rows, 24), generator=g, device=DEVICE))
        x += 4 * torch.randn((rows, 1), generator=g, device=DEVICE)
        s["logits"] = x.to(dtype)[:, :vocab]
        likely = torch.rand((rows,), generator=g, device=DEVICE) < 0.7
        other = torch.randint(vocab, (rows,), generator=g, device=DEVICE)
        s["tokens"] = torch.where(likely, peaks[:, 0], other).to(torch.int32)
        return s
    n, hd = case["n"], case["hd"]
    dq, dkv = case["heads"] * hd, case["kv_heads"] * hd
    cache = TORCH[case["cache"]]
    if case["op"] == "append":
        starts, news = _ints(case["starts"]), _ints(case["news"])
        lens = [a + b if a >= 0 else 0 for a, b in zip(starts, news)]
        T = sum(news)
        counts = torch.tensor(news, device=DEVICE)
        begin = torch.tensor(starts, device=DEVICE)
        seq = torch.repeat_interleave(torch.arange(len(news), device=DEVICE), counts)
        pos = torch.arange(T, device=DEVICE) - (counts.cumsum(0) - counts)[seq] + begin[seq]
        s["seq"] = seq.to(torch.int32)
        s["pos"] = torch.where(begin[seq] >= 0, pos, -1).to(torch.int32)
        qkv = _normal((n, T, dq + 2 * dkv), dtype, g)     # one projection's columns Q | K | V
        s["q"], s["k"], s["v"] = qkv[..., :dq], qkv[..., dq:dq + dkv], qkv[..., dq + dkv:]
        s["q_out"] = torch.zeros((n, T, dq), dtype=dtype, device=DEVICE)
        s["k_out"] = torch.zeros((n, T, dkv), dtype=dtype, device=DEVICE) \
            if case["keys_out"] else None
        i = torch.arange(case["rot"] // 2, dtype=torch.float64)
        s["inv_freq"] = 10000.0 ** (-2 * i / case["rot"])     # on the host, radians per position
    else:
        lens = _ints(case["lens"])
        s["q"] = _normal((n, len(lens), dq), dtype, g)
        s["out"] = torch.empty_like(s["q"])
        s["lens"], s["max_len"] = torch.tensor(lens, dtype=torch.int32, device=DEVICE), max(lens)
    pages, s["table"] = _table(lens, case["page"], g)
    s["pages"] = _normal((n, 2, pages, case["kv_heads"], case["page"], hd), cache, g)
    # scales of the benchmark's rows: values ~ N(0, 1) up to about 6 onto the type's range
    s["scales"] = (0.013 + 0.004 * torch.rand((n, 2, case["kv_heads"]), generator=g, device=DEVICE)
                   if case["cache"] == "e4m3" else None)
    return s


# ------------------------------------------------------------------------------------ plain forms

def _turn(x, cos, sin, hd, rot, pairs):
    """x [n][T][heads * hd] in fp32 with the first rot dimensions of each head rotated."""
    x = x.float().unflatten(-1, (-1, hd))
    cos, sin = cos[None, :, None], sin[None, :, None]
    if pairs == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(s):
    hd, page, rot = s["hd"], s["page"], s["rot"]
    rows = torch.nonzero(s["pos"] >= 0)[:, 0]
    pos = s["pos"][rows].long()
    angle = pos[:, None].double() * s["inv_freq"].to(DEVICE)
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _turn(s["q"][:, rows], cos, sin, hd, rot, s["pairs"])
    k = _turn(s["k"][:, rows], cos, sin, hd, rot, s["pairs"])
    v = s["v"][:, rows].float().unflatten(-1, (-1, hd))
    s["q_out"][:, rows] = q.flatten(-2).to(s["q_out"].dtype)
    if s["k_out"] is not None:
        s["k_out"][:, rows] = k.flatten(-2).to(s["k_out"].dtype)
    pages = s["pages"]
    kv = torch.stack([k, v], 1)                               # [n][2][rows][kv_heads][hd]
    if s["scales"] is not None:
        kv = (kv / s["scales"][:, :, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
    kv = kv.to(pages.dtype)
    place = s["table"][s["seq"][rows].long(), pos // page].long()
    bits = pages.view(torch.uint8) if s["scales"] is not None else pages
    values = kv.view(torch.uint8) if s["scales"] is not None else kv
    bits[:, :, place, :, pos % page] = values.permute(2, 0, 1, 3, 4)
    return {"q": s["q_out"], "k": s["k_out"], "pages": pages}


def _plain_attention(s):
    n, hd, kv_heads, group = s["n"], s["hd"], s["kv_heads"], s["heads"] // s["kv_heads"]
    B, width = s["table"].shape
    kv = s["pages"][:, :, s["table"].long().clamp(min=0)]     # [n][2][B][width][heads][page][hd]
    kv = kv.float().permute(0, 1, 2, 4, 3, 5, 6).flatten(4, 5)
    if s["scales"] is not None:
        kv = kv * s["scales"][:, :, None, :, None, None]
    q = s["q"].float().view(n, B, kv_heads, group, hd).transpose(-1, -2).contiguous()
    score = torch.matmul(kv[:, 0], q) / math.sqrt(hd)         # [n][B][kv_heads][keys][group]
    there = torch.arange(score.shape[3], device=DEVICE)[:, None] < s["lens"][:, None, None, None]
    score = torch.where(there, score, -math.inf)
    top = score.amax(3, keepdim=True)
    e = torch.where(there, torch.exp(score - top), 0.0)
    p = (e / e.sum(3, keepdim=True).clamp(min=1e-30)).transpose(-1, -2).contiguous()
    s["out"].copy_(torch.matmul(p, kv[:, 1]).reshape(n, B, -1))
    return s["out"]


def _plain_logprobs(s):
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    t = x - m
    e = torch.exp(t)
    total = e.sum(1)
    log_total = torch.log(total)
    r = {"logprob": t.gather(1, s["tokens"].long()[:, None])[:, 0] - log_total,
         "entropy": log_total - (e * t).sum(1) / total}
    if s["top"]:
        best, ids = torch.sort(t, dim=1, descending=True, stable=True)
        r["top_ids"] = ids[:, :s["top"]].to(torch.int32)
        r["top_logprobs"] = best[:, :s["top"]] - log_total[:, None]
    return r


# ------------------------------------------------------------------------------------ the calls

def _own_append(s):
    from paper_2408_07802_amd import kraken
    kraken.op_paged_append(s["q"], s["k"], s["v"], s["pages"], s["table"], s["pos"], s["q_out"],
                           seq=s["seq"], k_out=s["k_out"], inv_freq=s["inv_freq"],
                           neighbours=s["pairs"] == "neighbours", scales=s["scales"])
    return {"q": s["q_out"], "k": s["k_out"], "pages": s["pages"]}


def _own_attention(s):
    from paper_2408_07802_amd import kraken
    return kraken.op_paged_attention(s["q"], s["pages"], s["table"], s["lens"], s["max_len"],
                                     s["out"], scales=s["scales"])


def _own_logprobs(s):
    from paper_2408_07802_amd import kraken
    r = kraken.op_token_logprobs(s["logits"], s["tokens"], top=s["top"])
    return {k: v for k, v in r._asdict().items() if v is not None}


def run(state):
    if own:
        return {"append": _own_append, "attention": _own_attention,
                "logprobs": _own_logprobs}[state["op"]](state)
    return {"append": _plain_append, "attention": _plain_attention,
            "logprobs": _plain_logprobs}[state["op"]](state)


# ------------------------------------------------------------------------------------ in 64 bits

def _exact_append(s):
    n, hd, page, rot = s["n"], s["hd"], s["page"], s["rot"]
    pos, T = s["pos"].long(), s["pos"].numel()
    live = pos >= 0
    freq = torch.zeros(hd // 2, dtype=torch.float64)
    freq[:rot // 2] = s["inv_freq"]
    # the rotation as a complex factor; pairs that are not rotated have frequency 0
    turn = torch.polar(torch.ones((T, hd // 2), dtype=torch.float64, device=DEVICE),
                       pos[:, None] * freq.to(DEVICE))
    dims = torch.arange(hd, device=DEVICE)
    if s["pairs"] == "halves":
        order = torch.cat([torch.stack([dims[:rot // 2], dims[rot // 2:rot]], 1).flatten(),
                           dims[rot:]])
    else:
        order = dims
    back = torch.argsort(order)

    def rotated(x):
        z = torch.view_as_complex(x.double().view(T, -1, hd)[..., order]
                                  .reshape(T, -1, hd // 2, 2).contiguous())
        return torch.view_as_real(z * turn[:, None]).flatten(-2)[..., back]

    q, k = s["q_out"].double(), None if s["k_out"] is None else s["k_out"].double()
    pages = s["pages"].double()
    place = s["table"].long()[s["seq"].long()[live], pos[live] // page]
    for i in range(n):
        q[i][live] = rotated(s["q"][i])[live].flatten(1)
        keys = rotated(s["k"][i])[live]
        if k is not None:
            k[i][live] = keys.flatten(1)
        for j, x in enumerate((keys, s["v"][i].double().view(T, -1, hd)[live])):
            if s["scales"] is not None:
                x = (x / s["scales"][i, j].double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
            pages[i, j][place, :, pos[live] % page] = x
    return {"q": q, "k": k, "pages": pages}


def _exact_attention(s):
    n, hd, kv_heads, group = s["n"], s["hd"], s["kv_heads"], s["heads"] // s["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, length in enumerate(_ints(s["lens"] if isinstance(s["lens"], str) else
                                     _text(s["lens"].tolist()))):
        if length == 0:
            continue
        used = s["table"][b, :-(-length // s["page"])].long()
        for i in range(n):
            k, v = (s["pages"][i, j][used].double().transpose(0, 1).reshape(kv_heads, -1, hd)
                    [:, :length] * (1.0 if s["scales"] is None
                                    else s["scales"][i, j].double()[:, None, None])
                    for j in (0, 1))
            q = s["q"][i, b].double().view(kv_heads, group, hd)
            p = torch.softmax(torch.bmm(q, k.transpose(1, 2).contiguous()) * hd ** -0.5, dim=-1)
            out[i, b] = torch.bmm(p, v).flatten()
    return out


def _exact_logprobs(s):
    parts = []
    for first in range(0, s["rows"], 256):
        logp = torch.log_softmax(s["logits"][first:first + 256].double(), dim=1)
        tokens = s["tokens"][first:first + 256].long()
        part = [logp[torch.arange(len(tokens), device=DEVICE), tokens],
                -(logp.exp() * logp).sum(1)]
        if s["top"]:
            part.append(torch.topk(logp, s["top"], dim=1).values)
        parts.append(part)
    joined = [torch.cat(p) for p in zip(*parts)]
    r = {"logprob": joined[0], "entropy": joined[1]}
    if s["top"]:
        r["top_ids"], r["top_logprobs"] = None, joined[2]
    return r


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention,
            "logprobs": _exact_logprobs}[case["op"]](s)
