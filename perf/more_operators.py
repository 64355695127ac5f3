"""The operators of a serving step over a cache held in 8 bits, as calls whose
speed is followed: head norms, position rotation and the append that quantises
(``append``), decode and verify attention over that cache (``decode``), attention
of chunks over it (``chunk``), and what stands between the model's logits and the
draw: penalties, biases and grammar masks (``rules``).

With ``own`` false, ``run`` computes an operator in elementary torch operations
in 32 bits (64 where 32 lose what matters); with ``own`` true it makes the call
that a user makes of the package's binding.

The cache holds e4m3 codes and, for each page of 16 tokens and KV head, a power
of two for its keys and one for its values (e8m0): a value is code times power.
A case is a dict of plain values; its lengths are drawn from its ``len_seed``, so
its work is known without a GPU.
"""
import math
import random

import torch

own = False

PAGE = 16
VOCAB = 151936              # the vocabulary of the package's step benchmark
EPS = 1e-6
MAX_SCORES = 2.1e9          # twice the scores of a drawn chunk case: what the largest listed one has
MAX_VALUES = 1.2e9          # keys and values of the largest decode case, about
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
LOWEST, HIGHEST = 27, 227   # the exponent bytes that an append writes: 2^-100 to 2^100


def _seqs(kind, name, batch, heads, q_lo, q_hi, past_lo, past_hi, singles=0, len_seed=0):
    """``batch`` sequences with q_lo..q_hi new tokens behind past_lo..past_hi
    cached ones; the first ``singles`` of them have one new token."""
    q_heads, kv_heads, head_dim = heads
    return dict(name=name, kind=kind, batch=batch, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                q_lo=q_lo, q_hi=q_hi, past_lo=past_lo, past_hi=past_hi, singles=singles, len_seed=len_seed)


def _append(name, batch, heads, q_lo, q_hi, past_lo, past_hi, rot, norm, interleaved, len_seed=0):
    c = _seqs("append", name, batch, heads, q_lo, q_hi, past_lo, past_hi, 0, len_seed)
    c.update(rot=rot, norm=norm, interleaved=interleaved)
    return c


def _rules(name, batch, vocab, dtype, hist_lo, hist_hi, biases, masked, len_seed=0):
    """Rows with hist_lo..hist_hi tokens behind them, and up to ``biases`` biased tokens each."""
    return dict(name=name, kind="rules", batch=batch, vocab=vocab, dtype=dtype, hist_lo=hist_lo, hist_hi=hist_hi,
                biases=biases, masked=masked, len_seed=len_seed)


def listed():
    return [
        # the tail pool's decode step: a handful of tokens, latency only
        _append("append_decode_b8", 8, (32, 8, 128), 1, 1, 500, 3000, 128, False, False, len_seed=1),
        # a prompt's chunk in a model with head norms, starting inside a page
        _append("append_prompt_8k", 2, (32, 8, 128), 4096, 4096, 100, 3000, 128, True, False, len_seed=2),
        # ragged chunks, half of the dimensions rotated, pairs side by side
        _append("append_ragged_b24", 24, (16, 2, 64), 1, 300, 0, 900, 32, False, True, len_seed=3),
        # the last straggler of a rollout step: one sequence, latency only
        _seqs("decode", "decode_b1", 1, (32, 8, 128), 1, 1, 1600, 1600, len_seed=4),
        # the bulk pool at high concurrency
        _seqs("decode", "decode_bulk_b256", 256, (32, 8, 128), 1, 1, 500, 8000, len_seed=5),
        # the tail pool's verify over long contexts
        _seqs("decode", "verify_b8_q4", 8, (32, 8, 128), 4, 4, 16384, 65536, len_seed=6),
        # continuous batching: decoding sequences and two chunks in one launch
        _seqs("chunk", "chunk_mixed_b32", 32, (32, 8, 128), 200, 256, 500, 4000, singles=30, len_seed=7),
        # ragged prompts, eight query heads per KV head
        _seqs("chunk", "chunk_ragged_b16", 16, (32, 4, 128), 1, 1024, 0, 3000, len_seed=8),
        # one long prompt from its first token
        _seqs("chunk", "chunk_prompt_8k", 1, (32, 8, 128), 8192, 8192, 0, 0, len_seed=9),
        # the tail pool: few rows with long histories behind them
        _rules("rules_b8", 8, VOCAB, "float32", 1000, 30000, 0, False, len_seed=10),
        # structured output at high concurrency: grammar masks, requests with their own biases
        _rules("rules_b200", 200, VOCAB, "bfloat16", 100, 8000, 100, True, len_seed=11),
        # an odd vocabulary, whose rows start at any element
        _rules("rules_odd_b48", 48, 50257, "bfloat16", 0, 2000, 20, True, len_seed=12),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    kind = rng.choice(["append", "decode", "decode", "chunk", "chunk", "rules"])
    if kind == "rules":
        c = _rules("", log(1, 200), rng.choice([VOCAB, log(1000, VOCAB), log(1000, VOCAB)]),
                   rng.choice(["float32", "bfloat16"]), 0, 0, rng.choice([0, log(1, 300)]), rng.random() < 0.5,
                   rng.randrange(1 << 30))
        c["hist_hi"] = min(log(1, 30000), 1600000 // c["batch"])
        c["hist_lo"] = rng.choice([0, c["hist_hi"]])
    elif kind == "append":
        heads = rng.choice([(32, 8, 128), (32, 4, 128), (64, 4, 128), (8, 2, 64), (16, 2, 64)])
        batch = log(1, 32)
        q_hi = log(1, (8192 if heads[0] < 64 else 4096) // batch)
        c = _append("", batch, heads, rng.choice([1, q_hi]), q_hi, 0, log(16, 6000) // batch + 1,
                    rng.choice([heads[2], heads[2], heads[2] // 2]), rng.random() < 0.5, rng.random() < 0.3,
                    rng.randrange(1 << 30))
    elif kind == "decode":
        heads = rng.choice([(32, 8, 128)] * 3 + [(16, 4, 128), (32, 4, 128), (64, 4, 128), (8, 2, 64), (16, 2, 64)])
        most = min(16, 64 // (heads[0] // heads[1]))
        q_hi = rng.choice([1, 1, rng.randint(1, most)])
        batch = log(1, 256)
        past = min(log(1, 65536), int(MAX_VALUES / (batch * heads[1] * heads[2])))
        c = _seqs("decode", "", batch, heads, rng.choice([1, q_hi]), q_hi, rng.choice([0, past // 2]), past, 0,
                  rng.randrange(1 << 30))
    else:
        heads = rng.choice([(32, 8, 128)] * 3 + [(16, 4, 128), (32, 4, 128), (64, 4, 128), (8, 2, 64), (16, 2, 64)])
        batch = log(1, 32)
        q_hi = log(1, 6000)
        c = _seqs("chunk", "", batch, heads, rng.choice([1, (q_hi + 1) // 2, q_hi]), q_hi, 0, log(1, 16000),
                  rng.choice([0, 0, batch // 2]), rng.randrange(1 << 30))
        while c["batch"] * heads[0] * c["q_hi"] * (c["q_hi"] + 2 * c["past_hi"]) > MAX_SCORES:
            key = max(("batch", "q_hi", "past_hi"), key=lambda k: c[k] / dict(batch=8, q_hi=600, past_hi=2000)[k])
            c[key] = max(1, c[key] * 3 // 4)
            c["q_lo"] = min(c["q_lo"], c["q_hi"])
            c["singles"] = min(c["singles"], c["batch"] // 2)
    del c["name"]
    return c


# ---- shapes ---------------------------------------------------------------------

def _lens(case):
    """Context length (the new tokens included) and new tokens per sequence."""
    r = random.Random(case["len_seed"])
    ctx, ql = [], []
    for b in range(case["batch"]):
        q = 1 if b < case["singles"] else r.randint(case["q_lo"], case["q_hi"])
        ql.append(q)
        ctx.append(q + r.randint(case["past_lo"], case["past_hi"]))
    return ctx, ql


def _rule_lens(case):
    """Tokens behind each row, how many of them are its prompt, and its biases."""
    r = random.Random(case["len_seed"])
    hist = [r.randint(case["hist_lo"], case["hist_hi"]) for _ in range(case["batch"])]
    return hist, [r.randint(0, n) for n in hist], [r.randint(0, case["biases"]) for _ in hist]


def work(case):
    if case["kind"] == "rules":
        hist, _, biases = _rule_lens(case)
        n = case["batch"] * case["vocab"]
        size = 4 if case["dtype"] == "float32" else 2
        return dict(bytes=2 * size * n + (n // 8 if case["masked"] else 0) + 4 * sum(hist) + 8 * sum(biases),
                    flops=n + 4 * sum(hist))
    ctx, ql = _lens(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["kind"] == "append":
        rows = sum(ql)
        return dict(bytes=rows * (4 * hq + 6 * hkv) * d, flops=rows * (6 * hq + 12 * hkv) * d)
    visible = sum(q * (n - q) + q * (q + 1) // 2 for n, q in zip(ctx, ql))
    pages = sum((n + PAGE - 1) // PAGE for n in ctx)
    return dict(bytes=sum(ctx) * hkv * d * 2 + sum(ql) * hq * d * 4 + pages * (4 + 2 * hkv),
                flops=4 * hq * d * visible)


# ---- inputs ---------------------------------------------------------------------

def _paged(case, gen):
    """A paged cache over a random page permutation: codes of normal values, and
    powers of two around 2^-7, so that the values' size is about 1."""
    ctx, ql = _lens(case)
    hkv, d = case["kv_heads"], case["head_dim"]
    npg = [(n + PAGE - 1) // PAGE for n in ctx]
    total = sum(npg)
    perm = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(max(npg), device="cuda")[None, :]
    counts = torch.tensor(npg, device="cuda")
    first = torch.cumsum(counts, 0) - counts
    table = torch.where(col < counts[:, None], perm[(first[:, None] + col).clamp(max=total - 1)], 0).to(torch.int32)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731

    def codes():
        x = torch.empty(total, hkv, PAGE, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
        return x.mul_(100.0).clamp_(-448.0, 448.0).to(E4M3)

    scales = torch.randint(119, 122, (total, hkv, 2), generator=gen, device="cuda").to(torch.uint8).view(E8M0)
    starts = [0]
    for q in ql:
        starts.append(starts[-1] + q)
    return dict(k_pages=codes(), v_pages=codes(), scales=scales, table=table, ctx=i32(ctx), ql=i32(ql),
                starts=i32(starts), max_q=max(ql), max_ctx=max(ctx))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(kind=case["kind"])
    if case["kind"] == "rules":
        return _prepare_rules(case, gen, s)
    s.update(_paged(case, gen))
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    rows = sum(_lens(case)[1])
    normal = lambda *shape: torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)  # noqa: E731
    s["scale"] = d ** -0.5
    if case["kind"] == "decode":
        s["q"] = normal(case["batch"], s["max_q"], hq, d)
    else:   # views of one fused projection's output
        qkv = normal(rows, hq + 2 * hkv, d)
        s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:])
    s["out"] = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    if case["kind"] == "append":
        rot = case["rot"]
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, device="cuda").double() / rot)).float()
        weight = lambda: (1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(torch.bfloat16)  # noqa: E731
        s["q_norm"], s["k_norm"] = (weight(), weight()) if case["norm"] else (None, None)
        s["interleaved"] = case["interleaved"]
    return s


def _prepare_rules(case, gen, s):
    B, V = case["batch"], case["vocab"]
    hist, prompt, biases = _rule_lens(case)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")  # noqa: E731
    logits = torch.empty(B, V, device="cuda").normal_(generator=gen).mul_(3.0)
    logits[:, V - V // 200:] = -math.inf               # the padding of the vocabulary
    s["logits"] = logits.to(getattr(torch, case["dtype"]))
    s["out"] = torch.empty_like(s["logits"])
    # text: few tokens often, many seldom
    s["tokens"] = (V * uniform(B, max(max(hist), 1)) ** 4).to(torch.int32).clamp_(max=V - 1)
    s["lens"], s["prompt"] = i32(hist), i32(prompt)
    s["repetition"] = 1.0 + 0.3 * uniform(B)
    s["frequency"] = uniform(B) - 0.2
    s["presence"] = uniform(B) - 0.2
    s["bias_starts"] = s["bias_tokens"] = s["bias_values"] = s["allowed"] = None
    if case["biases"]:
        starts = [0]
        for n in biases:
            starts.append(starts[-1] + n)
        s["bias_starts"] = i32(starts)
        s["bias_tokens"] = torch.randint(0, V, (starts[-1],), generator=gen, device="cuda").to(torch.int32)
        s["bias_values"] = 10.0 * uniform(starts[-1]) - 5.0
    if case["masked"]:
        words = (V + 31) // 32
        mask = torch.randint(-2 ** 31, 2 ** 31, (B, words), generator=gen, device="cuda").to(torch.int32)
        few = torch.randint(-2 ** 31, 2 ** 31, (B, words), generator=gen, device="cuda").to(torch.int32)
        pick = torch.arange(B, device="cuda")[:, None] % 3     # half allowed, a quarter, everything
        s["allowed"] = torch.where(pick == 0, mask, torch.where(pick == 1, mask & few, -1))
    return s


def _call(s):
    from paper_2608_22788_amd import binding
    if s["kind"] == "append":
        binding.rope_append_kv8(s["q"], s["k"], s["v"], s["out"], s["k_pages"], s["v_pages"], s["scales"], s["table"],
                                s["ctx"], s["starts"], s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                                interleaved=s["interleaved"])
        return s["out"], s["k_pages"], s["v_pages"], s["scales"]
    if s["kind"] == "rules":
        binding.logit_rules(s["logits"], s["out"], tokens=s["tokens"], lens=s["lens"], prompt_lens=s["prompt"],
                            repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                            bias_starts=s["bias_starts"], bias_tokens=s["bias_tokens"],
                            bias_values=s["bias_values"], allowed=s["allowed"])
        return s["out"]
    # the workspace that a program makes once and hands to every call
    if s["kind"] == "decode":
        if "ws" not in s:
            s["ws"] = binding.new_workspace(binding.decode_kv8_workspace_size(
                binding.shape_of(s["q"], s["k_pages"], s["table"], s["max_ctx"])))
        binding.decode_attn_kv8(s["q"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["ql"],
                                s["out"], s["scale"], workspace=s["ws"], max_ctx_len=s["max_ctx"])
        return s["out"]
    if "ws" not in s:
        s["ws"] = binding.new_workspace(binding.chunk_kv8_workspace_size(
            binding.chunk_shape_of(s["q"], s["k_pages"], s["table"], s["max_q"], s["max_ctx"])))
    binding.chunk_attn_kv8(s["q"], s["k_pages"], s["v_pages"], s["scales"], s["table"], s["ctx"], s["starts"],
                           s["out"], s["scale"], workspace=s["ws"], max_q_len=s["max_q"], max_ctx_len=s["max_ctx"])
    return s["out"]


# ---- one pass -------------------------------------------------------------------

def run(s):
    if own:
        return _call(s)
    return dict(append=_plain_append, decode=_plain_decode, chunk=_plain_chunk, rules=_plain_rules)[s["kind"]](s)


def _power(byte):
    """2^(byte - 127), exactly (bytes 1 .. 254)."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _rows(s):
    """Sequence, row within it and position of every packed row."""
    at = torch.arange(s["q"].shape[0], device="cuda")
    starts = s["starts"].long()
    b = torch.searchsorted(starts[1:], at, right=True)
    i = at - starts[b]
    return b, i, s["ctx"].long()[b] - (starts[1:] - starts[:-1])[b] + i


def _cached(s, name, which, lm):
    """Every sequence's keys or values, [B * Hkv][lm][D] in 32 bits."""
    B, Hkv, D = s["ctx"].numel(), s["k_pages"].shape[1], s["k_pages"].shape[3]
    table = s["table"].long()
    x = s[name][table].float() * _power(s["scales"].view(torch.uint8)[table][..., which])[..., None, None]
    return x.permute(0, 2, 1, 3, 4).reshape(B * Hkv, lm, D)


def _plain_attention(s, q, last):
    """q [B][Qm][Hq][D] in 32 bits, last [B][Qm]: the last key that a row sees."""
    B, Qm, Hq, D = q.shape
    Hkv = s["k_pages"].shape[1]
    G, Lm = Hq // Hkv, s["table"].shape[1] * PAGE
    q = q.view(B, Qm, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B * Hkv, Qm * G, D)
    x = torch.matmul(q, _cached(s, "k_pages", 0, Lm).transpose(1, 2).contiguous()).mul_(s["scale"])
    hidden = torch.arange(Lm, device="cuda") > last[:, :, None]
    x.view(B, Hkv, Qm, G, Lm).masked_fill_(hidden[:, None, :, None], -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    v = _cached(s, "v_pages", 1, Lm)
    v.view(B, Hkv, Lm, D).masked_fill_((torch.arange(Lm, device="cuda") >= s["ctx"][:, None])[:, None, :, None], 0.0)
    o = torch.matmul(x, v) / total.clamp(min=1e-30)
    return o.view(B, Hkv, Qm, G, D).permute(0, 2, 1, 3, 4).reshape(B, Qm, Hq, D)


def _plain_decode(s):
    i = torch.arange(s["max_q"], device="cuda")
    used = i < s["ql"][:, None]
    last = torch.where(used, (s["ctx"] - s["ql"])[:, None] + i, -1)
    o = _plain_attention(s, s["q"].float(), last).to(torch.bfloat16)
    s["out"].copy_(torch.where(used[:, :, None, None], o, s["out"]))
    return s["out"]


def _plain_chunk(s):
    B, (T, Hq, D) = s["ctx"].numel(), s["q"].shape
    b, i, pos = _rows(s)
    q = torch.zeros(B, s["max_q"], Hq, D, device="cuda")
    q[b, i] = s["q"].float()
    last = torch.full((B, s["max_q"]), -1, device="cuda")
    last[b, i] = pos
    return _plain_attention(s, q, last)[b, i].to(torch.bfloat16)


def _plain_append(s):
    b, _, pos = _rows(s)
    angle = pos.double()[:, None, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()
        half = cos.shape[-1]
        a, c = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if s["interleaved"] else (x[..., :half],
                                                                                     x[..., half:2 * half])
        a, c = a * cos - c * sin, c * cos + a * sin
        y = torch.stack((a, c), -1).flatten(-2) if s["interleaved"] else torch.cat((a, c), -1)
        return torch.cat((y, x[..., 2 * half:]), -1)

    s["out"].copy_(turned(s["q"], s["q_norm"]).to(torch.bfloat16))
    page, slot = s["table"].long()[b, pos // PAGE], pos % PAGE
    # each sequence's first page, and the tokens that it holds already
    past = (s["ctx"] - s["ql"]).long()
    head = s["table"].long().gather(1, (past // PAGE)[:, None])[:, 0]
    held = torch.arange(PAGE, device="cuda") < (past % PAGE)[:, None]
    scales = s["scales"].view(torch.uint8)
    for which, (pages, x) in enumerate(((s["k_pages"], turned(s["k"], s["k_norm"])), (s["v_pages"], s["v"].float()))):
        size = x.abs().amax(-1)
        most = torch.zeros(pages.shape[:2], device="cuda").index_reduce_(0, page, size, "amax")
        m, e = torch.frexp(most)             # most <= 448 * 2^k, 448 = 0.875 * 2^9
        byte = torch.where(most > 0, e - torch.where(m <= 0.875, 9, 8) + 127, LOWEST).clamp(LOWEST, HIGHEST)
        old = scales[head][..., which].int()
        byte[head] = torch.where(held.any(1)[:, None], torch.maximum(byte[head], old), byte[head])
        kept = pages[head].float() * (_power(old) / _power(byte[head]))[..., None, None]
        pages[head] = torch.where(held[:, None, :, None], kept, pages[head].float()).to(E4M3)
        code = (x / _power(byte[page])[..., None]).clamp(-448.0, 448.0).to(E4M3)
        pages.view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
        touched = torch.zeros(pages.shape[0], dtype=torch.bool, device="cuda")
        touched[page] = True
        scales[..., which] = torch.where(touched[:, None], byte.to(torch.uint8), scales[..., which])
    return s["out"], s["k_pages"], s["v_pages"], s["scales"]


def _plain_rules(s):
    x = s["logits"].float()
    B, V = x.shape
    at = torch.arange(s["tokens"].shape[1], device="cuda")
    tokens = s["tokens"].long()
    given = at < s["lens"][:, None]
    answer = given & (at >= s["prompt"][:, None])
    seen = torch.zeros(B, V, device="cuda").scatter_add_(1, tokens, given.float()) > 0
    count = torch.zeros(B, V, device="cuda").scatter_add_(1, tokens, answer.float())
    r = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias_tokens"] is not None:
        n = s["bias_tokens"].numel()
        row = torch.searchsorted(s["bias_starts"][1:].long(), torch.arange(n, device="cuda"), right=True)
        x = x + torch.zeros(B, V, device="cuda").index_put_((row, s["bias_tokens"].long()), s["bias_values"],
                                                            accumulate=True)
    if s["allowed"] is not None:
        bit = (s["allowed"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        x = x.masked_fill(bit.reshape(B, -1)[:, :V] == 0, -math.inf)
    s["out"].copy_(x)
    return s["out"]


# ---- exact results ----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rules":
        return _exact_rules(s)
    ctx, ql = _lens(case)
    if case["kind"] == "append":
        return _exact_append(s, ctx, ql)
    return _exact_attention(s, ctx, ql, case["kind"] == "decode")


def _exact_cache(s, b, n):
    """Keys and values of sequence b, [Hkv][n][D] in 64 bits."""
    pages = s["table"][b, :(n + PAGE - 1) // PAGE].long()
    for which, name in enumerate(("k_pages", "v_pages")):
        power = torch.exp2(s["scales"].view(torch.uint8)[pages][..., which].double() - 127.0)
        x = s[name][pages].double() * power[..., None, None]
        yield x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]


def _exact_attention(s, ctx, ql, padded):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    r = 0
    for b, (n, Q) in enumerate(zip(ctx, ql)):
        k, v = _exact_cache(s, b, n)
        q, o = (s["q"][b, :Q], out[b, :Q]) if padded else (s["q"][r:r + Q], out[r:r + Q])
        G = q.shape[1] // k.shape[0]
        seen = torch.arange(n, device="cuda") <= torch.arange(n - Q, n, device="cuda")[:, None]
        for h in range(q.shape[1]):
            a = (q[:, h].double() @ k[h // G].T.contiguous()) * s["scale"]
            o[:, h] = torch.where(seen, a, -math.inf).softmax(-1) @ v[h // G]
        r += Q
    return out


def _exact_append(s, ctx, ql):
    """New codes without their rounding: value over power."""
    out, kp, vp = (s[x].double() for x in ("out", "k_pages", "v_pages"))
    power = torch.exp2(s["scales"].view(torch.uint8).double() - 127.0)
    half = s["inv_freq"].numel()
    r = 0
    for b, (n, Q) in enumerate(zip(ctx, ql)):
        turn = torch.polar(torch.ones(Q, 1, half, dtype=torch.float64, device="cuda"),
                           torch.arange(n - Q, n, device="cuda").double()[:, None, None] * s["inv_freq"].double())
        new = {}
        for name, weight in (("q", s["q_norm"]), ("k", s["k_norm"])):
            x = s[name][r:r + Q].double()
            if weight is not None:
                x = x / ((x ** 2).mean(-1, keepdim=True) + EPS).sqrt() * weight.double()
            pairs = (x[..., :2 * half].unflatten(-1, (half, 2)) if s["interleaved"] else
                     x[..., :2 * half].unflatten(-1, (2, half)).transpose(-1, -2)).contiguous()
            y = torch.view_as_real(torch.view_as_complex(pairs) * turn)
            y = y.flatten(-2) if s["interleaved"] else y.transpose(-1, -2).flatten(-2)
            new[name] = torch.cat((y, x[..., 2 * half:]), -1)
        out[r:r + Q] = new["q"]
        new["v"] = s["v"][r:r + Q].double()
        held, first = (n - Q) % PAGE, (n - Q) // PAGE
        pids = s["table"][b, first:(n + PAGE - 1) // PAGE].long()
        for which, (pages, x) in enumerate(((kp, new["k"]), (vp, new["v"]))):
            # the new rows laid out page by page, from the first page's first slot
            room = torch.zeros(len(pids) * PAGE, *x.shape[1:], dtype=torch.float64, device="cuda")
            room[held:held + Q] = x
            room = room.view(len(pids), PAGE, *x.shape[1:]).transpose(1, 2)
            most = room.abs().amax((-1, -2))
            scale = torch.exp2(torch.ceil(torch.log2(most / 448.0)).clamp(LOWEST - 127, HIGHEST - 127))
            if held:
                was = power[pids[0], :, which].clone()
                scale[0] = torch.maximum(scale[0], was)
                room[0, :, :held] = pages[pids[0], :, :held] * was[:, None, None]
            room = room / scale[..., None, None]
            end = held + Q - (len(pids) - 1) * PAGE      # slots in use of the last page
            room[-1, :, end:] = pages[pids[-1], :, end:]
            pages[pids] = room
            power[pids, :, which] = scale
        r += Q
    return out, kp, vp, power


def _exact_rules(s):
    x = s["logits"].double()
    out = torch.empty_like(x)
    B, V = x.shape
    starts = None if s["bias_starts"] is None else s["bias_starts"].tolist()
    for b, (n, p) in enumerate(zip(s["lens"].tolist(), s["prompt"].tolist())):
        row = x[b].clone()
        ids = s["tokens"][b, :n].long().unique()
        r = float(s["repetition"][b])
        row[ids] = torch.where(row[ids] > 0, row[ids] / r, row[ids] * r)
        ids, count = s["tokens"][b, p:n].long().unique(return_counts=True)
        row[ids] -= float(s["frequency"][b]) * count.double() + float(s["presence"][b])
        if starts is not None:
            at = slice(starts[b], starts[b + 1])
            row += torch.bincount(s["bias_tokens"][at].long(), weights=s["bias_values"][at].double(), minlength=V)
        if s["allowed"] is not None:
            v = torch.arange(V, device="cuda")
            row[(s["allowed"][b][v // 32].long() >> (v % 32)) % 2 == 0] = -math.inf
        out[b] = row
    return out
