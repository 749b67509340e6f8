"""Cases of the operators that serve the layers in 8-bit floating point, and of the draw of a token.

Beside the calls of ``operators.py`` a program that serves a model makes these:

* ``linear``: activations quantised to e4m3 with a scale for each token and 128
  channels, and their product with an e4m3 weight that has a scale for each
  block of 128 x 128;
* ``kv``: new tokens' keys and values added to a paged cache in e4m3 with a
  scale for each 32 tokens and head, and the blocks they went to read back;
* ``attn``: attention over that cache, for single tokens and for prompts;
* ``sample``: a token drawn from the logits of each row, with temperature,
  top-k, top-p and min-p, from given uniform numbers.

Hidden and intermediate sizes are those of the synthetic workloads; lengths,
batches, vocabularies and odd sizes are generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False                           # True: the framework's operators; False: their plain forms

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
HIDDEN = [512, 1024, 4096, 5120, 8192, 12288, 14336]
E4M3 = torch.float8_e4m3fn
MOST = 448.0                          # largest e4m3 value
BLOCK = 32                            # tokens of the cache that share a scale


def listed():
    return [
        # one token through an up projection: the weight is read once
        {"name": "linear_token", "kind": "linear", "M": 1, "K": 4096, "N": 14336, "type": "fp16", "bias": False},
        # a decode batch, odd, through a layer with a bias whose sizes are no multiples of the blocks
        {"name": "linear_batch", "kind": "linear", "M": 131, "K": 5000, "N": 8191, "type": "fp16", "bias": True},
        # a long prefill through the largest up projection
        {"name": "linear_prompt", "kind": "linear", "M": 8192, "K": 8192, "N": 28672, "type": "bf16", "bias": False},
        # a decode step of 32 sequences: one token each, into blocks that hold some already
        {"name": "kv_token", "kind": "kv", "B": 32, "H": 8, "D": 128, "new": 1, "old": 1501, "page": 32, "type": "fp16"},
        # prompts of 16381 tokens in all, the second part of contexts that have begun
        {"name": "kv_prompt", "kind": "kv", "B": 5, "H": 8, "D": 128, "new": 4095, "old": 777, "page": 64, "type": "bf16"},
        # one sequence, one token, small heads: latency
        {"name": "attn_token", "kind": "attn", "B": 1, "Hq": 32, "H": 8, "D": 64, "q": 1, "lo": 1003, "hi": 1003,
         "page": 32, "type": "fp16"},
        # two long contexts: the work is along the cache
        {"name": "attn_long", "kind": "attn", "B": 2, "Hq": 64, "H": 8, "D": 128, "q": 1, "lo": 100001, "hi": 131072,
         "page": 64, "type": "bf16"},
        # a decode batch of ragged contexts
        {"name": "attn_batch", "kind": "attn", "B": 64, "Hq": 32, "H": 8, "D": 128, "q": 1, "lo": 257, "hi": 8191,
         "page": 64, "type": "fp16"},
        # prompts' chunks of up to 2047 tokens at the end of contexts of up to 4095
        {"name": "attn_prompt", "kind": "attn", "B": 4, "Hq": 32, "H": 8, "D": 128, "q": 2047, "lo": 1025, "hi": 4095,
         "page": 128, "type": "bf16"},
        # one row, fp32 logits of the 8-bit projection, few tokens kept: latency
        {"name": "sample_token", "kind": "sample", "rows": 1, "V": 32003, "type": "fp32", "spread": 3.0, "filters": "kp"},
        # a decode batch over a large vocabulary with every filter
        {"name": "sample_batch", "kind": "sample", "rows": 128, "V": 131071, "type": "fp32", "spread": 3.0, "filters": "kpm"},
        # many rows of flat 16-bit logits, with many equal ones, and only top-p: most tokens are candidates
        {"name": "sample_flat", "kind": "sample", "rows": 203, "V": 50000, "type": "bf16", "spread": 0.7, "filters": "p"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "kv", "attn", "attn", "sample"])
    dtype = rng.choice(["fp16", "bf16"])
    if kind == "linear":
        k = rng.choice(HIDDEN + [8 * _log(rng, 8, 3584)])
        n = rng.choice(HIDDEN + [_log(rng, 64, 50000)])
        return {"kind": kind, "M": max(1, min(_log(rng, 1, 8192), 8192 * 8192 * 28672 // (n * k))), "K": k, "N": n,
                "type": dtype, "bias": rng.random() < 0.5}
    if kind == "sample":
        v = _log(rng, 1000, 262144)
        return {"kind": kind, "rows": max(1, min(_log(rng, 1, 512), 128 * 131071 // v)), "V": v,
                "type": rng.choice(["fp32", "fp16", "bf16"]), "spread": rng.uniform(0.5, 6.0),
                "filters": rng.choice(["", "k", "p", "m", "kp", "pm", "kpm"])}
    h, g, d = rng.choice([(1, 8), (2, 4), (4, 4), (8, 1), (8, 4), (8, 5), (8, 8), (16, 1), (32, 1)]) + (rng.choice([64, 128]),)
    page = rng.choice([32, 64, 128])
    if kind == "kv":
        b = _log(rng, 1, 128)
        new = rng.choice([1, max(1, min(_log(rng, 1, 8191), 16381 * 8 * 128 // (b * h * d)))])
        return {"kind": kind, "B": b, "H": h, "D": d, "new": new, "old": rng.choice([0, _log(rng, 1, 2000)]), "page": page,
                "type": dtype}
    if rng.random() < 0.6:
        b = _log(rng, 1, 128)
        hi = max(32, min(_log(rng, 32, 131072), 64 * 8192 * 8 * 128 // (b * h * d)))
        return {"kind": kind, "B": b, "Hq": h * g, "H": h, "D": d, "q": 1, "lo": rng.randint(1, hi), "hi": hi, "page": page,
                "type": dtype}
    b, q = rng.randint(1, 4), _log(rng, 2, 2047)
    hi = max(q, min(_log(rng, 32, 8192), 4 * 32 * 2047 * 4095 // (b * h * g * q)))
    return {"kind": kind, "B": b, "Hq": h * g, "H": h, "D": d, "q": q, "lo": rng.randint(1, hi), "hi": hi, "page": page,
            "type": dtype}


def _lens(case):
    """Lengths of the sequences, spread between two bounds, and how many tokens at their ends are new (or ask)."""
    if case["kind"] == "kv":
        new = [max(1, case["new"] - (b * case["new"]) // (2 * case["B"])) for b in range(case["B"])]
        return [n + int(case["old"] * ((0.5 + b * 0.618034) % 1.0)) for b, n in enumerate(new)], new
    kv = [case["lo"] + int((case["hi"] - case["lo"]) * ((b * 0.618034) % 1.0)) for b in range(case["B"])]
    kv[-1] = case["hi"]
    q = [max(1, min(case["q"] - (b * case["q"]) // (3 * case["B"]), n)) for b, n in enumerate(kv)]
    return kv, q


def work(case):
    kind = case["kind"]
    if kind == "linear":
        m, k, n = case["M"], case["K"], case["N"]
        g, size = -(-k // 128), 2
        return {"bytes": size * m * k + 2 * m * k + 8 * m * g + n * k + 4 * (-(-n // 128)) * g + size * m * n
                + (size * n if case["bias"] else 0), "flops": 2 * m * n * k}
    if kind == "sample":
        n = case["rows"] * case["V"]
        return {"bytes": n * (4 if case["type"] == "fp32" else 2) + 32 * case["rows"], "flops": 20 * n}
    kv, q = _lens(case)
    if kind == "kv":
        rows, back = sum(q) * case["H"], sum(n - (n - a) // BLOCK * BLOCK for n, a in zip(kv, q)) * case["H"]
        return {"bytes": 2 * case["D"] * (2 * rows + rows + back + 2 * back), "flops": 8 * rows * case["D"]}
    seen = sum(a * n - a * (a - 1) // 2 for n, a in zip(kv, q))
    return {"bytes": 2 * sum(kv) * case["H"] * case["D"] + sum(kv) * case["H"] // 16 + 4 * sum(q) * case["Hq"] * case["D"],
            "flops": 4 * seen * case["Hq"] * case["D"]}


# ------------------------------------------------------------------ inputs --
def _starts(counts):
    return torch.tensor([0, *counts], device="cuda").cumsum(0).int()


def _inputs(case, seed):
    """The data of a case, the same for every form of the operators."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=dev)

    kind, dtype = case["kind"], TYPES[case["type"]]
    if kind == "linear":
        m, k, n = case["M"], case["K"], case["N"]
        x = normal(m, k)
        x[:, torch.randint(0, k, (4,), generator=gen, device=dev)] *= 30.0      # outlier channels, as in the synthetic workloads
        return {"x": x.to(dtype), "w": normal(n, k).mul_(120.0).clamp_(-MOST, MOST).to(E4M3),
                "sw": 1e-4 * (0.5 + uniform(-(-n // 128), -(-k // 128))), "bias": normal(n).to(dtype) if case["bias"] else None}
    if kind == "sample":
        r, v = case["rows"], case["V"]
        return {"logits": normal(r, v).mul_(case["spread"]).to(dtype), "u": uniform(r), "temperature": 0.5 + uniform(r),
                "top_k": torch.randint(1, 1000, (r,), generator=gen, device=dev).int() if "k" in case["filters"] else None,
                "top_p": 0.5 + 0.49 * uniform(r) if "p" in case["filters"] else None,
                "min_p": 0.002 + 0.1 * uniform(r) if "m" in case["filters"] else None}
    h, d, page = case["H"], case["D"], case["page"]
    kv, q = _lens(case)
    counts = torch.tensor([-(-n // page) for n in kv], device=dev)
    pages = sum(-(-n // page) for n in kv) + 1
    order = torch.randperm(pages, generator=gen, device=dev)                # pages of a sequence need not be neighbours
    column = torch.arange(-(-max(kv) // page), device=dev)
    first = torch.cumsum(counts, 0) - counts
    table = torch.where(column < counts[:, None], order[torch.clamp(first[:, None] + column, max=pages - 1)], 0).int()
    total = sum(kv)
    k = torch.empty((total, h, d), dtype=dtype, device=dev)
    v = torch.empty_like(k)
    for at in range(0, total, 65536):
        rows = min(65536, total - at)
        block = normal(rows, h, d)
        block[..., ::16] += 4.0                     # keys have channels with a mean of their own
        k[at:at + rows] = block
        v[at:at + rows] = normal(rows, h, d)
    a = {"k": k, "v": v, "pages": pages, "table": table, "kv_lens": torch.tensor(kv, dtype=torch.int32, device=dev),
         "cu_kv": _starts(kv), "cu_q": _starts(q), "max_q": max(q), "max_kv": max(kv)}
    if kind == "attn":
        a["q"] = normal(sum(q), case["Hq"], d).to(dtype)
        return a
    # of each sequence the tokens that were there, and the new ones; and the slots of the blocks that the new ones go to
    seq = torch.repeat_interleave(torch.arange(len(kv), device=dev), a["kv_lens"].long())
    at = torch.arange(total, device=dev) - a["cu_kv"][seq]
    had = (a["kv_lens"] - (a["cu_q"][1:] - a["cu_q"][:-1]))
    a["old_lens"], a["cu_old"] = had, torch.nn.functional.pad(had.cumsum(0), (1, 0)).int()
    new, touched = at >= had[seq], at >= had[seq] // BLOCK * BLOCK
    a["slots"] = (table[seq, at // page].long() * page + at % page)[touched]
    a["old_k"], a["old_v"], a["k"], a["v"] = k[~new], v[~new], k[new], v[new]
    a["blocks"] = sum(-(-n // BLOCK) - (n - c) // BLOCK for n, c in zip(kv, q))
    a["old_blocks"] = sum(-(-(n - c) // BLOCK) for n, c in zip(kv, q))
    return a


def _plain_cache(case, s):
    n, h, d = s["pages"] * case["page"], case["H"], case["D"]
    return [(torch.zeros((n, h, d), dtype=torch.uint8, device="cuda"), torch.zeros((n // BLOCK, h), device="cuda")) for _ in range(2)]


def _plain_append(case, cache, k, v, table, lens, starts, blocks):
    """New tokens, rows starts[b] .. of k and v, at the ends of sequences of `lens` tokens with them; they reach
    `blocks` blocks of 32 tokens."""
    page = case["page"]
    had = lens.long() - (starts[1:] - starts[:-1]).long()
    begin = had // BLOCK
    many = torch.clamp(-(-lens.long() // BLOCK) - begin, min=0)
    seq = torch.repeat_interleave(torch.arange(lens.numel(), device="cuda"), many, output_size=blocks)
    block = begin[seq] + torch.arange(blocks, device="cuda") - (many.cumsum(0) - many)[seq]
    at = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    old, there = at < had[seq, None], at < lens[seq, None]
    slot = table[seq[:, None], torch.clamp(at // page, max=table.shape[1] - 1)].long() * page + at % page
    row = torch.where(there & ~old, starts[seq, None] + at - had[seq, None], 0)
    has_old = old[:, :1].expand(-1, cache[0][0].shape[1])
    for x, (codes, exponent) in zip((k, v), cache):
        fresh = torch.where((there & ~old)[:, :, None, None], x[row].float(), 0.0)
        mantissa, e = torch.frexp(fresh.abs().amax((1, 3)))                 # largest = mantissa 2^e, 1/2 <= mantissa < 1
        e = (e - 9 + (mantissa > MOST / 512).int()).float()
        held = exponent[slot[:, 0] // BLOCK]
        e = torch.where(has_old, torch.maximum(e, held), e)
        moved = codes[slot].view(E4M3).float() * torch.exp2(held - e)[:, None, :, None]
        new = torch.where(old[:, :, None, None], moved, fresh * torch.exp2(-e)[:, None, :, None])
        exponent[slot[:, 0] // BLOCK] = e
        codes[slot[there]] = new[there].to(E4M3).view(torch.uint8)


def _plain_values(held, slots):
    codes, exponent = held
    return codes[slots].view(E4M3).float() * torch.exp2(exponent[slots // BLOCK])[..., None]


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    kind = case["kind"]
    if kind == "attn":
        fill = [s.pop("k"), s.pop("v"), s["table"], s["kv_lens"], s.pop("cu_kv")]
        blocks = sum(-(-n // BLOCK) for n in _lens(case)[0])
    elif kind == "kv":
        fill = [s.pop("old_k"), s.pop("old_v"), s["table"], s.pop("old_lens"), s.pop("cu_old")]
        blocks = s.pop("old_blocks")
    if own:
        import paper_2606_15652_amd as mq
        if kind == "linear":                        # weights laid out once, as a loader does
            s["pw"] = mq.repack_weight_fp8(s.pop("w"), s.pop("sw"))
        if kind in ("kv", "attn"):
            s["cache"] = mq.kv8_cache(s["pages"], case["page"], case["H"], case["D"], device="cuda")
            mq.kv8_append(s["cache"], *fill[:4], cu_new=fill[4])
    elif kind in ("kv", "attn"):
        s["cache"] = _plain_cache(case, s)
        _plain_append(case, s["cache"], *fill, blocks)
    return s


# --------------------------------------------------------------------- run --
def _plain_linear(s):
    dtype, x = TYPES[s["case"]["type"]], s["x"].float()
    m, k = x.shape
    n, groups = s["w"].shape[0], -(-k // 128)
    x = torch.nn.functional.pad(x, (0, groups * 128 - k)).reshape(m, groups, 128)
    scale = x.abs().amax(-1) / torch.full((), MOST, device="cuda")     # (by a Python number torch multiplies by its reciprocal)
    code = torch.where(scale[..., None] > 0, x / scale[..., None], 0.0).clamp_(-MOST, MOST).to(E4M3)
    values = (code.float() * scale[..., None]).reshape(m, -1)[:, :k]
    weight = s["w"].float()
    weight *= torch.repeat_interleave(torch.repeat_interleave(s["sw"], 128, 0)[:n], 128, 1)[:, :k]
    y = torch.matmul(values, weight.t())
    return [code.reshape(m, -1)[:, :k], scale, (y if s["bias"] is None else y + s["bias"].float()).to(dtype)]


def _plain_kv(s):
    dtype = TYPES[s["case"]["type"]]
    _plain_append(s["case"], s["cache"], s["k"], s["v"], s["table"], s["kv_lens"], s["cu_q"], s["blocks"])
    return [_plain_values(held, s["slots"]).to(dtype) for held in s["cache"]]


def _plain_attn(s):
    case = s["case"]
    b, hq, h, d, page = (case[n] for n in ("B", "Hq", "H", "D", "page"))
    g, most_q, most = hq // h, s["max_q"], s["table"].shape[1] * page
    token = (s["table"].long()[:, :, None] * page + torch.arange(page, device="cuda")).reshape(b, most)
    k, v = (_plain_values(held, token).transpose(1, 2).contiguous() for held in s["cache"])
    start, count = s["cu_q"][:-1].long(), (s["cu_q"][1:] - s["cu_q"][:-1]).long()
    i = torch.arange(most_q, device="cuda")
    row = torch.clamp(start[:, None] + i, max=s["q"].shape[0] - 1)
    q = s["q"][row].float().reshape(b, most_q, h, g, d).permute(0, 2, 3, 1, 4).reshape(b, h, g * most_q, d)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).reshape(b, h, g, most_q, most).mul_(1.0 / math.sqrt(d))
    last = s["kv_lens"].long()[:, None] - count[:, None] + i
    hidden = torch.arange(most, device="cuda") > last[:, :, None]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(score.reshape(b, h, g * most_q, most), v) / score.sum(-1).reshape(b, h, g * most_q, 1)
    o = o.reshape(b, h, g, most_q, d).permute(0, 3, 1, 2, 4).reshape(b, most_q, hq, d)
    return o[i < count[:, None]].to(TYPES[case["type"]])


def _plain_sample(s):
    x, order = torch.sort(s["logits"].float(), dim=-1, descending=True, stable=True)
    # in 64 bits: sums of a whole vocabulary next to a border
    w = torch.exp((x.double() - x[:, :1].double()) / s["temperature"].double()[:, None])
    keep = torch.ones_like(x, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= torch.arange(x.shape[1], device="cuda") < s["top_k"][:, None]
    if s["top_p"] is not None:
        kept = w * keep
        total = kept.cumsum(-1)
        keep &= total - kept < s["top_p"].double()[:, None] * total[:, -1:]
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    total = (w * keep).cumsum(-1)
    sums = total[:, -1:]
    at = (total > s["u"].double()[:, None] * sums).int().argmax(-1, keepdim=True)
    return [order.gather(1, at)[:, 0], (w.gather(1, at) / sums).float()[:, 0]]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return {"linear": _plain_linear, "kv": _plain_kv, "attn": _plain_attn, "sample": _plain_sample}[kind](s)
    import paper_2606_15652_amd as mq
    dtype = TYPES[case["type"]]
    if kind == "linear":
        codes, scale = mq.quantize_rows_fp8(s["x"])
        return [codes, scale, mq.gemm_fp8(codes, scale, s["pw"], bias=s["bias"], out_dtype=dtype)]
    if kind == "kv":
        mq.kv8_append(s["cache"], s["k"], s["v"], s["table"], s["kv_lens"], cu_new=s["cu_q"] if case["new"] > 1 else None)
        return list(mq.kv8_read(s["cache"], s["slots"], dtype))
    if kind == "sample":
        return list(mq.sample(s["logits"], s["u"], s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"]))
    return mq.attention_kv8(s["q"], s["cache"], s["table"], s["kv_lens"], cu_q=s["cu_q"] if s["max_q"] > 1 else None,
                            max_q=s["max_q"], max_kv=s["max_kv"])


# ------------------------------------------------------- the definition, in 64 bits --
def _exact_round(x):
    """The e4m3 value nearest to x, of two the one with an even last digit; |x| <= 448 or a little more."""
    step = torch.exp2(torch.floor(torch.log2(torch.clamp(x.abs(), min=2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-MOST, MOST)


def _exact_exponent(x):
    """Least e with |x| <= 448 2^e throughout the last two dimensions."""
    big = x.abs().amax((-1, -2), keepdim=True) / MOST
    e = torch.ceil(torch.log2(big))
    e = torch.where(torch.exp2(e - 1) >= big, e - 1, e)
    return torch.where(torch.exp2(e) < big, e + 1, e)


def _exact_cache(x):
    """What a sequence's rows x [n, H, D], written at once, stand for."""
    n, h, d = x.shape
    blocks = torch.nn.functional.pad(x.double(), (0, 0, 0, 0, 0, -n % BLOCK)).reshape(-1, BLOCK, h, d).transpose(1, 2)
    unit = torch.exp2(_exact_exponent(blocks))
    return (_exact_round(blocks / unit) * unit).transpose(1, 2).reshape(-1, h, d)[:n]


def _exact_kv(a, case):
    out = [[], []]
    at, was = a["cu_q"].tolist(), a["cu_old"].tolist()
    for b, n in enumerate(a["kv_lens"].tolist()):
        had = was[b + 1] - was[b]
        at_block = had // BLOCK * BLOCK
        for o, name in zip(out, ("k", "v")):
            new = a[name][at[b]:at[b + 1]].double()
            part = a["old_" + name][was[b] + at_block:was[b + 1]].double()      # what the first block holds
            if part.shape[0] == 0:
                o.append(_exact_cache(new))
                continue
            m = min(BLOCK - part.shape[0], new.shape[0])
            e_old = _exact_exponent(part.transpose(0, 1))
            held = _exact_round(part.transpose(0, 1) / torch.exp2(e_old)) * torch.exp2(e_old)
            e = torch.maximum(e_old, _exact_exponent(new[:m].transpose(0, 1)))
            both = torch.cat((held, new[:m].transpose(0, 1)), 1) / torch.exp2(e)
            o.append((_exact_round(both) * torch.exp2(e)).transpose(0, 1))
            if m < new.shape[0]:
                o.append(_exact_cache(new[m:]))
    return [torch.cat(o) for o in out]


def _exact_sample(a, rows):
    x = a["logits"].double().cpu().numpy()
    given = {n: None if a[n] is None else a[n].double().cpu().numpy() for n in ("u", "temperature", "top_k", "top_p", "min_p")}
    tokens, probs = [], []
    for r in range(rows):
        order = np.lexsort((np.arange(x.shape[1]), -x[r]))
        w = np.exp((x[r][order] - x[r].max()) / given["temperature"][r])
        if given["top_k"] is not None:
            w = w[:int(given["top_k"][r])]
        if given["top_p"] is not None:
            sums = np.cumsum(w.astype(np.longdouble))
            w = w[:int(np.searchsorted(sums, given["top_p"][r] * sums[-1])) + 1]
        if given["min_p"] is not None:
            w = w[:int((w >= given["min_p"][r]).sum())]
        sums = np.cumsum(w.astype(np.longdouble))
        at = int(np.searchsorted(sums, given["u"][r] * sums[-1], side="right"))
        tokens.append(int(order[at]))
        probs.append(float(w[at] / sums[-1]))
    return [torch.tensor(tokens, device="cuda"), torch.tensor(probs, dtype=torch.float64, device="cuda")]


def exact(case, seed):
    a = _inputs(case, seed)
    kind = case["kind"]
    if kind == "linear":
        m, k = a["x"].shape
        groups = -(-k // 128)
        x = torch.zeros((m, groups * 128), dtype=torch.float64, device="cuda")
        x[:, :k] = a["x"].double()
        scale = (x.reshape(m, groups, 128).abs().amax(-1) / MOST).float().double()
        # codes are of the quotient by the scale that is kept, once rounded to 32 bits
        code = _exact_round((x / torch.clamp(scale, min=1e-300).repeat_interleave(128, 1)).float().double())[:, :k]
        values = code * scale.repeat_interleave(128, 1)[:, :k]
        y = torch.zeros((m, case["N"]), dtype=torch.float64, device="cuda")
        for nb in range(a["sw"].shape[0]):          # weights by rows of blocks
            rows = slice(nb * 128, min(nb * 128 + 128, case["N"]))
            w = a["w"][rows].double() * a["sw"][nb].double().repeat_interleave(128)[:k]
            y[:, rows] = torch.mm(values, w.t().contiguous())
        return [code, scale, y if a["bias"] is None else y + a["bias"].double()]
    if kind == "kv":
        return _exact_kv(a, case)
    if kind == "sample":
        return _exact_sample(a, case["rows"])
    h, g, d = case["H"], case["Hq"] // case["H"], case["D"]
    out = torch.empty(a["q"].shape, dtype=torch.float64, device="cuda")
    at, row = a["cu_q"].tolist(), a["cu_kv"].tolist()
    for b, n in enumerate(a["kv_lens"].tolist()):
        t = torch.arange(n, device="cuda")
        k, v = _exact_cache(a["k"][row[b]:row[b + 1]]), _exact_cache(a["v"][row[b]:row[b + 1]])
        q = a["q"][at[b]:at[b + 1]].double()
        c = q.shape[0]
        seen = t <= (n - c + torch.arange(c, device="cuda"))[:, None]
        for j in range(h):
            kt = k[:, j].t().contiguous()
            vj = v[:, j].contiguous()
            for i in range(g):
                w = torch.mm(q[:, j * g + i].contiguous(), kt) / math.sqrt(d)
                w = torch.softmax(torch.where(seen, w, -math.inf), -1)
                out[at[b]:at[b + 1], j * g + i] = torch.mm(w, vj)
    return out
