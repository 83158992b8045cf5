"""The calls by which the speed of the generation operators is measured.

Between the prompt's prefill and the answer's tokens a program around the
library has three things done: the rotary positions of q and k with the append
of keys and values to a paged cache (`rope_append`), the attention of each
sequence's new token over that cache (`paged_attention`), and the draw of a
token from each row of logits (`sample`). The decoders are those of the LLaVA
workloads (32 and 40 heads of 128, and grouped heads), the sequences pruned
images with text, or long conversations.

With `own` false `run` computes the operators in elementary torch operations,
else through the Python binding.
"""
import math

import torch

own = False


def listed():
    return [
        # One decode step of one interactive request on the 7B decoder: the new
        # token's position rotation and its key and value into the cache.
        {"name": "append-one-token", "kind": "append", "tokens": 1, "seqs": 1, "H": 32, "Hkv": 32, "dh": 128,
         "page": 16, "dtype": "fp16", "rot": 128, "interleaved": False, "k_rows": False},
        # A decode step of 96 sequences with grouped heads in bfloat16.
        {"name": "append-batch-96", "kind": "append", "tokens": 96, "seqs": 96, "H": 32, "Hkv": 8, "dh": 128,
         "page": 64, "dtype": "bf16", "rot": 128, "interleaved": False, "k_rows": False},
        # Prefill of 32 pruned LLaVA-NeXT images on the 13B decoder (704
        # positions each, kept tokens at their original positions); the rotated
        # key rows are wanted too, for the prompt's attention.
        {"name": "append-prefill-13b-b32", "kind": "append", "tokens": 32 * 704, "seqs": 32, "H": 40, "Hkv": 40,
         "dh": 128, "page": 16, "dtype": "fp16", "rot": 128, "interleaved": False, "k_rows": True},
        # One interactive request: a pruned image and its text, 13B decoder.
        {"name": "attend-one-short", "kind": "attend", "seqs": 1, "longest": 704, "fill": "even", "H": 40,
         "Hkv": 40, "dh": 128, "page": 16, "dtype": "fp16"},
        # One long conversation with grouped heads: all of the work is one
        # sequence's.
        {"name": "attend-one-long", "kind": "attend", "seqs": 1, "longest": 32011, "fill": "even", "H": 32,
         "Hkv": 8, "dh": 128, "page": 64, "dtype": "bf16"},
        # 24 requests of unequal length decoded together on the 13B decoder.
        {"name": "attend-batch-24", "kind": "attend", "seqs": 24, "longest": 2048, "fill": "ragged", "H": 40,
         "Hkv": 40, "dh": 128, "page": 16, "dtype": "fp16"},
        # A loaded server: 128 conversations of very unequal length, grouped
        # heads, one of them much longer than the others.
        {"name": "attend-batch-128", "kind": "attend", "seqs": 128, "longest": 8190, "fill": "skewed", "H": 32,
         "Hkv": 8, "dh": 128, "page": 16, "dtype": "bf16"},
        # A decoder layer's decode step as a model makes it: append, then
        # attention over what the cache holds now.
        {"name": "step-batch-16", "kind": "step", "seqs": 16, "longest": 768, "fill": "ragged", "H": 32, "Hkv": 32,
         "dh": 128, "page": 16, "dtype": "fp16"},
        # The next token of one request, nucleus sampling.
        {"name": "sample-one", "kind": "sample", "rows": 1, "vocab": 32000, "pad": 0, "dtype": "fp16", "mode": "top_p"},
        # A batch whose requests ask for different things.
        {"name": "sample-batch-64", "kind": "sample", "rows": 64, "vocab": 32000, "pad": 64, "dtype": "fp16",
         "mode": "mixed"},
        # A large batch over a large vocabulary of an odd size, fp32 logits.
        {"name": "sample-batch-256-large", "kind": "sample", "rows": 256, "vocab": 131_071, "pad": 5, "dtype": "fp32",
         "mode": "mixed"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "append", "attend", "attend", "attend", "step", "sample", "sample"))
    heads = rng.choice(((32, 32), (40, 40), (32, 8), (40, 8), (28, 4), (24, 2), (8, 1)))
    form = {"H": heads[0], "Hkv": heads[1], "dh": rng.choice((128, 128, 64)), "page": rng.choice((8, 16, 32, 64, 256)),
            "dtype": rng.choice(("fp16", "bf16"))}
    if kind == "append":
        tokens = _log_int(rng, 1, 32 * 704)
        rot = rng.choice((form["dh"], form["dh"], form["dh"] // 2))
        return {"kind": kind, "tokens": tokens, "seqs": min(tokens, _log_int(rng, 1, 128)), **form, "rot": rot,
                "interleaved": rng.random() < 0.3, "k_rows": rng.random() < 0.5}
    if kind in ("attend", "step"):
        longest = _log_int(rng, 1, 40000)
        # at most as many keys as the largest listed case reads
        most = int(1.0e9 / (4 * longest * heads[1] * form["dh"]))
        return {"kind": kind, "seqs": max(1, min(most, _log_int(rng, 1, 192))), "longest": longest,
                "fill": rng.choice(("even", "ragged", "skewed")), **form}
    vocab = rng.choice((32000, 32064, 49_999, rng.randint(1000, 150_000)))
    return {"kind": kind, "rows": _log_int(rng, 1, 256), "vocab": vocab, "pad": rng.choice((0, 0, 3, 64)),
            "dtype": rng.choice(("fp16", "bf16", "fp32")), "mode": rng.choice(("plain", "top_k", "top_p", "min_p", "mixed"))}


# ---------------------------------------------------------------- inputs
_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _spread(case):
    """Cached positions per sequence; the first has the longest, the others are spread evenly, or most of them short."""
    n, longest = case["seqs"], case["longest"]
    power = {"even": 0, "ragged": 1, "skewed": 3}[case["fill"]]
    return [longest] + [min(longest, max(1, int(longest * ((i + 0.5) / (n - 1)) ** power))) for i in range(n - 1)]


def _lengths(case, g):
    """The same lengths for every seed, in an order of its own (int64, on the GPU)."""
    lens = torch.tensor(_spread(case), device="cuda")
    return lens[torch.randperm(lens.numel(), generator=g, device="cuda")]


def _pages(g, lens, longest, page):
    """A page table [seqs, pages of the longest] of shuffled pages (-1 past a sequence's last), and their number."""
    n = lens.numel()
    per = (longest + page - 1) // page
    need = (lens + page - 1) // page
    have = torch.arange(per, device="cuda")[None, :] < need[:, None]
    order = torch.randperm(n * per, generator=g, device="cuda").view(n, per)
    # the pages in use, numbered by a random order: pages of one sequence lie apart
    rank = torch.argsort(torch.argsort(torch.where(have, order, order + n * per).reshape(-1))).view(n, per)
    total = int(need.sum())
    return torch.where(have, rank, -1).to(torch.int32), total


def _cache(g, pages, case):
    shape = (pages, case["page"], case["Hkv"], case["dh"])
    dt = _TYPES[case["dtype"]]
    return _randn(g, shape, dt), _randn(g, shape, dt)


def _rope_tables(positions, rot):
    inv = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv[None, :]
    return a.cos().float(), a.sin().float()


def _fused_rows(g, tokens, case):
    """q, k, v as column blocks of one fused projection output."""
    h, hk, dh = case["H"], case["Hkv"], case["dh"]
    y = _randn(g, (tokens, (h + 2 * hk) * dh), _TYPES[case["dtype"]])
    return y[:, :h * dh], y[:, h * dh:(h + hk) * dh], y[:, (h + hk) * dh:]


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = {"case": case, "kind": kind}
    if kind == "sample":
        _prepare_sample(case, g, s)
        return s
    h, hk, dh, page = case["H"], case["Hkv"], case["dh"], case["page"]
    dt = _TYPES[case["dtype"]]
    if kind == "append":
        n, t = case["seqs"], case["tokens"]
        if t == n:  # a decode step: one token each, at the end of what the cache holds
            lens = 1 + torch.randperm(n, generator=g, device="cuda") * 704 // n
            pos = lens - 1
            seq = None
        else:  # a packed prefill: the tokens of sequence after sequence
            base, extra = t // n, t % n
            lens = torch.full((n,), base, device="cuda", dtype=torch.long)
            lens[:extra] += 1
            seq = torch.repeat_interleave(torch.arange(n, device="cuda"), lens)
            start = torch.cumsum(lens, 0) - lens
            pos = torch.arange(t, device="cuda") - start[seq]
        longest = int(lens.max())
        s["seq"] = None if seq is None else seq.to(torch.int32)
        s["pos"] = pos.to(torch.int32)
        # pruned sequences keep their tokens' original positions, which rise faster
        s["rot_pos"] = (pos * 4 + torch.randint(0, 4, (t,), generator=g, device="cuda")).to(torch.int32)
        s["cos"], s["sin"] = _rope_tables(4 * longest, case["rot"])
        s["table"], pages = _pages(g, lens, longest, page)
        s["k_cache"], s["v_cache"] = _cache(g, pages, case)
        s["q"], s["k"], s["v"] = _fused_rows(g, t, case)
        s["q_out"] = torch.empty((t, h * dh), dtype=dt, device="cuda")
        s["k_out"] = torch.empty((t, hk * dh), dtype=dt, device="cuda") if case["k_rows"] else None
        return s
    lens = _lengths(case, g)
    n = case["seqs"]
    s["lens"] = lens.to(torch.int32)
    s["table"], pages = _pages(g, lens, case["longest"], page)
    s["k_cache"], s["v_cache"] = _cache(g, pages, case)
    s["out"] = torch.empty((n, h * dh), dtype=dt, device="cuda")
    s["lse"] = torch.empty((n, h), dtype=torch.float32, device="cuda")
    s["scratch"] = torch.zeros((24 << 20,), dtype=torch.uint8, device="cuda")  # the attention's workspace
    s["q"], s["k"], s["v"] = _fused_rows(g, n, case)
    if kind == "step":
        s["pos"] = (lens - 1).to(torch.int32)
        s["cos"], s["sin"] = _rope_tables(case["longest"], dh)
        s["q_out"] = torch.empty((n, h * dh), dtype=dt, device="cuda")
    return s


def _prepare_sample(case, g, s):
    rows, vocab, mode = case["rows"], case["vocab"], case["mode"]
    x = torch.randn((rows, vocab + case["pad"]), generator=g, device="cuda", dtype=torch.float32) * 2.5
    # a model's logits: a broad bulk, and a few tokens far above it
    top = torch.randint(0, vocab, (rows, 24), generator=g, device="cuda")
    lift = torch.rand((rows, 24), generator=g, device="cuda") * 10.0
    x.scatter_add_(1, top, lift)
    s["logits"] = x.to(_TYPES[case["dtype"]])[:, :vocab]
    s["u"] = torch.rand((rows,), generator=g, device="cuda", dtype=torch.float32)
    pick = torch.randint(0, 4, (rows,), generator=g, device="cuda")
    rand = torch.rand((rows,), generator=g, device="cuda", dtype=torch.float32)
    s["temperature"] = 0.6 + 0.8 * rand if mode != "plain" else None
    s["top_k"] = s["top_p"] = s["min_p"] = None
    if mode == "mixed":  # some greedy rows, and each row with filters of its own
        s["temperature"] = torch.where(pick == 3, torch.zeros_like(rand), 0.6 + 0.8 * rand)
        s["top_k"] = torch.where(pick == 1, torch.zeros_like(pick), 1 + (rand * 199).long()).to(torch.int32)
        s["top_p"] = torch.where(pick == 2, torch.ones_like(rand), 0.7 + 0.29 * rand)
        s["min_p"] = torch.where(pick == 0, torch.zeros_like(rand), 0.08 * rand)
    elif mode == "top_k":
        s["top_k"] = (1 + (rand * 199).long()).to(torch.int32)
    elif mode == "top_p":
        s["top_p"] = 0.7 + 0.29 * rand
    elif mode == "min_p":
        s["min_p"] = 0.02 + 0.08 * rand
    s["token"] = torch.empty((rows,), dtype=torch.int32, device="cuda")
    s["logprob"] = torch.empty((rows,), dtype=torch.float32, device="cuda")


# ---------------------------------------------------------------- a pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2609_34867_gb300 import p4q

    kind = s["kind"]
    if kind == "sample":
        p4q.p4q_sample(s["logits"], s["u"], s["token"], s["logprob"], temperature=s["temperature"], top_k=s["top_k"],
                       top_p=s["top_p"], min_p=s["min_p"])
        return {"token": s["token"], "logprob": s["logprob"]}
    if kind == "append":
        p4q.p4q_rope_append(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["pos"], s["k_cache"], s["v_cache"],
                            s["table"], s["q_out"], k_out=s["k_out"], seq=s["seq"], rot_pos=s["rot_pos"],
                            interleaved=s["case"]["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    q = s["q"]
    if kind == "step":
        p4q.p4q_rope_append(q, s["k"], s["v"], s["cos"], s["sin"], s["pos"], s["k_cache"], s["v_cache"], s["table"],
                            s["q_out"])
        q = s["q_out"]
    p4q.p4q_paged_attention(q, s["k_cache"], s["v_cache"], s["table"], s["lens"], s["out"], s["scratch"], lse=s["lse"])
    if kind == "step":
        return {"out": s["out"], "lse": s["lse"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return {"out": s["out"], "lse": s["lse"]}


def _run_plain(s):
    kind = s["kind"]
    if kind == "sample":
        return _sample_plain(s)
    if kind == "append":
        return _append_plain(s, s["rot_pos"], s["case"]["rot"], s["case"]["interleaved"])
    if kind == "step":
        r = _append_plain(s, s["pos"], s["case"]["dh"], False)
        return {**_attend_plain(s, r["q"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    return _attend_plain(s, s["q"])


def _rotate_plain(x, cos, sin, rot, interleaved):
    """x [T, heads, dh] fp32, cos and sin [T, rot / 2] -> the rotated rows."""
    a, rest = x[..., :rot], x[..., rot:]
    c, d = cos[:, None, :], sin[:, None, :]
    if interleaved:
        lo, hi = a[..., 0::2], a[..., 1::2]
        r = torch.stack((lo * c - hi * d, hi * c + lo * d), dim=-1).flatten(-2)
    else:
        lo, hi = a[..., :rot // 2], a[..., rot // 2:]
        r = torch.cat((lo * c - hi * d, hi * c + lo * d), dim=-1)
    return torch.cat((r, rest), dim=-1)


def _append_plain(s, rot_pos, rot, interleaved):
    case = s["case"]
    h, hk, dh, page = case["H"], case["Hkv"], case["dh"], case["page"]
    t = s["q"].shape[0]
    at = rot_pos.long()
    cos, sin = s["cos"][at], s["sin"][at]
    q = _rotate_plain(s["q"].float().view(t, h, dh), cos, sin, rot, interleaved).to(s["q"].dtype)
    k = _rotate_plain(s["k"].float().view(t, hk, dh), cos, sin, rot, interleaved).to(s["q"].dtype)
    pos = s["pos"].long()
    seq = torch.arange(t, device="cuda") if s.get("seq") is None else s["seq"].long()
    where = s["table"].long()[seq, pos // page], pos % page
    s["k_cache"].index_put_(where, k)
    s["v_cache"].index_put_(where, s["v"].view(t, hk, dh))
    return {"q": q.view(t, h * dh), "k": k.view(t, hk * dh) if s.get("k_out") is not None else None,
            "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend_plain(s, q):
    case = s["case"]
    n, h, hk, dh = case["seqs"], case["H"], case["Hkv"], case["dh"]
    at = s["table"].long().clamp(min=0)
    k = s["k_cache"][at].flatten(1, 2).float()  # [n, positions, hk, dh]
    v = s["v_cache"][at].flatten(1, 2).float()
    live = torch.arange(k.shape[1], device="cuda")[None, :] < s["lens"][:, None]
    scores = torch.einsum("bhgd,blhd->bhgl", q.float().view(n, hk, h // hk, dh), k) * (1.0 / math.sqrt(dh))
    scores = scores.masked_fill(~live[:, None, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - top)
    z = e.sum(-1, keepdim=True)
    v = torch.where(live[:, :, None, None], v, torch.zeros((), device="cuda"))
    o = torch.einsum("bhgl,blhd->bhgd", e, v) / z
    lse = (top + torch.log(z)).reshape(n, h)
    return {"out": o.reshape(n, h * dh).to(q.dtype), "lse": lse}


def _sample_plain(s):
    """The operator in whole weights: w = 2^31 exp((x - max) / T), rounded."""
    x = s["logits"].float()
    rows, vocab = x.shape
    x = torch.where(torch.isnan(x), -math.inf, x)
    one = torch.ones((rows,), device="cuda")
    t = one if s["temperature"] is None else s["temperature"]
    greedy = ~(t > 0)
    t = torch.where(greedy, one, t)
    k = torch.zeros((rows,), dtype=torch.long, device="cuda") if s["top_k"] is None else s["top_k"].long()
    k = torch.where((k <= 0) | (k > vocab), vocab, k)
    k = torch.where(greedy, 1, k)
    top_p = one if s["top_p"] is None else s["top_p"]
    min_p = one * 0 if s["min_p"] is None else s["min_p"]
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    top = x[:, :1]
    d = torch.where(x == top, torch.zeros((), device="cuda"), (top - x) * (1.0 / t)[:, None])
    e = torch.exp(-d)
    w = torch.round(e * 2147483648.0).long()
    w = w * (torch.arange(vocab, device="cuda")[None, :] < k[:, None])
    mass = torch.cumsum(w, 1)
    need = torch.ceil(top_p.double() * mass[:, -1].double())
    w = w * (((mass - w).double() < need[:, None].clamp(min=1)) | (top_p >= 1)[:, None])
    w = w * (e >= min_p.clamp(max=1)[:, None])
    by_index = torch.zeros_like(w).scatter_(1, order, w)
    mass = torch.cumsum(by_index, 1)
    total = mass[:, -1]
    r = torch.floor(s["u"].double() * total.double()).long().clamp(min=0)
    r = torch.minimum(r, total - 1)
    token = (mass <= r[:, None]).sum(1)
    d = torch.zeros_like(d).scatter_(1, order, d)
    share = (total.double() * 2.0 ** -31).float()
    logprob = -d.gather(1, token[:, None])[:, 0] - torch.log(share)
    return {"token": token.to(torch.int32), "logprob": logprob}


# ---------------------------------------------------------------- the work and the exact results
def work(case):
    kind = case["kind"]
    if kind == "sample":
        size = {"fp16": 2, "bf16": 2, "fp32": 4}[case["dtype"]]
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * 28, "flops": 4 * n}
    h, hk, dh = case["H"], case["Hkv"], case["dh"]
    if kind == "append":
        t = case["tokens"]
        moved = 2 * (h + 2 * hk) + (hk if case["k_rows"] else 0)
        return {"bytes": t * (moved * dh * 2 + case["rot"] * 4 + 16), "flops": 3 * t * (h + hk) * case["rot"]}
    keys, n = sum(_spread(case)), case["seqs"]
    w = {"bytes": 4 * keys * hk * dh + 4 * n * h * dh + 4 * n * h + 4 * keys / case["page"], "flops": 4 * keys * h * dh}
    if kind == "step":
        w["bytes"] += n * (4 * (h + 2 * hk) * dh + dh * 4)
    return w


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(s)
    h, hk, dh, page = case["H"], case["Hkv"], case["dh"], case["page"]
    q = s["q"].double()
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    if kind in ("append", "step"):
        t = q.shape[0]
        at = (s["rot_pos"] if kind == "append" else s["pos"]).long()
        rot = case["rot"] if kind == "append" else dh
        inter = kind == "append" and case["interleaved"]
        # pair (a, b) of each dimension, and its angle's column
        i = torch.arange(rot // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)

        def turned(x, heads):
            x = x.reshape(t, heads, dh)
            z = torch.complex(x[..., a], x[..., b]) * torch.complex(s["cos"].double(), s["sin"].double())[at][:, None, :]
            y = x.clone()
            y[..., a], y[..., b] = z.real, z.imag
            return y

        q, k = turned(q, h).reshape(t, h * dh), turned(s["k"].double(), hk)
        seq = torch.arange(t, device="cuda") if s.get("seq") is None else s["seq"].long()
        pos = s["pos"].long()
        slot = s["table"].long()[seq, torch.div(pos, page, rounding_mode="floor")] * page + pos % page
        kc.view(-1, hk, dh)[slot] = k
        vc.view(-1, hk, dh)[slot] = s["v"].double().reshape(t, hk, dh)
        if kind == "append":
            return {"q": q, "k": k.reshape(t, hk * dh) if case["k_rows"] else None, "k_cache": kc, "v_cache": vc}
    out, lse = [], []
    for n in range(case["seqs"]):
        length = int(s["lens"][n])
        used = s["table"][n, :(length + page - 1) // page].long()
        k, v = (c[used].reshape(-1, hk, dh)[:length].repeat_interleave(h // hk, 1) for c in (kc, vc))
        scores = (k * q[n].view(1, h, dh)).sum(-1) / math.sqrt(dh)  # [length, h]
        p = torch.softmax(scores, 0)
        out.append((p[:, :, None] * v).sum(0).reshape(h * dh))
        lse.append(torch.logsumexp(scores, 0))
    r = {"out": torch.stack(out), "lse": torch.stack(lse)}
    if kind == "step":
        r["k_cache"], r["v_cache"] = kc, vc
    return r


def _exact_sample(s):
    """One row at a time on the host, the weights from 64-bit exponentials."""
    x_all = s["logits"].double().cpu()
    rows, vocab = x_all.shape
    u = s["u"].cpu().tolist()
    value = {name: None if s[name] is None else s[name].cpu().tolist() for name in ("temperature", "top_k", "top_p", "min_p")}
    token, logprob = [], []
    for n in range(rows):
        x = x_all[n]
        t = 1.0 if value["temperature"] is None else value["temperature"][n]
        if t <= 0:
            token.append(int(x.argmax()))
            logprob.append(0.0)
            continue
        e = torch.exp((x - x.max()) / t)
        w = torch.round(e * 2.0 ** 31).long()
        order = torch.argsort(x, descending=True, stable=True)
        k = value["top_k"][n] if value["top_k"] is not None and 0 < value["top_k"][n] < vocab else vocab
        kept = order[:k]
        if value["top_p"] is not None and value["top_p"][n] < 1:
            mass = torch.cumsum(w[kept], 0)
            need = max(1, math.ceil(value["top_p"][n] * int(mass[-1])))
            kept = kept[:int(torch.searchsorted(mass, need)) + 1]
        if value["min_p"] is not None:
            kept = kept[e[kept] >= min(1.0, value["min_p"][n])]
        kept = torch.sort(kept).values
        mass = torch.cumsum(w[kept], 0)
        total = int(mass[-1])
        r = min(max(0, int(u[n] * total)), total - 1)
        i = int(kept[int(torch.searchsorted(mass, r, right=True))])
        token.append(i)
        logprob.append(math.log(float(e[i])) - math.log(total / 2.0 ** 31))
    return {"token": torch.tensor(token, dtype=torch.int32), "logprob": torch.tensor(logprob, dtype=torch.float64)}
