"""The calls by which the speed of the compact and the shared cache is measured.

A server that answers many questions at once spends its decode steps on reading
keys and values. Two things make them fewer: a cache of 8 or 4 bits, whose codes
are written as the tokens are appended (`rope_append_quant`) and read back by the
attention of each sequence's new token (`paged_attention_quant`); and one reading of
a prefix that several sequences share, a pruned image with the questions about
it or one prompt with many samples (`prefix_attention`). The decoders are those of
the LLaVA workloads (32 and 40 heads of 128) and of grouped heads.

A written cache comes back as its codes and scales, which the operator defines bit
for bit, and with "rows" as the values that they stand for.

With `own` false `run` computes the operators in elementary torch operations,
else through the Python binding.
"""
import math

import torch

own = False


def listed():
    return [
        # One decode step of one interactive request on the 7B decoder: the new
        # token's rotation, its key and value into a cache of 8 bits.
        {"name": "append-one-token-8bit", "kind": "append", "tokens": 1, "seqs": 1, "H": 32, "Hkv": 32, "dh": 128,
         "page": 16, "dtype": "fp16", "bits": 8, "rot": 128, "interleaved": False, "rows": False},
        # A decode step of 96 sequences with grouped heads, 4 bits.
        {"name": "append-batch-96-4bit", "kind": "append", "tokens": 96, "seqs": 96, "H": 32, "Hkv": 8, "dh": 128,
         "page": 64, "dtype": "bf16", "bits": 4, "rot": 128, "interleaved": False, "rows": False},
        # Prefill of 32 pruned LLaVA-NeXT images on the 13B decoder (704
        # positions each, kept tokens at their original positions); the keys and
        # values that the cache stands for are wanted too, for the prompt's attention.
        {"name": "append-prefill-13b-4bit", "kind": "append", "tokens": 32 * 704, "seqs": 32, "H": 40, "Hkv": 40,
         "dh": 128, "page": 16, "dtype": "fp16", "bits": 4, "rot": 128, "interleaved": False, "rows": True},
        # One interactive request: a pruned image and its text, 13B decoder.
        {"name": "attend-one-short-8bit", "kind": "attend", "seqs": 1, "longest": 704, "fill": "even", "H": 40,
         "Hkv": 40, "dh": 128, "page": 16, "dtype": "fp16", "bits": 8},
        # One long conversation with grouped heads.
        {"name": "attend-one-long-4bit", "kind": "attend", "seqs": 1, "longest": 32011, "fill": "even", "H": 32,
         "Hkv": 8, "dh": 128, "page": 64, "dtype": "bf16", "bits": 4},
        # 24 requests of unequal length decoded together on the 13B decoder.
        {"name": "attend-batch-24-8bit", "kind": "attend", "seqs": 24, "longest": 2048, "fill": "ragged", "H": 40,
         "Hkv": 40, "dh": 128, "page": 16, "dtype": "fp16", "bits": 8},
        # A loaded server: 128 conversations of very unequal length, grouped heads.
        {"name": "attend-batch-128-4bit", "kind": "attend", "seqs": 128, "longest": 8190, "fill": "skewed", "H": 32,
         "Hkv": 8, "dh": 128, "page": 16, "dtype": "bf16", "bits": 4},
        # A decoder layer's decode step as a model makes it: append, then
        # attention over what the cache holds now.
        {"name": "step-batch-16-4bit", "kind": "step", "seqs": 16, "longest": 768, "fill": "ragged", "H": 32,
         "Hkv": 32, "dh": 128, "page": 16, "dtype": "fp16", "bits": 4},
        # Sixteen questions about one pruned LLaVA-NeXT image on the 13B decoder.
        {"name": "prefix-image-16", "kind": "prefix", "seqs": 16, "groups": 1, "prefix": 661, "longest": 96,
         "fill": "ragged", "H": 40, "Hkv": 40, "dh": 128, "page": 16, "dtype": "fp16"},
        # Five documents of several thousand tokens with 96 readers between them, unequally.
        {"name": "prefix-documents-5", "kind": "prefix", "seqs": 96, "groups": 5, "prefix": 6007, "longest": 300,
         "fill": "skewed", "H": 24, "Hkv": 2, "dh": 64, "page": 32, "dtype": "fp16"},
        # 64 conversations behind one long system prompt, grouped heads.
        {"name": "prefix-prompt-64", "kind": "prefix", "seqs": 64, "groups": 1, "prefix": 4093, "longest": 512,
         "fill": "ragged", "H": 32, "Hkv": 8, "dh": 128, "page": 64, "dtype": "bf16"},
        # 32 samples of one answer to a very long context, a head of keys for each of queries.
        {"name": "prefix-long-32", "kind": "prefix", "seqs": 32, "groups": 1, "prefix": 16384, "longest": 700,
         "fill": "even", "H": 32, "Hkv": 32, "dh": 128, "page": 16, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "append", "attend", "attend", "attend", "step", "prefix", "prefix", "prefix"))
    heads = rng.choice(((32, 32), (40, 40), (32, 8), (40, 8), (28, 4), (24, 2), (8, 1)))
    form = {"H": heads[0], "Hkv": heads[1], "dh": rng.choice((128, 128, 64)), "page": rng.choice((8, 16, 32, 64, 256)),
            "dtype": rng.choice(("fp16", "bf16"))}
    if kind == "append":
        tokens = _log_int(rng, 1, 32 * 704)
        rot = rng.choice((form["dh"], form["dh"], form["dh"] // 2))
        return {"kind": kind, "tokens": tokens, "seqs": min(tokens, _log_int(rng, 1, 128)), **form,
                "bits": rng.choice((4, 8)), "rot": rot, "interleaved": rng.random() < 0.3, "rows": rng.random() < 0.5}
    fill = rng.choice(("even", "ragged", "skewed"))
    if kind in ("attend", "step"):
        longest = _log_int(rng, 1, 40000)
        # at most as many keys as the largest listed case reads
        most = int(1.0e9 / (4 * longest * heads[1] * form["dh"]))
        return {"kind": kind, "seqs": max(1, min(most, _log_int(rng, 1, 192))), "longest": longest, "fill": fill,
                **form, "bits": rng.choice((4, 8))}
    prefix, longest = _log_int(rng, 1, 30000), _log_int(rng, 1, 1000)
    # no more than the largest listed case: of keys for the sequences one by one
    most = int(32 * 17000 * 32 * 128 / ((prefix + longest) * heads[1] * form["dh"]))
    seqs = max(1, min(most, _log_int(rng, 1, 160)))
    return {"kind": kind, "seqs": seqs, "groups": min(seqs, rng.choice((1, 1, 2, 5, 12))), "prefix": prefix,
            "longest": longest, "fill": fill, **form}


# ---------------------------------------------------------------- inputs
_TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _spread(n, longest, fill):
    """Positions per sequence: the first has the longest, the others are spread evenly, or most of them short."""
    power = {"even": 0, "ragged": 1, "skewed": 3}[fill]
    return [longest] + [min(longest, max(1, int(longest * ((i + 0.5) / (n - 1)) ** power))) for i in range(n - 1)]


def _members(case):
    """Sequences per group: the first groups have the most."""
    n, k = case["seqs"], case["groups"]
    share = [(k - i) ** 2 for i in range(k)]
    got = [max(1, n * s // sum(share)) for s in share]
    for i in range(k):  # what rounding left over, or gave too much
        got[i] = max(1, got[i] + n - sum(got))
    return got


def _prefixes(case):
    """Shared positions of each group: the first has the longest."""
    return [max(1, case["prefix"] * (i + 1) // case["groups"]) for i in range(case["groups"])][::-1]


def _pages(g, need, cols):
    """A page table [sequences, cols] of shuffled pages (-1 past need[b] of them), and their number."""
    n = need.numel()
    have = torch.arange(cols, device="cuda")[None, :] < need[:, None]
    order = torch.randperm(n * cols, generator=g, device="cuda").view(n, cols)
    # the pages in use, numbered by a random order: pages of one sequence lie apart
    rank = torch.argsort(torch.argsort(torch.where(have, order, order + n * cols).reshape(-1))).view(n, cols)
    return torch.where(have, rank, -1).to(torch.int32), int(need.sum())


def _codes(g, pages, case):
    """Keys (or values) of a cache in use: codes [pages, page, Hkv, dh or dh / 2 bytes] and their scales."""
    page, hk, dh = case["page"], case["Hkv"], case["dh"]
    if case["bits"] == 8:
        c = torch.randint(-127, 128, (pages, page, hk, dh), generator=g, device="cuda", dtype=torch.int8)
    else:
        c = torch.randint(-7, 8, (pages, page, hk, dh), generator=g, device="cuda", dtype=torch.int8)
        c = ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8)
    top = 1.5 + 2.0 * torch.rand((pages, hk, page), generator=g, device="cuda")
    return c, (top / (127.0 if case["bits"] == 8 else 7.0)).transpose(1, 2)


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
    h, hk, dh, page = case["H"], case["Hkv"], case["dh"], case["page"]
    dt = _TYPES[case["dtype"]]
    s = {"case": case, "kind": kind}
    if kind == "append":
        n, t = case["seqs"], case["tokens"]
        if t == n:  # a decode step: one token each, at the end of what the cache holds
            lens = 1 + torch.randperm(n, generator=g, device="cuda") * 704 // n
            pos, seq = lens - 1, None
        else:  # a packed prefill: the tokens of sequence after sequence
            lens = torch.full((n,), t // n, device="cuda", dtype=torch.long)
            lens[:t % n] += 1
            seq = torch.repeat_interleave(torch.arange(n, device="cuda"), lens)
            pos = torch.arange(t, device="cuda") - (torch.cumsum(lens, 0) - lens)[seq]
        longest = int(lens.max())
        s["seq"] = None if seq is None else seq.to(torch.int32)
        s["pos"] = pos.to(torch.int32)
        # pruned sequences keep their tokens' original positions, which rise faster
        s["rot_pos"] = (pos * 4 + torch.randint(0, 4, (t,), generator=g, device="cuda")).to(torch.int32)
        s["cos"], s["sin"] = _rope_tables(4 * longest, case["rot"])
        s["table"], pages = _pages(g, (lens + page - 1) // page, (longest + page - 1) // page)
        s["q"], s["k"], s["v"] = _fused_rows(g, t, case)
        s["q_out"] = torch.empty((t, h * dh), dtype=dt, device="cuda")
        for name in ("k_out", "v_out"):
            s[name] = torch.empty((t, hk * dh), dtype=dt, device="cuda") if case["rows"] else None
    else:
        n = case["seqs"]
        own_lens = torch.tensor(_spread(n, case["longest"], case["fill"]), device="cuda")
        own_lens = own_lens[torch.randperm(n, generator=g, device="cuda")]
        lens, longest = own_lens, case["longest"]
        if kind == "prefix":
            members = torch.tensor(_members(case), device="cuda")
            prefix = torch.tensor(_prefixes(case), device="cuda")
            starts = torch.cumsum(members, 0) - members
            group = torch.repeat_interleave(torch.arange(case["groups"], device="cuda"), members)
            lens, longest = own_lens + prefix[group], case["longest"] + case["prefix"]
            cols = (longest + page - 1) // page
            # every sequence's own pages, then the pages that lie whole within the prefix from the group's first one
            shared = (prefix // page)[group]
            first = starts[group] == torch.arange(n, device="cuda")
            need = (lens + page - 1) // page
            own_pages, pages = _pages(g, torch.where(first, need, need - shared), cols)
            at = torch.arange(cols, device="cuda")[None, :]
            back = torch.where(first, torch.zeros_like(shared), shared)[:, None]
            mine = own_pages.gather(1, (at - back).clamp(min=0))
            s["table"] = torch.where(at < back, mine[starts[group]], mine).contiguous()
            s["group_start"] = torch.cat((starts, starts.new_tensor([n]))).to(torch.int32)
            s["prefix_lens"] = prefix.to(torch.int32)
            units = hk * (case["groups"] + n * (h // hk) // 128 + 1)
            s["scratch"] = torch.empty(((32 << 20) + (256 + units) * 128 * (dh + 4) * 4,), dtype=torch.uint8, device="cuda")
        else:
            s["table"], pages = _pages(g, (lens + page - 1) // page, (longest + page - 1) // page)
            s["scratch"] = torch.empty((24 << 20,), dtype=torch.uint8, device="cuda")
        s["lens"] = lens.to(torch.int32)
        s["q"], s["k"], s["v"] = _fused_rows(g, n, case)
        s["out"] = torch.empty((n, h * dh), dtype=dt, device="cuda")
        s["lse"] = torch.empty((n, h), dtype=torch.float32, device="cuda")
        if kind == "step":
            s["pos"] = (lens - 1).to(torch.int32)
            s["cos"], s["sin"] = _rope_tables(longest, dh)
            s["q_out"] = torch.empty((n, h * dh), dtype=dt, device="cuda")
    if kind == "prefix":
        s["k_cache"], s["v_cache"] = (_randn(g, (pages, page, hk, dh), dt) for _ in range(2))
    else:
        (s["k_cache"], s["k_scale"]), (s["v_cache"], s["v_scale"]) = (_codes(g, pages, case) for _ in range(2))
    return s


# ---------------------------------------------------------------- a pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _cache(s):
    return {name: s[name] for name in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _run_own(s):
    from paper_2609_34867_gb300 import p4q

    kind, case = s["kind"], s["case"]
    if kind == "prefix":
        p4q.p4q_prefix_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["group_start"],
                                 s["prefix_lens"], s["out"], s["scratch"], lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    cache = s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"]
    if kind == "append":
        p4q.p4q_rope_append_quant(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["pos"], *cache, s["q_out"],
                                  k_out=s["k_out"], v_out=s["v_out"], seq=s["seq"], rot_pos=s["rot_pos"],
                                  interleaved=case["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"], **_cache(s)}
    q = s["q"]
    if kind == "step":
        p4q.p4q_rope_append_quant(q, s["k"], s["v"], s["cos"], s["sin"], s["pos"], *cache, s["q_out"])
        q = s["q_out"]
    p4q.p4q_paged_attention_quant(q, *cache, s["lens"], s["out"], s["scratch"], lse=s["lse"])
    if kind == "step":
        return {"out": s["out"], "lse": s["lse"], **_cache(s)}
    return {"out": s["out"], "lse": s["lse"]}


def _run_plain(s):
    kind, case = s["kind"], s["case"]
    if kind == "append":
        return _append_plain(s, s["rot_pos"], case["rot"], case["interleaved"])
    if kind == "step":
        r = _append_plain(s, s["pos"], case["dh"], False)
        return {**_attend_plain(s, r["q"]), **_cache(s)}
    return _attend_plain(s, s["q"])


def _rotate_plain(x, cos, sin, rot, interleaved):
    """x [T, heads, dh] fp32, cos and sin [T, rot / 2] -> the rotated rows, each operation rounded to fp32."""
    a, rest = x[..., :rot], x[..., rot:]
    c, d = cos[:, None, :], sin[:, None, :]
    if interleaved:
        lo, hi = a[..., 0::2], a[..., 1::2]
        r = torch.stack((lo * c - hi * d, hi * c + lo * d), dim=-1).flatten(-2)
    else:
        lo, hi = a[..., :rot // 2], a[..., rot // 2:]
        r = torch.cat((lo * c - hi * d, hi * c + lo * d), dim=-1)
    return torch.cat((r, rest), dim=-1)


def _quantise_plain(x, bits):
    """x [T, heads, dh] fp32 -> whole codes as fp32, and one scale per head: the largest magnitude over 127 or 7."""
    most = 127.0 if bits == 8 else 7.0
    scale = x.abs().amax(-1) / torch.full((1, 1), most, device="cuda")
    code = torch.round(x / torch.where(scale > 0, scale, 1.0)[..., None]).clamp(-most, most)
    return code, scale


def _append_plain(s, rot_pos, rot, interleaved):
    case = s["case"]
    h, hk, dh, page = case["H"], case["Hkv"], case["dh"], case["page"]
    t, dt = s["q"].shape[0], s["q"].dtype
    at = rot_pos.long()
    cos, sin = s["cos"][at], s["sin"][at]
    q = _rotate_plain(s["q"].float().view(t, h, dh), cos, sin, rot, interleaved).to(dt)
    k = _rotate_plain(s["k"].float().view(t, hk, dh), cos, sin, rot, interleaved).to(dt).float()
    pos = s["pos"].long()
    seq = torch.arange(t, device="cuda") if s.get("seq") is None else s["seq"].long()
    where = s["table"].long()[seq, pos // page], pos % page
    back = []
    for x, cache, scales in ((k, "k_cache", "k_scale"), (s["v"].float().view(t, hk, dh), "v_cache", "v_scale")):
        code, scale = _quantise_plain(x, case["bits"])
        c = code.to(torch.int8)
        if case["bits"] == 4:
            c = ((c[..., 0::2] & 15) | (c[..., 1::2] << 4)).view(torch.uint8)
        s[cache][where] = c
        s[scales][where] = scale
        back.append((code * scale[..., None]).to(dt).view(t, hk * dh) if s.get("k_out") is not None else None)
    return {"q": q.view(t, h * dh), "k": back[0], "v": back[1], **_cache(s)}


def _values_plain(codes, scales, at, bits):
    """The values that the positions of pages at [n, columns] stand for, [n, positions, Hkv, dh] fp32."""
    c = codes[at].flatten(1, 2)
    if bits == 4:
        c = c.view(torch.int8)
        c = torch.stack(((c << 4) >> 4, c >> 4), dim=-1).flatten(-2)
    return c.float() * scales[at].flatten(1, 2)[..., None]


def _attend_plain(s, q):
    case = s["case"]
    n, h, hk, dh = case["seqs"], case["H"], case["Hkv"], case["dh"]
    at = s["table"].long()
    if s["kind"] == "prefix":
        page = case["page"]
        members = (s["group_start"][1:] - s["group_start"][:-1]).long()
        group = torch.repeat_interleave(torch.arange(case["groups"], device="cuda"), members, output_size=n)
        j = torch.arange(at.shape[1] * page, device="cuda")
        # a position of the prefix lies where the first sequence of the group has it
        row = torch.where(j[None, :] < s["prefix_lens"].long()[group][:, None], s["group_start"].long()[group][:, None],
                          torch.arange(n, device="cuda")[:, None])
        where = at[row, j // page].clamp(min=0), (j % page)[None, :]
        k, v = s["k_cache"][where].float(), s["v_cache"][where].float()
    else:
        at = at.clamp(min=0)
        k = _values_plain(s["k_cache"], s["k_scale"], at, case["bits"])
        v = _values_plain(s["v_cache"], s["v_scale"], at, case["bits"])
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


# ---------------------------------------------------------------- the work and the exact results
def work(case):
    kind, h, hk, dh = case["kind"], case["H"], case["Hkv"], case["dh"]
    if kind == "prefix":
        n = case["seqs"]
        mine, shared = sum(_spread(n, case["longest"], case["fill"])), _prefixes(case)
        seen = mine + sum(m * p for m, p in zip(_members(case), shared))
        keys = mine + sum(shared)
        return {"bytes": 4 * keys * hk * dh + 4 * n * h * dh + 4 * n * h + 4 * keys / case["page"], "flops": 4 * seen * h * dh}
    held = 2 * hk * (dh * case["bits"] / 8 + 4)  # a position's keys and values
    if kind == "append":
        t = case["tokens"]
        moved = (2 * h + 2 * hk + (2 * hk if case["rows"] else 0)) * dh * 2
        return {"bytes": t * (moved + held + case["rot"] * 4 + 16), "flops": 3 * t * (h + hk) * case["rot"] + 6 * t * hk * dh}
    n = case["seqs"]
    keys = sum(_spread(n, case["longest"], case["fill"]))
    w = {"bytes": keys * held + 4 * n * h * dh + 4 * n * h + 4 * keys / case["page"], "flops": 4 * keys * h * dh}
    if kind == "step":
        w["bytes"] += n * (2 * (h + 2 * hk) * dh + held + dh * 4)
    return w


def exact(case, seed):
    s = prepare(case, seed)
    kind, h, hk, dh, page = case["kind"], case["H"], case["Hkv"], case["dh"], case["page"]
    q = s["q"].double()
    most = 127 if case.get("bits") == 8 else 7
    if kind == "prefix":
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
    else:
        kc, vc = (_exact_values(s[c], s[c[0] + "_scale"], case["bits"]) for c in ("k_cache", "v_cache"))
        scales = {name: s[name].double() for name in ("k_scale", "v_scale")}
    if kind in ("append", "step"):
        t = q.shape[0]
        at = (s["rot_pos"] if kind == "append" else s["pos"]).long()
        rot = case["rot"] if kind == "append" else dh
        inter = kind == "append" and case["interleaved"]
        i = torch.arange(rot // 2, device="cuda")
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + rot // 2)
        c, d = s["cos"].double()[at][:, None, :], s["sin"].double()[at][:, None, :]

        def fl(x):  # the operator's roundings to 32 bits, of products and sums made in 64
            return x.float().double()

        def turned(x, heads):
            x = x.double().reshape(t, heads, dh)
            y = x.clone()
            y[..., a] = fl(fl(x[..., a] * c) - fl(x[..., b] * d))
            y[..., b] = fl(fl(x[..., b] * c) + fl(x[..., a] * d))
            return y

        def held(x):
            """The values that the cache has of rows x, and their scales."""
            scale = fl(x.abs().amax(-1) / most)
            code = torch.round(fl(x / scale.clamp(min=1e-300)[..., None])).clamp(-most, most)
            return code * scale[..., None], scale

        q_turned = turned(s["q"], h).reshape(t, h * dh)
        q = q_turned.to(s["q"].dtype).double()
        seq = torch.arange(t, device="cuda") if s.get("seq") is None else s["seq"].long()
        pos = s["pos"].long()
        slot = s["table"].long()[seq, torch.div(pos, page, rounding_mode="floor")] * page + pos % page
        rows = {}
        for name, x, cache in (("k", turned(s["k"], hk).to(s["q"].dtype).double(), kc),
                               ("v", s["v"].double().reshape(t, hk, dh), vc)):
            values, scale = held(x)
            cache.view(-1, hk, dh)[slot] = values
            scales[name + "_scale"][torch.div(slot, page, rounding_mode="floor"), slot % page] = scale
            rows[name] = values.reshape(t, hk * dh) if case.get("rows") else None
        if kind == "append":
            return {"q": q_turned, **rows, "k_cache": None, "v_cache": None, **scales}
    lens = s["lens"].tolist()
    first, shared = list(range(case["seqs"])), [0] * case["seqs"]
    if kind == "prefix":
        start = s["group_start"].tolist()
        for g, p in enumerate(s["prefix_lens"].tolist()):
            for n in range(start[g], start[g + 1]):
                first[n], shared[n] = start[g], p
    out, lse = [], []
    for n, length in enumerate(lens):
        j = torch.arange(length, device="cuda")
        row = torch.where(j < shared[n], first[n], n)
        slot = s["table"].long()[row, torch.div(j, page, rounding_mode="floor")] * page + j % page
        k, v = (c.view(-1, hk, dh)[slot] for c in (kc, vc))
        qn = q[n].view(hk, h // hk, dh)
        scores = torch.matmul(qn, k.permute(1, 2, 0)) / math.sqrt(dh)  # [hk, heads of the group, length]
        out.append(torch.matmul(torch.softmax(scores, -1), v.transpose(0, 1)).reshape(h * dh))
        lse.append(torch.logsumexp(scores, -1).reshape(h))
    r = {"out": torch.stack(out), "lse": torch.stack(lse)}
    if kind == "step":
        r.update({"k_cache": None, "v_cache": None, **scales})
    return r


def _exact_values(codes, scales, bits):
    """Codes and scales -> values in 64 bits (4 bits: the even dimension in a byte's low half, two's complement)."""
    if bits == 4:
        b = codes.to(torch.int16)
        nibble = torch.stack((b % 16, torch.div(b, 16, rounding_mode="floor")), dim=-1).flatten(-2)
        codes = torch.where(nibble > 7, nibble - 16, nibble)
    return codes.double() * scales.double()[..., None]
