"""Text generation on pruned images: the whole path of an answer, small.

  python -m paper_2609_34867_gb300.generate [--images B] [--new T] [--layers L] [--top-p P] [--seed S]

The selector prunes each image's visual tokens and appends the question's text
rows (p4q_select_gather_quant); a decoder of random W4A4 weights prefills that
sequence (rotary positions of the kept tokens' original places, keys and values
into a paged cache, causal attention) and then answers token by token: per layer
one rotary append and one paged attention between its four linears, at the end
one draw from the logits. The decode step is captured once as a CUDA graph and
replayed. Weights and inputs are synthetic (workloads.py), so the tokens mean
nothing; the calls are those of a real decoder.
"""
from __future__ import annotations

import argparse
import dataclasses
import time

import torch

from . import p4q
from . import workloads as wl

EPS = 1e-5


@dataclasses.dataclass(frozen=True)
class Config:
    d: int = 1024
    heads: int = 8
    kv_heads: int = 4
    ffn: int = 2816
    layers: int = 2
    vocab: int = 4000
    page: int = 16

    @property
    def qkv(self) -> int:
        return (self.heads + 2 * self.kv_heads) * 128


def _weight(g, n, k):
    return p4q.quant_weight((torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).half())


class Decoder:
    """A decoder with random weights: W4A4 linears, FP16 norms, keys and values."""

    def __init__(self, c: Config, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.c = c
        self.layers = [{"qkv": _weight(g, c.qkv, c.d), "o": _weight(g, c.d, c.heads * 128),
                        "gate_up": _weight(g, 2 * c.ffn, c.d), "down": _weight(g, c.d, c.ffn),
                        "norm1": torch.ones((c.d,), dtype=torch.float16, device="cuda"),
                        "norm2": torch.ones((c.d,), dtype=torch.float16, device="cuda")} for _ in range(c.layers)]
        self.norm = torch.ones((c.d,), dtype=torch.float16, device="cuda")
        self.head = _weight(g, c.vocab, c.d)
        self.embedding = torch.randn((c.vocab, c.d), generator=g, device="cuda").half()

    def rope(self, positions: int):
        inv = 10000.0 ** (-torch.arange(0, 128, 2, device="cuda", dtype=torch.float64) / 128)
        a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
        return a.cos().float(), a.sin().float()

    def _linear(self, codes, w):
        y = torch.empty((codes[0].shape[0], w[0].shape[0]), dtype=torch.float16, device="cuda")
        p4q.p4q_w4a4_linear(codes[0], codes[1], w[0], w[1], y)
        return y

    def _norm_codes(self, x, w):
        q = torch.empty((x.shape[0], x.shape[1] // 2), dtype=torch.uint8, device="cuda")
        s = torch.empty((x.shape[0],), dtype=torch.float32, device="cuda")
        p4q.p4q_rmsnorm_quant_expanded(x, w, EPS, q, s)
        return q, s

    def forward(self, x, cache, attend, pos, seq=None, rot_pos=None):
        """x [rows, d] fp16 -> the last layer's rows. attend(layer, q, k, v) gives the attention's rows."""
        c = self.c
        for n, w in enumerate(self.layers):
            y = self._linear(self._norm_codes(x, w["norm1"]), w["qkv"])
            q, k, v = y[:, :c.heads * 128], y[:, c.heads * 128:(c.heads + c.kv_heads) * 128], y[:, (c.heads + c.kv_heads) * 128:]
            # rotated in place; keys and values into the cache
            p4q.p4q_rope_append(q, k, v, cache.cos, cache.sin, pos, cache.k[n], cache.v[n], cache.table, q, k_out=k,
                                seq=seq, rot_pos=rot_pos)
            x = x + self._linear(p4q.quant_act(attend(n, q, k, v)), w["o"])
            y = self._linear(self._norm_codes(x, w["norm2"]), w["gate_up"])
            codes = (torch.empty((x.shape[0], c.ffn // 2), dtype=torch.uint8, device="cuda"),
                     torch.empty((x.shape[0],), dtype=torch.float32, device="cuda"))
            p4q.p4q_swiglu_quant_expanded(y[:, :c.ffn], y[:, c.ffn:], *codes)
            x = x + self._linear(codes, w["down"])
        return x

    def logits(self, x):
        return self._linear(self._norm_codes(x, self.norm), self.head)


class Cache:
    """Paged keys and values of every layer for `seqs` sequences of up to `most` positions."""

    def __init__(self, decoder: Decoder, seqs: int, most: int, positions: int, seed: int = 0):
        c = decoder.c
        per = (most + c.page - 1) // c.page
        pages = seqs * per
        g = torch.Generator(device="cuda").manual_seed(seed)
        # pages in no order, as a running server's free list leaves them
        self.table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(seqs, per)
        shape = (c.layers, pages, c.page, c.kv_heads, 128)
        self.k, self.v = (torch.zeros(shape, dtype=torch.float16, device="cuda") for _ in range(2))
        self.lens = torch.zeros((seqs,), dtype=torch.int32, device="cuda")
        self.cos, self.sin = decoder.rope(positions)
        self.workspace = p4q.paged_attention_workspace("cuda")


def prefill(decoder: Decoder, cache: Cache, x, rot_pos):
    """x [B, S, d] fp16, rot_pos [B, S] int32 -> the last rows' logits."""
    c, (B, S, d) = decoder.c, x.shape
    seq = torch.arange(B, dtype=torch.int32, device="cuda").repeat_interleave(S)
    pos = torch.arange(S, dtype=torch.int32, device="cuda").repeat(B)

    def attend(_, q, k, v):
        o = torch.empty((B * S, c.heads * 128), dtype=torch.float16, device="cuda")
        p4q.p4q_causal_attention(q, k, v, o, B, S, c.heads, c.kv_heads)
        return o

    y = decoder.forward(x.reshape(B * S, d), cache, attend, pos, seq, rot_pos.reshape(-1))
    cache.lens.fill_(S)
    return decoder.logits(y.view(B, S, d)[:, -1].contiguous())


def decode(decoder: Decoder, cache: Cache, token, rot_pos):
    """One token per sequence (int32) at rotary positions rot_pos [B] -> the next logits."""
    c = decoder.c
    cache.lens.add_(1)

    def attend(n, q, k, v):
        o = torch.empty(q.shape, dtype=torch.float16, device="cuda")
        p4q.p4q_paged_attention(q, cache.k[n], cache.v[n], cache.table, cache.lens, o, cache.workspace)
        return o

    y = decoder.forward(decoder.embedding[token.long()], cache, attend, cache.lens - 1, rot_pos=rot_pos)
    return decoder.logits(y)


def pruned_prompt(images: int, c: Config, seed: int, N: int = 192, K: int = 64, T: int = 16):
    """Pruned synthetic images with text: rows [B, K + T, d] and their original positions."""
    w = wl.Workload("generate", B=images, N=N, d=c.d, K=K, T=T, J=3, seed=seed, heavy_tail=False, linears=())
    x = wl.selector_inputs(w)
    up = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    idx, rows, _, _ = p4q.select_gather_quant(up(x.V), up(x.Q), up(x.A), up(x.text), K)
    text = torch.arange(N, N + T, dtype=torch.int32, device="cuda").expand(images, T)
    return rows, torch.cat((idx, text), dim=1).contiguous(), N + T


def generate(decoder: Decoder, rows, rot_pos, end: int, new: int, u, graph: bool = True, **params):
    """Answers of `new` tokens [B, new] to prompts rows [B, S, d] whose rotary
    positions end before `end`; u [new, B] uniform numbers; params: p4q.sample's.
    Also the seconds of the decode steps, and the cache."""
    B, S, _ = rows.shape
    cache = Cache(decoder, B, S + new, end + new)
    tokens = torch.empty((new, B), dtype=torch.int32, device="cuda")
    tokens[0], _ = p4q.sample(prefill(decoder, cache, rows, rot_pos), u[0], **params)
    token, at = tokens[0].clone(), torch.full((B,), end, dtype=torch.int32, device="cuda")
    draw, logits = u[0].clone(), None

    def step():
        nonlocal logits
        logits = decode(decoder, cache, token, at)
        p4q.p4q_sample(logits, draw, token, **params)
        at.add_(1)

    replay = step
    if graph and new > 1:
        saved = cache.lens.clone(), at.clone(), token.clone()
        step()  # (sets what launches need once; its appended rows are written again)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        for t, s in zip((cache.lens, at, token), saved):
            t.copy_(s)
        with torch.cuda.graph(g):
            step()
        replay = g.replay
    torch.cuda.synchronize()
    began = time.perf_counter()
    for n in range(1, new):
        draw.copy_(u[n])
        replay()
        tokens[n].copy_(token)
    torch.cuda.synchronize()
    return tokens.t().contiguous(), time.perf_counter() - began, cache


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--images", type=int, default=4)
    ap.add_argument("--new", type=int, default=32)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--top-p", type=float, default=0.9)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    c = Config(layers=a.layers)
    decoder = Decoder(c, a.seed)
    rows, rot_pos, end = pruned_prompt(a.images, c, a.seed)
    g = torch.Generator(device="cuda").manual_seed(a.seed)
    u = torch.rand((a.new, a.images), generator=g, device="cuda")
    top_p = torch.full((a.images,), a.top_p, device="cuda")
    tokens, seconds, _ = generate(decoder, rows, rot_pos, end, a.new, u, top_p=top_p)
    status = p4q.p4q_device_status()
    if status != p4q.P4Q_OK:
        raise p4q.P4QError(status, "generate")
    for b in range(a.images):
        print(f"image {b}: {' '.join(str(t) for t in tokens[b].tolist())}")
    if a.new > 1:
        print(f"{1e6 * seconds / (a.new - 1):.1f} us per decode step of {a.images} sequences, {c.layers} layers")
    return 0


if __name__ == "__main__":
    raise SystemExit(main())
