"""Generation with scales that are measured while the model runs: linear layers
on activations quantized token by token, a key/value cache in 8 bits with a
scale for each block of tokens and head, and the adjustments of logits before
a token is drawn, as cases that can be timed and compared.

* linear: every token's activations become 8-bit codes by their own largest
  magnitude, s = max |x| / 127; the product with 8- or 4-bit weights (a scale
  and, for asymmetric ones, a zero-point per channel) is exact in integers and
  leaves as ((acc * w_scale) * s) + bias.
* append: queries and keys are rotated by their position's angles; keys and
  values go to the pages that the sequence's page list names as 8-bit codes of
  their block's scale, max |x| / 127 over the block's tokens of the head.  A
  block that already holds tokens keeps its scale or gets a larger one, and
  then its codes are rounded anew.
* attend: softmax attention of the new tokens' queries over these caches,
  causal, or over a sliding window and a few first positions.
* adjust: penalties for the words that a sequence holds already, biases, and
  a bit mask of the words that a grammar allows, where the logits are.

Activations are float32, bfloat16 or float16.  What lies in 8 bits is returned
as the values that it stands for.
"""
import math
import random

import numpy as np
import torch

own = False

# query/key/value heads and head dimension: many heads over a few key/value
# heads of 64; eight heads over one of 256; four heads per key/value head of
# 128; one head per key/value head of 80
HEADS = {"32x4x64": (32, 4, 64), "8x1x256": (8, 1, 256), "32x8x128": (32, 8, 128),
         "12x12x80": (12, 12, 80)}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# the scratch memory that a serving program keeps for its calls
WORKSPACE = 64 << 20
TINY = 2.0 ** -60  # smallest magnitude that a scale is made for


def listed():
    return [
        # one generated token through an up projection: launch latency
        dict(name="linear_1_2048_5632", kind="linear", M=1, K=2048, N=5632, bits=8, asym=False,
             bias=False, type="bf16", out="bf16"),
        # one token's logits over 256000 words: weight bytes count
        dict(name="linear_1_2048_256000", kind="linear", M=1, K=2048, N=256000, bits=8, asym=False,
             bias=False, type="bf16", out="f32"),
        # a serving batch's step through a down projection with 4-bit weights
        dict(name="linear_16_5632_2048_w4", kind="linear", M=16, K=5632, N=2048, bits=4,
             asym=True, bias=False, type="bf16", out="bf16"),
        # a prompt through an up projection: products count
        dict(name="linear_2048_2048_5632", kind="linear", M=2048, K=2048, N=5632, bits=8,
             asym=False, bias=True, type="f16", out="f16"),
        # a serving batch's step, one token for each of 250 young sequences
        dict(name="append_250_seqs", kind="append", heads="8x1x256", B=250, new=1, L=60, page=32,
             block=16, ragged=True, type="bf16"),
        # a batch of prompts entering the cache
        dict(name="append_prompts_5x900", kind="append", heads="32x4x64", B=5, new=900, L=900,
             page=64, block=32, ragged=True, type="f16"),
        # one generated token, 1531 keys: launch latency and a memory round trip
        dict(name="attend_1_over_1531", kind="attend", heads="32x4x64", B=1, new=1, L=1531,
             page=16, block=16, ragged=False, window=0, sinks=0, type="bf16"),
        # two readers of a whole book: few rows, a long axis, cache bytes count
        dict(name="attend_2_over_120000", kind="attend", heads="8x1x256", B=2, new=1, L=120000,
             page=128, block=64, ragged=True, window=0, sinks=0, type="f32"),
        # endless streams over a sliding window and four first tokens, a few
        # drafted tokens each to check
        dict(name="attend_window_1000_of_9000", kind="attend", heads="12x12x80", B=24, new=4,
             L=9000, page=16, block=16, ragged=True, window=1000, sinks=4, type="f16"),
        # a chunk of a long prompt: products and vector arithmetic count
        dict(name="attend_chunk_500_over_16000", kind="attend", heads="32x8x128", B=1, new=500,
             L=16000, page=64, block=32, ragged=False, window=0, sinks=0, type="bf16"),
        # the next token of one long conversation, no grammar
        dict(name="adjust_1_of_256000", kind="adjust", M=1, V=256000, hist=9000, bias=300,
             mask=False, type="f32"),
        # a batch with grammars: mask bits and forbidden words count
        dict(name="adjust_200_of_32000_mask", kind="adjust", M=200, V=32000, hist=1500, bias=20,
             mask=True, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("linear", "append", "attend", "attend", "adjust"))
    dtype = rng.choice(sorted(TYPES))
    if kind == "linear":
        K, N = 32 * _log(rng, 8, 512), _log(rng, 200, 30000)
        M = _log(rng, 1, max(2, min(2048, 20000000000 // (K * N))))
        return dict(kind=kind, M=M, K=K, N=N, bits=rng.choice((8, 8, 4)), asym=rng.random() < 0.5,
                    bias=rng.random() < 0.3, type=dtype, out=rng.choice((dtype, "f32")))
    if kind == "adjust":
        V = _log(rng, 1000, 256000)
        return dict(kind=kind, M=_log(rng, 1, max(2, min(512, 16000000 // V))), V=V,
                    hist=_log(rng, 1, 16000), bias=rng.choice((0, _log(rng, 1, 300))),
                    mask=rng.random() < 0.5, type=dtype)
    heads = rng.choice(sorted(HEADS))
    page = rng.choice((16, 32, 64, 128))
    block = rng.choice([b for b in (16, 32, 64, 128) if b <= page])
    H, G, D = HEADS[heads]
    if kind == "append":
        new = _log(rng, 1, 1000)
        # at most 12 million codes of either cache
        most = max(1, 12000000 // (G * D))
        L = new + rng.randrange(max(1, min(600, most - new)))
        return dict(kind=kind, heads=heads, B=_log(rng, 1, max(2, min(5000 // new, most // L))),
                    new=new, L=L, page=page, block=block, ragged=rng.random() < 0.7, type=dtype)
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log(rng, 20, 4000), rng.randrange(9))
    if rng.random() < 0.6:  # a step of generation
        new, B = rng.randrange(1, 6), _log(rng, 1, 100)
        L = _log(rng, 8, 100000)
    else:  # a chunk of a prompt
        new, B = _log(rng, 16, 700), rng.randrange(1, 4)
        L = new + _log(rng, 1, 40000)
    # at most 100 million query-key pairs and 60 million codes of either cache
    L = max(new, min(L, 100000000 // (B * new * H), 60000000 // (B * G * D)))
    return dict(kind=kind, heads=heads, B=B, new=new, L=L, page=page, block=block,
                ragged=rng.random() < 0.6, window=window, sinks=sinks, type=dtype)


# ---------------------------------------------------------------------------
# Inputs.

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 2 + 1)


def prepare(case, seed):
    g = _generator(seed)
    return {"linear": _prepare_linear, "adjust": _prepare_adjust, "append": _prepare_cache,
            "attend": _prepare_cache}[case["kind"]](case, g)


def _prepare_linear(case, g):
    M, K, N, bits = case["M"], case["K"], case["N"], case["bits"]
    s = dict(kind="linear", M=M, K=K, N=N, bits=bits, out_type=TYPES[case["out"]])
    # activations with a few outlier channels, tokens of different size
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, torch.randint(0, K, (4,), generator=g, device="cuda")] *= 20.0
    x *= 0.5 + torch.rand((M, 1), generator=g, device="cuda")
    s["x"] = x.to(TYPES[case["type"]])
    top = 127 if bits == 8 else 7
    lo = -top - 1 if case["asym"] else -top
    w = torch.empty((N, K), dtype=torch.int8, device="cuda")
    for n in range(0, N, 16384):  # codes of normal weights
        part = torch.randn((min(16384, N - n), K), generator=g, device="cuda")
        w[n:n + 16384] = torch.round(part * (top / 4.0)).clamp_(lo, top).to(torch.int8)
    if bits == 4:  # two a byte, the even channel in the low nibble
        u = w.view(torch.uint8) & 15
        w = u[:, 0::2] | (u[:, 1::2] << 4)
    s["w"] = w.contiguous()
    s["w_scale"] = 0.02 * 4.0 / top * (0.5 + torch.rand(N, generator=g, device="cuda"))
    s["w_zp"] = torch.randint(lo // 8, top // 8 + 1, (N,), generator=g, device="cuda",
                              dtype=torch.int32) if case["asym"] else None
    s["bias"] = torch.randn(N, generator=g, device="cuda") * 0.1 if case["bias"] else None
    s["y"] = torch.empty((M, N), dtype=s["out_type"], device="cuda")
    s["workspace"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


def _batch(case, g):
    """Lengths, first rows and pages of the sequences: the pages of a pool in
    random order, a few of the pool left to others."""
    B, L, new, page = case["B"], case["L"], case["new"], case["page"]
    # the lengths are the case's own, so that its outputs have one shape
    r, ragged = random.Random(L), case["ragged"]
    n_new = [max(1, int(new * r.uniform(0.4, 1.0))) if ragged else new for _ in range(B)]
    lens = [m + int((L - new) * r.random()) if ragged else L for m in n_new]
    if ragged:  # the longest sequence is the case's
        n_new[0], lens[0] = new, L
    # the page list holds as many pages as the longest sequence and one more
    ld = -(-L // page) + 1
    need = [-(-n // page) for n in lens]
    pool = sum(need) + 3
    perm = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    first = torch.tensor([0] + need, device="cuda").cumsum(0)
    at = torch.arange(ld, device="cuda")[None, :]
    have = at < torch.tensor(need, device="cuda")[:, None]
    pages = torch.where(have, perm[(first[:-1, None] + at).clamp(max=pool - 1)], 0).to(torch.int32)
    starts = torch.tensor([0] + n_new, device="cuda").cumsum(0).to(torch.int32)
    s = dict(starts=starts, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             pages=pages.contiguous(), T=sum(n_new), L=L, new=max(n_new), page=page,
             block=case["block"])
    return s, pool


def _normal(g, shape, std):
    """Normal values, the last dimension's first and middle channel larger, as
    keys and queries have them."""
    x = torch.randn(shape, generator=g, device="cuda") * std
    x[..., 0] *= 3.0
    x[..., shape[-1] // 2] *= 2.0
    return x


def _prepare_cache(case, g):
    H, G, D = HEADS[case["heads"]]
    s, pool = _batch(case, g)
    T, page, block = s["T"], s["page"], s["block"]
    t = TYPES[case["type"]]
    s.update(kind=case["kind"], H=H, G=G, D=D)
    # a pool that earlier calls filled: keys [page][D] and values [page / 16][D][16]
    # of every page and head, codes that reach 127 in every block
    for name in ("k", "v"):
        x = _normal(g, (pool, G, page // block, block, D), 1.0)
        scale = x.abs().amax((3, 4)) / 127.0
        c = torch.round(x / scale[..., None, None]).clamp_(-127, 127).to(torch.int8)
        c = c.view(pool, G, page, D)
        if name == "v":
            c = c.view(pool, G, page // 16, 16, D).transpose(3, 4)
        s[name + "_cache"], s[name + "_scale"] = c.contiguous(), scale.contiguous()
    if case["kind"] == "append":
        s["q"] = _normal(g, (T, H, D), 1.3).view(T, H * D).to(t)
        s["k"] = _normal(g, (T, G, D), 1.0).view(T, G * D).to(t)
        s["v"] = torch.randn((T, G * D), generator=g, device="cuda").to(t)
        # cos and sin of pos * 10000^(-2i/D), one row of pairs per position:
        # the layout of the library's angle table
        i = torch.arange(D // 2, dtype=torch.float64, device="cuda")
        ang = torch.arange(case["L"], dtype=torch.float64, device="cuda")[:, None] * \
            torch.pow(10000.0, -2.0 * i / D)[None, :]
        s["table"] = torch.stack((torch.cos(ang), torch.sin(ang)), 2).view(-1)
        s["q_rot"] = torch.empty_like(s["q"])
        return s
    # heads differ in how far their logits spread
    spread = torch.linspace(0.5, 2.0, H, device="cuda")[:, None]
    s["q"] = (torch.randn((T, H, D), generator=g, device="cuda") * 1.2 * spread) \
        .view(T, H * D).to(t)
    s.update(window=case["window"], sinks=case["sinks"], scale=float(np.float32(D ** -0.5)))
    s["ctx"] = torch.empty((T, H * D), dtype=t, device="cuda")
    s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


def _prepare_adjust(case, g):
    M, V, n = case["M"], case["V"], case["hist"]
    s = dict(kind="adjust", M=M, V=V)
    s["logits"] = (torch.randn((M, V), generator=g, device="cuda") * 2.5).to(TYPES[case["type"]])
    # words by their rank, frequent ones again and again; conversations of
    # different lengths, about half of each the prompt
    u = torch.rand((M, n), generator=g, device="cuda", dtype=torch.float64)
    s["history"] = (V * u * u * u).to(torch.int32).clamp_(max=V - 1)
    r = random.Random(n)  # the lengths are the case's own
    lens = [n] + [1 + int(n * r.random()) for _ in range(M - 1)]
    s["hist_lens"] = torch.tensor([min(x, n) for x in lens], dtype=torch.int32, device="cuda")
    s["prompt_lens"] = torch.tensor([int(x * r.uniform(0.2, 0.8)) for x in lens],
                                    dtype=torch.int32, device="cuda")
    s["repetition"] = 1.0 + 0.3 * torch.rand(M, generator=g, device="cuda")
    s["presence"] = torch.rand(M, generator=g, device="cuda")
    s["frequency"] = 0.5 * torch.rand(M, generator=g, device="cuda")
    s["bias"] = s["mask"] = None
    if case["bias"]:
        b = [case["bias"] if m == 0 else r.randrange(case["bias"] + 1) for m in range(M)]
        starts = torch.tensor([0] + b, device="cuda").cumsum(0)
        row = torch.repeat_interleave(torch.arange(M, device="cuda"),
                                      torch.tensor(b, device="cuda"))
        j = torch.arange(int(sum(b)), device="cuda") - starts[row]
        first = torch.randint(0, V, (M,), generator=g, device="cuda")
        s["bias"] = (starts.to(torch.int32), ((first[row] + 3 * j) % V).to(torch.int32),
                     torch.randn(sum(b), generator=g, device="cuda") * 4.0)
    if case["mask"]:
        # a grammar allows a few words, most of them, or (in free text) all
        keep = torch.tensor([0.003, 0.03, 0.97, 2.0], device="cuda")
        keep = keep[torch.randint(0, 4, (M, 1), generator=g, device="cuda")]
        words = -(-V // 32)
        ok = torch.rand((M, words * 32), generator=g, device="cuda") < keep
        bits = ok.view(M, words, 32).to(torch.int64) << torch.arange(32, device="cuda")
        s["mask"] = bits.sum(2).to(torch.int32)
    return s


# ---------------------------------------------------------------------------
# The operators.

def run(s):
    if own:
        out = _run_own(s)
    else:
        out = {"linear": _linear, "append": _append, "attend": _attend, "adjust": _adjust}[
            s["kind"]](s)
    return _values(s) if out is None else out


def _values(s):
    """The updated cache as the values that its codes stand for."""
    n, G, page, D = s["k_cache"].shape
    nb = page // s["block"]
    k = s["k_cache"].view(n, G, nb, -1, D) * s["k_scale"][:, :, :, None, None]
    v = s["v_cache"].view(n, G, nb, -1, D, 16) * s["v_scale"][:, :, :, None, None, None]
    return {"q": s["q_rot"], "k": k, "v": v}


def _run_own(s):
    import paper_2408_13933_amd as mq
    if s["kind"] == "linear":
        return mq.mq_linear_tokens(s["x"], s["w"], s["bits"], s["w_scale"], w_zp=s["w_zp"],
                                   bias=s["bias"], out=s["y"], workspace=s["workspace"])
    if s["kind"] == "append":
        mq.mq_rope_append_blocks(s["q"], s["k"], s["v"], s["k_cache"], s["k_scale"], s["v_cache"],
                                 s["v_scale"], s["starts"], s["lens"], s["pages"],
                                 table=s["table"], out=s["q_rot"])
        return None
    if s["kind"] == "attend":
        return mq.mq_paged_attn_blocks(s["q"], s["k_cache"], s["k_scale"], s["v_cache"],
                                       s["v_scale"], s["starts"], s["lens"], s["pages"],
                                       s["scale"], window=s["window"], sinks=s["sinks"],
                                       max_len=s["L"], out=s["ctx"], workspace=s["workspace"])
    return mq.mq_adjust_logits(s["logits"], history=s["history"], hist_lens=s["hist_lens"],
                               prompt_lens=s["prompt_lens"], repetition=s["repetition"],
                               presence=s["presence"], frequency=s["frequency"], bias=s["bias"],
                               mask=s["mask"])


def _scale(most):
    """The scale of a largest magnitude, max(most, 2^-60) / 127, in 32 bits
    rounded once (a code next to a rounding border must not depend on more)."""
    return (most.double().clamp(min=TINY) / 127.0).float()


def _codes(x, inv):
    return torch.round(x * inv).clamp_(-127, 127)


def _linear(s):
    x = s["x"].float()
    scale = _scale(x.abs().amax(1, keepdim=True))
    c = _codes(x, 1.0 / scale)
    w = s["w"]
    if s["bits"] == 4:
        w = torch.stack((w & 15, w >> 4), 2).view(s["N"], s["K"]).to(torch.int8)
        w = torch.where(w > 7, w - 16, w)
    w = w.float()
    if s["w_zp"] is not None:
        w -= s["w_zp"][:, None]
    # whole numbers: exact in 32 bits while the sums stay below 2^24
    y = torch.matmul(c, w.t()) * s["w_scale"] * scale
    if s["bias"] is not None:
        y += s["bias"]
    return s["y"].copy_(y)


def _rows(s):
    """Sequence and position of every token row."""
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["starts"], t.to(torch.int32), right=True) - 1
    return b, s["lens"][b].long() - s["starts"][b + 1] + t


def _rotate(x, heads, cs):
    """Pairs (i, i + D/2) of every head by the position's angle, in 64 bits:
    a code next to a rounding border must not depend on the type."""
    u = x.double().view(x.shape[0], heads, 2, -1)
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    y = torch.stack((u[:, :, 0] * c - u[:, :, 1] * n, u[:, :, 1] * c + u[:, :, 0] * n), 2)
    return y.view(x.shape[0], heads, -1).float()


def _store(s, x, b, pos, cache, scale):
    """New values x [T][G][D] into a cache [pages][G][page][D] of codes and its
    block scales [pages][G][page / block]."""
    block, page = s["block"], s["page"]
    n, G = scale.shape[0], s["G"]
    at, slot = s["pages"][b, pos // page].long(), pos % page
    nb = page // block
    i = at * nb + slot // block  # the token's block among all
    # [pages * nb][G]: largest new magnitude, first new slot, old and new scale
    most = torch.zeros((n * nb, G), device="cuda")
    most.scatter_reduce_(0, i[:, None].expand(-1, G), x.abs().amax(2), "amax")
    first = torch.full((n * nb,), block, device="cuda", dtype=torch.int64)
    first.scatter_reduce_(0, i, slot % block, "amin")
    before = scale.transpose(1, 2).reshape(n * nb, G)
    old = torch.where((first > 0)[:, None], before, torch.zeros_like(before))
    new = torch.maximum(old, _scale(most))
    # what the block held before its first new slot, by the new scale
    c = cache.view(n, G, nb, block, -1).permute(0, 2, 1, 3, 4).reshape(n * nb, G, block, -1)
    held = torch.arange(block, device="cuda")[None, :] < first[:, None]
    held &= (first < block)[:, None]
    again = torch.round(c.float() * (old / new)[:, :, None, None])
    c = torch.where(held[:, None, :, None], again, c.float())
    c[i, :, slot % block] = _codes(x, (1.0 / new)[i][:, :, None])
    new = torch.where((first < block)[:, None], new, before)
    cache.copy_(c.view(n, nb, G, block, -1).permute(0, 2, 1, 3, 4).reshape_as(cache))
    scale.copy_(new.view(n, nb, G).transpose(1, 2))


def _append(s):
    b, pos = _rows(s)
    cs = s["table"].view(-1, s["D"] // 2, 2)[pos]
    s["q_rot"].copy_(_rotate(s["q"], s["H"], cs).view_as(s["q_rot"]))
    _store(s, _rotate(s["k"], s["G"], cs), b, pos, s["k_cache"], s["k_scale"])
    n, G, page, D = s["k_cache"].shape
    v = s["v_cache"].transpose(3, 4).reshape(n, G, page, D)
    _store(s, s["v"].float().view(-1, G, D), b, pos, v, s["v_scale"])
    s["v_cache"].copy_(v.view(n, G, page // 16, 16, D).transpose(3, 4))


def _attend(s):
    """Padded to the longest sequence, in 32 bits."""
    H, G, D, N, L, page = s["H"], s["G"], s["D"], s["new"], s["L"], s["page"]
    B, T, g = s["lens"].numel(), s["T"], s["H"] // s["G"]
    j = torch.arange(L, device="cuda")
    at, slot = s["pages"][:, j // page].long(), j % page
    ks = s["k_scale"][at, :, slot // s["block"]]         # [B][L][G]
    vs = s["v_scale"][at, :, slot // s["block"]]
    k = s["k_cache"][at, :, slot].float() * ks[..., None]  # [B][L][G][D]
    v = s["v_cache"][at, :, slot // 16, :, slot % 16].float() * vs[..., None]
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    # every sequence's rows in N places, the last of them its last token
    b, pos = _rows(s)
    n = pos - (s["lens"][b].long() - N)
    q = torch.zeros((B, N, G, g, D), device="cuda")
    q[b, n] = s["q"].float().view(T, G, g, D)
    q = q.permute(0, 2, 3, 1, 4).reshape(B, G, g * N, D)
    x = (torch.matmul(q, k) * s["scale"]).view(B, G, g, N, L)
    at_pos = (s["lens"][:, None].long() - N + torch.arange(N, device="cuda"))[:, :, None]
    see = j <= at_pos                                    # [B][N][L]
    if s["window"] > 0:
        see &= (j > at_pos - s["window"]) | (j < s["sinks"])
    x = x.masked_fill(~see[:, None, None], -math.inf)
    # (places before a sequence's first row may see nothing)
    w = torch.exp(x - x.amax(4, keepdim=True).clamp(min=-1e30)).view(B, G, g * N, L)
    o = torch.matmul(w, v) / w.sum(3, keepdim=True)
    o = o.view(B, G, g, N, D).permute(0, 3, 1, 2, 4)[b, n]
    s["ctx"].copy_(o.view(T, H * D))
    return s["ctx"]


def _adjust(s):
    M, V = s["M"], s["V"]
    x = s["logits"].float()
    j = torch.arange(s["history"].shape[1], device="cuda")[None, :]
    has = j < s["hist_lens"][:, None]
    drawn = has & (j >= s["prompt_lens"][:, None])
    # how often a word is there, and how often past the prompt
    words = s["history"].long()
    seen = torch.zeros((M, V), device="cuda").scatter_add_(1, words, has.float())
    count = torch.zeros((M, V), device="cuda").scatter_add_(1, words, drawn.float())
    r = s["repetition"][:, None]
    x = torch.where(seen > 0, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None] * count
    x = torch.where(count > 0, x - s["presence"][:, None], x)
    if s["bias"] is not None:
        starts, at, value = s["bias"]
        row = torch.searchsorted(starts, torch.arange(at.numel(), device="cuda",
                                                      dtype=torch.int32), right=True) - 1
        x[row, at.long()] += value
    if s["mask"] is not None:
        i = torch.arange(V, device="cuda")
        x = x.masked_fill(((s["mask"][:, i >> 5] >> (i & 31)) & 1) == 0, -math.inf)
    return s["logits"].copy_(x)


# ---------------------------------------------------------------------------

_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _mean_lens(case):
    """Expected new tokens and length of a sequence (prepare() draws them)."""
    if not case["ragged"]:
        return float(case["new"]), float(case["L"])
    new = max(1.0, 0.7 * case["new"])
    return new, new + 0.5 * (case["L"] - case["new"])


def work(case):
    e = _BYTES[case["type"]]
    if case["kind"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": float(M * K * e + N * K * case["bits"] // 8 + 8 * N +
                               M * N * _BYTES[case["out"]]),
                "flops": 2.0 * M * K * N}
    if case["kind"] == "adjust":
        M, V, n = case["M"], case["V"], case["hist"] * (0.5 if case["M"] > 1 else 1.0)
        # the conversation; the words in it, read and written (at most half of
        # its length are different ones); mask bits, forbidden words written
        b = 4 * n + 2 * e * min(V, n / 2) + (V / 8 + 0.5 * e * V if case["mask"] else 0.0)
        return {"bytes": M * (b + case["bias"] * (8 + 2 * e)), "flops": M * (4.0 * n + V)}
    H, G, D = HEADS[case["heads"]]
    new, L = _mean_lens(case)
    T = case["B"] * new
    if case["kind"] == "append":
        # queries in and out, keys and values in and out as codes, angles; the
        # cache's codes in and its values out
        pool = case["B"] * (L + case["page"] / 2.0) * G * D
        return {"bytes": T * (2.0 * e * H * D + 2.0 * e * G * D + 2.0 * G * D + 8.0 * D) +
                10.0 * pool, "flops": 5.0 * T * (H + G) * D}
    # keys that some row of the sequence sees, and pairs that a row sees
    seen, pairs = L, new * (L - (new - 1) / 2.0)
    if case["window"] > 0:
        seen = min(L, case["window"] + new - 1 + case["sinks"])
        pairs = min(pairs, new * float(min(L, case["window"] + case["sinks"])))
    return {"bytes": case["B"] * (2.0 * seen * G * (D + 4.0 / case["block"]) +
                                  2.0 * e * new * H * D),
            "flops": 4.0 * case["B"] * pairs * H * D}


# ---------------------------------------------------------------------------
# The same from the definitions, with numpy on the host.  Scales, their
# inverses and the products that are rounded to codes are 32-bit numbers by
# definition, each the nearest to the exact result of its operands; everything
# else is 64-bit.

def exact(case, seed):
    kind = case["kind"]
    if kind == "linear" and case["M"] * case["K"] * case["N"] > 30000000000:
        return None
    if kind == "attend" and \
            case["B"] * case["new"] * HEADS[case["heads"]][0] * case["L"] > 60 << 20:
        return None
    if kind == "adjust" and case["M"] * case["V"] > 24 << 20:
        return None
    h = {}
    for k, v in prepare(case, seed).items():
        if isinstance(v, torch.Tensor):
            v = v.cpu()
            v = (v.float() if v.dtype == torch.bfloat16 else v).numpy()
        h[k] = tuple(x.cpu().numpy() for x in v) if isinstance(v, tuple) else v
    return {"linear": _exact_linear, "append": _exact_append, "attend": _exact_attend,
            "adjust": _exact_adjust}[kind](h)


def _f32(x):
    return np.asarray(x, np.float64).astype(np.float32)


def _np_scale(most):
    return _f32(np.maximum(np.float64(most), TINY) / 127.0).astype(np.float64)


def _np_codes(x, scale):
    inv = _f32(1.0 / scale).astype(np.float64)
    return np.clip(np.rint(_f32(np.asarray(x, np.float64) * inv).astype(np.float64)), -127, 127)


def _exact_linear(h):
    M, N, K = h["M"], h["N"], h["K"]
    c, scale = np.empty((M, K)), np.empty(M)
    for m in range(M):
        scale[m] = _np_scale(np.abs(h["x"][m].astype(np.float64)).max())
        c[m] = _np_codes(h["x"][m], scale[m])
    y = np.empty((M, N))
    for n in range(0, N, 4096):
        w = h["w"][n:n + 4096]
        if h["bits"] == 4:
            both = np.empty((w.shape[0], K), np.int8)
            both[:, 0::2], both[:, 1::2] = (w << 4).astype(np.uint8).view(np.int8) >> 4, \
                w.view(np.int8) >> 4
            w = both
        w = w.astype(np.float64)
        if h["w_zp"] is not None:
            w -= h["w_zp"][n:n + 4096, None]
        y[:, n:n + 4096] = (c @ w.T) * h["w_scale"][n:n + 4096].astype(np.float64)
    y *= scale[:, None]
    return y if h["bias"] is None else y + h["bias"].astype(np.float64)


def _exact_append(h):
    D, G, P, block = h["D"], h["G"], h["page"], h["block"]
    half = D // 2
    n = h["k_cache"].shape[0]
    q = np.empty(h["q"].shape)
    kc = h["k_cache"].astype(np.float64)
    vc = h["v_cache"].astype(np.float64).swapaxes(3, 4).reshape(n, G, P, D)
    ks, vs = h["k_scale"].astype(np.float64), h["v_scale"].astype(np.float64)
    for b in range(len(h["lens"])):
        t0, t1, L = int(h["starts"][b]), int(h["starts"][b + 1]), int(h["lens"][b])
        p0 = L - (t1 - t0)
        ang = h["table"].reshape(-1, half, 2)[p0:L]
        turn = np.empty((t1 - t0, half), np.complex128)
        turn.real, turn.imag = ang[..., 0], ang[..., 1]
        rows = {}
        for name, heads in (("q", h["H"]), ("k", G)):
            x = h[name][t0:t1].astype(np.float64).reshape(t1 - t0, heads, D)
            y = (x[..., :half] + 1j * x[..., half:]) * turn[:, None, :]
            rows[name] = np.concatenate((y.real, y.imag), -1)
        q[t0:t1] = rows["q"].reshape(t1 - t0, -1)
        new = {"k": _f32(rows["k"]), "v": h["v"][t0:t1].reshape(t1 - t0, G, D)}
        for i in range(p0 // block, (L - 1) // block + 1):
            lo, hi = max(p0, i * block), min(L, (i + 1) * block)
            pg, s0 = int(h["pages"][b, i * block // P]), i * block % P
            for g in range(G):
                for name, cache, scales in (("k", kc, ks), ("v", vc, vs)):
                    x = new[name][lo - p0:hi - p0, g].astype(np.float64)
                    s = _np_scale(np.abs(x).max())
                    if lo > i * block:
                        old = scales[pg, g, s0 // block]
                        s = max(s, old)
                        ratio = _f32(old / s).astype(np.float64)
                        part = cache[pg, g, s0:s0 + lo - i * block]
                        part[...] = np.rint(_f32(part * ratio).astype(np.float64))
                    scales[pg, g, s0 // block] = s
                    cache[pg, g, s0 + lo - i * block:s0 + hi - i * block] = _np_codes(x, s)
    nb = P // block
    k = kc.reshape(n, G, nb, block, D) * ks[:, :, :, None, None]
    v = vc.reshape(n, G, P // 16, 16, D).swapaxes(3, 4).reshape(n, G, nb, -1, D, 16)
    return {"q": q, "k": k, "v": v * vs[:, :, :, None, None, None]}


def _exact_attend(h):
    H, G, D, P = h["H"], h["G"], h["D"], h["page"]
    y = np.zeros((h["T"], H, D))
    for b in range(len(h["lens"])):
        L, t0, t1 = int(h["lens"][b]), int(h["starts"][b]), int(h["starts"][b + 1])
        pos = np.arange(L)
        pg, slot = h["pages"][b, pos // P], pos % P
        for hd in range(H):
            g = hd // (H // G)
            k = h["k_cache"][pg, g, slot].astype(np.float64)
            v = h["v_cache"][pg, g, slot // 16, :, slot % 16].astype(np.float64)
            k *= h["k_scale"][pg, g, slot // h["block"]].astype(np.float64)[:, None]
            v *= h["v_scale"][pg, g, slot // h["block"]].astype(np.float64)[:, None]
            x = (h["q"][t0:t1, hd * D:(hd + 1) * D].astype(np.float64) @ k.T) * h["scale"]
            at = np.arange(L - (t1 - t0), L)[:, None]
            sees = pos[None, :] <= at
            if h["window"] > 0:
                sees &= (pos > at - h["window"]) | (pos < h["sinks"])
            x = np.where(sees, x, -np.inf)
            w = np.exp(x - x.max(1, keepdims=True))
            y[t0:t1, hd] = (w @ v) / w.sum(1, keepdims=True)
    return y.reshape(h["T"], H * D)


def _exact_adjust(h):
    x = h["logits"].astype(np.float64)
    f64 = {k: h[k].astype(np.float64) for k in ("repetition", "presence", "frequency")}
    for m in range(h["M"]):
        words = h["history"][m, :h["hist_lens"][m]]
        at = np.unique(words)
        r = f64["repetition"][m]
        x[m, at] = np.where(x[m, at] > 0, x[m, at] / r, x[m, at] * r)
        at, count = np.unique(words[h["prompt_lens"][m]:], return_counts=True)
        x[m, at] -= f64["frequency"][m] * count + f64["presence"][m]
        if h["bias"] is not None:
            lo, hi = h["bias"][0][m], h["bias"][0][m + 1]
            x[m, h["bias"][1][lo:hi]] += h["bias"][2][lo:hi].astype(np.float64)
        if h["mask"] is not None:
            bits = np.unpackbits(h["mask"][m].view(np.uint8), bitorder="little")[:h["V"]]
            x[m, bits == 0] = -np.inf
    return x
