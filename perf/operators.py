"""Text generation over a paged key/value cache: appending rotated keys and
values to its pages, attention of the new tokens over them, and sampling of
the next tokens, as cases that can be timed and compared.

Every operator works on the library's static integer formats: a code c of
format (scale, zp) stands for scale * (c - zp).

* append: the new tokens' query and key codes are rotated by their position's
  angles and requantized (queries to 16 bits, keys to 8), the keys and the
  8-bit value codes go to the pages that the sequence's page list names.
* attend: each query sees the keys at or before its position, all of them or
  those of a sliding window and of a few first positions.  Logits are the exact
  integer products; in each aligned block of 128 key positions the weights are
  integers, rint(32512 exp(logit - the block's largest)), and the blocks are
  joined in 64 bits.  The context is requantized to 16 bits (the input of a
  linear layer on 16-bit activations).
* sample: weights are integers too, rint(2^40 exp((x - max x) / temperature)),
  so that every sum is exact; ties in the order go to the lowest index.

All outputs are whole numbers, the updated pages among them.
"""
import math
import random

import numpy as np
import torch

own = False

# query/key/value heads and head dimension of the decoder blocks used here:
# many heads over a few key/value heads of 64; eight heads over one of 256;
# four heads per key/value head of 128; one head per key/value head of 80
HEADS = {"32x4x64": (32, 4, 64), "8x1x256": (8, 1, 256), "32x8x128": (32, 8, 128),
         "12x12x80": (12, 12, 80)}
# the scratch memory that a serving program keeps for its calls
WORKSPACE = 64 << 20
BLOCK = 128
W_MAX = 32512.0
SAMPLE_ONE = float(1 << 40)


def listed():
    return [
        # one generated token in a chat with 1530 tokens before it: launch latency
        dict(name="append_1_at_1531", kind="append", heads="32x4x64", B=1, new=1, L=1531,
             page=16, ragged=False),
        # a serving batch's step, one token for each of 250 sequences
        dict(name="append_250_seqs", kind="append", heads="8x1x256", B=250, new=1, L=3000,
             page=64, ragged=True),
        # a batch of prompts entering the cache
        dict(name="append_prompts_7x900", kind="append", heads="32x4x64", B=7, new=900, L=900,
             page=32, ragged=True),
        # one generated token, 1531 keys: launch latency and one memory round trip
        dict(name="attend_1_over_1531", kind="attend", heads="32x4x64", B=1, new=1, L=1531,
             page=16, ragged=False, window=0, sinks=0),
        # a serving batch's step over contexts of every length: cache bytes count
        dict(name="attend_64_over_4096", kind="attend", heads="32x4x64", B=64, new=1, L=4096,
             page=32, ragged=True, window=0, sinks=0),
        # two readers of a whole book: few rows, a long axis
        dict(name="attend_2_over_120000", kind="attend", heads="8x1x256", B=2, new=1, L=120000,
             page=128, ragged=True, window=0, sinks=0),
        # the first chunk of a prompt
        dict(name="attend_prompt_1024", kind="attend", heads="32x4x64", B=1, new=1024, L=1024,
             page=64, ragged=False, window=0, sinks=0),
        # a later chunk of a long prompt: vector arithmetic and products count
        dict(name="attend_chunk_500_over_16000", kind="attend", heads="32x8x128", B=1, new=500,
             L=16000, page=64, ragged=False, window=0, sinks=0),
        # endless streams: a sliding window and four first tokens, a few
        # drafted tokens each to check
        dict(name="attend_window_1000_of_9000", kind="attend", heads="12x12x80", B=24, new=4,
             L=9000, page=16, ragged=True, window=1000, sinks=4),
        # the next token of one sequence from a 256000-word vocabulary
        dict(name="sample_1_of_256000", kind="sample", M=1, V=256000, bits=32, mix="topk"),
        # a batch's tokens from 16-bit logit codes over 32000 words
        dict(name="sample_48_of_32000_codes", kind="sample", M=48, V=32000, bits=16,
             mix="nucleus"),
        # every row of a large batch with its own settings: logit bytes count
        dict(name="sample_512_of_256000", kind="sample", M=512, V=256000, bits=32, mix="all"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append", "attend", "attend", "sample"))
    if kind == "sample":
        M = _log(rng, 1, 512)
        return dict(kind=kind, M=M, V=_log(rng, 1000, 256000), bits=rng.choice((32, 16)),
                    mix=rng.choice(("topk", "nucleus", "all", "plain")))
    heads = rng.choice(sorted(HEADS))
    page = rng.choice((16, 32, 64, 128))
    H, G, D = HEADS[heads]
    if kind == "append":
        new = _log(rng, 1, 1000)
        L = new + rng.randrange(3000)
        return dict(kind=kind, heads=heads, B=_log(rng, 1, max(2, min(6000 // new, 300000 // L))),
                    new=new, L=L, page=page, ragged=rng.random() < 0.7)
    window, sinks = (0, 0) if rng.random() < 0.6 else (_log(rng, 20, 4000), rng.randrange(9))
    if rng.random() < 0.6:  # a step of generation
        new, B = rng.randrange(1, 6), _log(rng, 1, 100)
        L = _log(rng, 8, 100000)
    else:  # a chunk of a prompt
        new, B = _log(rng, 16, 700), rng.randrange(1, 4)
        L = new + _log(rng, 1, 40000)
    # at most 100 million query-key pairs and 120 million codes of either cache
    L = max(new, min(L, 100000000 // (B * new * H), 120000000 // (B * G * D)))
    return dict(kind=kind, heads=heads, B=B, new=new, L=L, page=page, ragged=rng.random() < 0.6,
                window=window, sinks=sinks)


# ---------------------------------------------------------------------------
# Inputs.

def _fmt(lo, hi, bits):
    """Static format of a float range (the range widened to hold 0)."""
    lo, hi = min(lo, 0.0), max(hi, 0.0)
    top = 2 ** bits - 1
    a = float(np.float32((hi - lo) / top))
    return a, int(min(max(round(-lo / a), 0), top)) - 2 ** (bits - 1)


# formats before the rotation (queries, keys), after it, of the values, and of
# the context
Q_IN, K_IN = _fmt(-9.0, 10.0, 16), _fmt(-7.5, 8.0, 16)
Q_ROT, K_ROT = _fmt(-11.0, 10.0, 16), _fmt(-8.0, 9.0, 8)
V_FMT, CTX_FMT = _fmt(-4.0, 4.5, 8), _fmt(-3.0, 3.5, 16)


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 2 + 1)


def _codes(g, shape, std, fmt, bits, dtype):
    """Codes of normal values, the last dimension's first and middle channel
    larger, as keys and queries have them."""
    x = torch.randn(shape, generator=g, device="cuda") * std
    x[..., 0] *= 3.0
    x[..., shape[-1] // 2] *= 2.0
    lo = -(1 << (bits - 1))
    return (torch.round(x / fmt[0]) + fmt[1]).clamp_(lo, -lo - 1).to(dtype)


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
    # entries past a sequence's last page are the pool's first page, as a
    # freshly cleared list has them
    first = torch.tensor([0] + need, device="cuda").cumsum(0)
    at = torch.arange(ld, device="cuda")[None, :]
    have = at < torch.tensor(need, device="cuda")[:, None]
    pages = torch.where(have, perm[(first[:-1, None] + at).clamp(max=pool - 1)], 0).to(torch.int32)
    starts = torch.tensor([0] + n_new, device="cuda").cumsum(0).to(torch.int32)
    s = dict(starts=starts, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
             pages=pages.contiguous(), T=sum(n_new), L=L, new=max(n_new), page=page)
    return s, pool


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"] == "sample":
        return _prepare_sample(case, g)
    H, G, D = HEADS[case["heads"]]
    s, pool = _batch(case, g)
    s.update(kind=case["kind"], H=H, G=G, D=D)
    T = s["T"]
    s["k_cache"] = torch.randint(-128, 128, (pool, G, s["page"], D), generator=g, device="cuda",
                                 dtype=torch.int8)
    s["v_cache"] = torch.randint(-128, 128, (pool, G, D, s["page"]), generator=g, device="cuda",
                                 dtype=torch.int8)
    if case["kind"] == "append":
        s["q"] = _codes(g, (T, H, D), 1.3, Q_IN, 16, torch.int16).view(T, H * D)
        s["k"] = _codes(g, (T, G, D), 1.2, K_IN, 16, torch.int16).view(T, G * D)
        s["v"] = _codes(g, (T, G, D), 1.0, V_FMT, 8, torch.int8).view(T, G * D)
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
    q = torch.randn((T, H, D), generator=g, device="cuda") * 1.2 * spread
    s["q"] = (torch.round(q / Q_ROT[0]) + Q_ROT[1]).clamp_(-32768, 32767).to(torch.int16) \
        .view(T, H * D)
    s["k_cache"].copy_(_codes(g, tuple(s["k_cache"].shape), 1.0, K_ROT, 8, torch.int8))
    s["v_cache"].copy_(_codes(g, tuple(s["v_cache"].shape), 1.0, V_FMT, 8, torch.int8))
    s.update(window=case["window"], sinks=case["sinks"], scale=float(np.float32(D ** -0.5)))
    s["ctx"] = torch.empty((T, H * D), dtype=torch.int16, device="cuda")
    s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


def _prepare_sample(case, g):
    M, V, mix = case["M"], case["V"], case["mix"]
    x = torch.randn((M, V), generator=g, device="cuda") * 2.5
    # a few likely words a row
    at = torch.randint(0, V, (M, 12), generator=g, device="cuda")
    x.scatter_(1, at, 7.0 + 4.0 * torch.rand((M, 12), generator=g, device="cuda"))
    s = dict(kind="sample", M=M, V=V, alpha=1.0, zp=0)

    def pick(values, dtype):
        v = torch.tensor(values, device="cuda", dtype=dtype)
        return v[torch.randint(0, len(values), (M,), generator=g, device="cuda")]

    f = torch.float32
    s["temperature"] = 0.5 + 0.8 * torch.rand(M, generator=g, device="cuda")
    s["top_k"] = s["top_p"] = s["min_p"] = None
    if mix == "topk":
        s["top_k"] = pick([20, 50, 64], torch.int32)
        s["top_p"] = pick([0.9, 0.95], f)
    elif mix == "nucleus":
        s["top_p"] = pick([0.8, 0.9, 0.95, 0.99], f)
        s["min_p"] = pick([0.0, 0.02, 0.05], f)
    elif mix == "all":
        # every request its own settings: some off, some greedy
        s["temperature"] = s["temperature"] * pick([0.0, 1.0, 1.0, 1.0], f)
        s["top_k"] = pick([0, 1, 40, 1000], torch.int32)
        s["top_p"] = pick([0.7, 0.95, 1.0], f)
        s["min_p"] = pick([0.0, 0.01, 0.1], f)
    if case["bits"] == 16:
        s["alpha"], s["zp"] = _fmt(-18.0, 20.0, 16)
        x = (torch.round(x / s["alpha"]) + s["zp"]).clamp_(-32768, 32767).to(torch.int16)
    else:
        # words that a grammar forbids at this place
        x[:, V // 3:V // 3 + V // 50] = -math.inf
    s["logits"] = x
    s["u"] = torch.rand(M, generator=g, device="cuda")
    s["tokens"] = torch.empty(M, dtype=torch.int32, device="cuda")
    s["workspace"] = torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# The operators.

def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "attend": _attend, "sample": _sample}[s["kind"]](s)


def _run_own(s):
    import paper_2408_13933_amd as mq
    if s["kind"] == "append":
        mq.mq_rope_append(s["q"], s["k"], s["v"], *Q_IN, *Q_ROT, *K_IN, *K_ROT, s["k_cache"],
                          s["v_cache"], s["starts"], s["lens"], s["pages"], table=s["table"],
                          out=s["q_rot"])
        return {"q": s["q_rot"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if s["kind"] == "attend":
        return mq.mq_paged_attn(s["q"], *Q_ROT, s["k_cache"], K_ROT[0], s["v_cache"], *V_FMT,
                                s["starts"], s["lens"], s["pages"], s["scale"], *CTX_FMT, 16,
                                window=s["window"], sinks=s["sinks"], max_len=s["L"],
                                out=s["ctx"], workspace=s["workspace"])
    return mq.mq_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                        top_p=s["top_p"], min_p=s["min_p"], alpha=s["alpha"], zp=s["zp"],
                        out=s["tokens"], workspace=s["workspace"])


def _code(v, fmt, bits):
    """Requantization of fp64 values: rint(v / scale) + zp, limited to the range."""
    lo = -(1 << (bits - 1))
    return (torch.round(v / fmt[0]) + fmt[1]).clamp_(lo, -lo - 1)


def _rows(s):
    """Sequence and position of every token row."""
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["starts"], t.to(torch.int32), right=True) - 1
    return b, s["lens"][b].long() - s["starts"][b + 1] + t


def _rotate(x, heads, fmt, cs, out_fmt, bits):
    """Pairs (i, i + D/2) of every head by the position's angle, in 64 bits:
    a code next to a rounding border must not depend on the type."""
    u = (fmt[0] * (x.double() - fmt[1])).view(x.shape[0], heads, 2, -1)
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    y = torch.stack((u[:, :, 0] * c - u[:, :, 1] * n, u[:, :, 1] * c + u[:, :, 0] * n), 2)
    return _code(y.view(x.shape[0], heads, -1), out_fmt, bits)


def _append(s):
    b, pos = _rows(s)
    cs = s["table"].view(-1, s["D"] // 2, 2)[pos]
    s["q_rot"].copy_(_rotate(s["q"], s["H"], Q_IN, cs, Q_ROT, 16).view_as(s["q_rot"]))
    k = _rotate(s["k"], s["G"], K_IN, cs, K_ROT, 8).to(torch.int8)
    at, slot = s["pages"][b, pos // s["page"]].long(), pos % s["page"]
    s["k_cache"][at, :, slot] = k
    s["v_cache"][at, :, :, slot] = s["v"].view(s["T"], s["G"], s["D"])
    return {"q": s["q_rot"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend(s):
    """Padded to the longest sequence.  64 bits: the integer logits and the
    weights next to a rounding border need them."""
    H, G, D, N, page = s["H"], s["G"], s["D"], s["new"], s["page"]
    B, T, g = s["lens"].numel(), s["T"], s["H"] // s["G"]
    P = -(-s["L"] // BLOCK) * BLOCK
    j = torch.arange(P, device="cuda")
    at = s["pages"][:, (j // page).clamp(max=s["pages"].shape[1] - 1)].long()
    k = s["k_cache"][at, :, j % page].double()          # [B][P][G][D]
    v = s["v_cache"][at, :, :, j % page].double() - V_FMT[1]
    k, v = (x.permute(0, 2, 1, 3) for x in (k, v))
    # every sequence's rows in N places, the last of them its last token
    b, pos = _rows(s)
    n = pos - (s["lens"][b].long() - N)
    q = torch.zeros((B, N, G, g, D), dtype=torch.float64, device="cuda")
    q[b, n] = s["q"].double().view(T, G, g, D) - Q_ROT[1]
    q = q.permute(0, 2, 3, 1, 4).reshape(B, G, g * N, D)
    c = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, G, g, N, P)
    at_pos = (s["lens"][:, None].long() - N + torch.arange(N, device="cuda"))[:, :, None]
    see = j <= at_pos                                    # [B][N][P]
    if s["window"] > 0:
        see &= (j > at_pos - s["window"]) | (j < s["sinks"])
    see = see[:, None, None]
    c = c.masked_fill(~see, -math.inf).view(B, G, g, N, P // BLOCK, BLOCK)
    sigma = np.float64(np.float32(Q_ROT[0])) * np.float64(np.float32(K_ROT[0])) * \
        np.float64(np.float32(s["scale"]))
    top = c.amax(5, keepdim=True)
    most = top.amax(4, keepdim=True)
    e = torch.exp(sigma * (c - top.clamp(min=-1e18)))
    w = torch.round(W_MAX * e) * torch.exp(sigma * (top - most.clamp(min=-1e18)))
    w = w.view(B, G, g * N, P)
    z = w.sum(3, keepdim=True)
    o = torch.matmul(w, v.contiguous())
    o = torch.where(z > 0, np.float64(np.float32(V_FMT[0])) * o / z.clamp(min=1e-300),
                    torch.zeros_like(o))
    o = o.view(B, G, g, N, D).permute(0, 3, 1, 2, 4)[b, n]
    s["ctx"].copy_(_code(o, CTX_FMT, 16).view(T, H * D))
    return s["ctx"]


def _sample(s):
    M, V = s["M"], s["V"]
    # the order, ties by index; a row's weights as integers, in 64 bits
    x = s["logits"]
    order = torch.sort(x, dim=1, descending=True, stable=True)[1]
    x = s["alpha"] * (x.double() - s["zp"])
    most = x.amax(1, keepdim=True)
    t = s["temperature"].double()[:, None]
    greedy = ~(t > 0)
    t = torch.where(greedy, torch.ones_like(t), t)
    w = torch.round(SAMPLE_ONE * torch.exp((x - most) / t)).to(torch.int64)
    rank = torch.arange(V, device="cuda")[None, :]
    ws = w.gather(1, order)
    k = torch.full((M, 1), V, device="cuda") if s["top_k"] is None else s["top_k"].long()[:, None]
    k = torch.where(k > 0, k, V)
    k = torch.where(greedy, torch.ones_like(k), k)
    ws = ws * (rank < k)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        total = ws.sum(1, keepdim=True).double()
        before = (ws.cumsum(1) - ws).double()
        ws = ws * ((before < p * total) | (p >= 1) | (rank == 0))
    if s["min_p"] is not None:
        ws = ws * (ws.double() >= s["min_p"].double()[:, None] * SAMPLE_ONE)
    w = torch.zeros_like(w).scatter_(1, order, ws)
    c = w.cumsum(1)
    total = c[:, -1:]
    r = torch.floor(s["u"].double()[:, None] * total.double()).to(torch.int64)
    r = torch.minimum(r, total - 1)
    s["tokens"].copy_((c <= r).sum(1))
    return s["tokens"]


# ---------------------------------------------------------------------------

def _mean_lens(case):
    """Expected new tokens and length of a sequence (prepare() draws them)."""
    if not case["ragged"]:
        return float(case["new"]), float(case["L"])
    new = max(1.0, 0.7 * case["new"])
    return new, new + 0.5 * (case["L"] - case["new"])


def work(case):
    if case["kind"] == "sample":
        n = case["M"] * case["V"]
        # every logit read once; a weight and a comparison or two each
        return {"bytes": float(n * case["bits"] // 8 + case["M"] * 24), "flops": 20.0 * n}
    H, G, D = HEADS[case["heads"]]
    new, L = _mean_lens(case)
    T = case["B"] * new
    if case["kind"] == "append":
        # queries in and out, keys in 16 bits and out in 8, values in and out;
        # a position's angles
        return {"bytes": T * (4.0 * H * D + 3.0 * G * D + 2.0 * G * D + 8.0 * D),
                "flops": 5.0 * T * (H + G) * D}
    # keys that some row of the sequence sees, and pairs that a row sees
    seen, pairs = L, new * (L - (new - 1) / 2.0)
    if case["window"] > 0:
        seen = min(L, case["window"] + new - 1 + case["sinks"])
        pairs = min(pairs, new * float(min(L, case["window"] + case["sinks"])))
    return {"bytes": case["B"] * (2.0 * seen * G * D + 4.0 * new * H * D),
            "flops": 4.0 * case["B"] * pairs * H * D}


# ---------------------------------------------------------------------------
# The same from the definitions, with numpy on the host.

def exact(case, seed):
    n = {"append": lambda: case["B"] * case["new"] * 2048,
         "attend": lambda: case["B"] * case["new"] * HEADS[case["heads"]][0] * case["L"],
         "sample": lambda: case["M"] * case["V"]}[case["kind"]]()
    if n > (12 << 20 if case["kind"] == "sample" else 40 << 20):
        return None
    s = prepare(case, seed)
    h = {k: v.cpu().numpy() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[
        case["kind"]](h)


def _np_code(v, fmt, bits):
    half = 2 ** (bits - 1)
    return np.clip(np.rint(v / np.float64(np.float32(fmt[0]))) + fmt[1], -half, half - 1)


def _exact_append(h):
    D, P = h["D"], h["page"]
    q, kc, vc = h["q"].copy(), h["k_cache"], h["v_cache"]
    half = D // 2
    for b in range(len(h["lens"])):
        t0, t1 = int(h["starts"][b]), int(h["starts"][b + 1])
        pos = np.arange(t0, t1) + int(h["lens"][b]) - t1
        ang = h["table"].reshape(-1, half, 2)[pos]
        turn = np.empty((t1 - t0, half), np.complex128)
        turn.real, turn.imag = ang[..., 0], ang[..., 1]
        for name, heads, fi, fo, bits in (("q", h["H"], Q_IN, Q_ROT, 16),
                                          ("k", h["G"], K_IN, K_ROT, 8)):
            x = np.float64(np.float32(fi[0])) * (h[name][t0:t1].astype(np.float64) - fi[1])
            x = x.reshape(t1 - t0, heads, D)
            y = (x[..., :half] + 1j * x[..., half:]) * turn[:, None, :]
            y = _np_code(np.concatenate((y.real, y.imag), -1), fo, bits)
            if name == "q":
                q[t0:t1] = y.reshape(t1 - t0, -1)
            else:
                for i, p in enumerate(pos):
                    kc[h["pages"][b, p // P], :, p % P] = y[i]
                    vc[h["pages"][b, p // P], :, :, p % P] = h["v"][t0 + i].reshape(h["G"], D)
    return {"q": q, "k_cache": kc, "v_cache": vc}


def _exact_attend(h):
    H, G, D, P = h["H"], h["G"], h["D"], h["page"]
    sigma = np.float64(np.float32(Q_ROT[0])) * np.float64(np.float32(K_ROT[0])) * \
        np.float64(np.float32(h["scale"]))
    y = np.zeros((h["T"], H, D))
    for b in range(len(h["lens"])):
        L, t0, t1 = int(h["lens"][b]), int(h["starts"][b]), int(h["starts"][b + 1])
        pos = np.arange(L)
        pg = h["pages"][b, pos // P]
        for hd in range(H):
            k = h["k_cache"][pg, hd // (H // G), pos % P].astype(np.float64)
            v = h["v_cache"][pg, hd // (H // G), :, pos % P].astype(np.float64)
            for t in range(t0, t1):
                at = L - t1 + t
                sees = np.arange(at + 1)
                if h["window"] > 0:
                    sees = sees[(sees > at - h["window"]) | (sees < h["sinks"])]
                if not len(sees):
                    continue
                c = k[sees] @ (h["q"][t, hd * D:(hd + 1) * D].astype(np.float64) - Q_ROT[1])
                num, den = np.zeros(D), 0.0
                for i in np.unique(sees // BLOCK):
                    m = sees // BLOCK == i
                    top = c[m].max()
                    w = np.rint(W_MAX * np.exp(sigma * (c[m] - top)))
                    f = np.exp(sigma * (top - c.max()))
                    num += f * (w @ (v[sees[m]] - V_FMT[1]))
                    den += f * w.sum()
                y[t, hd] = np.float64(np.float32(V_FMT[0])) * num / den
    return _np_code(y, CTX_FMT, 16).astype(np.int16).reshape(h["T"], H * D)


def _exact_sample(h):
    out = np.empty(h["M"], np.int32)
    for m in range(h["M"]):
        x = np.float64(np.float32(h["alpha"])) * (h["logits"][m].astype(np.float64) - h["zp"])
        order = np.argsort(-x, kind="stable")
        t = float(h["temperature"][m])
        kept = len(x) if h["top_k"] is None or h["top_k"][m] <= 0 else int(h["top_k"][m])
        if not t > 0:
            kept, t = 1, 1.0
        order = order[:kept]
        w = [int(i) for i in np.rint(np.exp((x[order] - x[order[0]]) / t) * SAMPLE_ONE)]
        w = np.array(w, dtype=object) if len(w) < 2000 else np.array(w, dtype=np.int64)
        if h["top_p"] is not None and h["top_p"][m] < 1:
            before = np.cumsum(w) - w
            ok = before.astype(np.float64) < np.float64(h["top_p"][m]) * float(w.sum())
            ok[0] = True
            order, w = order[ok], w[ok]
        if h["min_p"] is not None:
            ok = w.astype(np.float64) >= np.float64(h["min_p"][m]) * SAMPLE_ONE
            order, w = order[ok], w[ok]
        back = np.argsort(order)
        order, w = order[back], w[back]
        total = int(w.sum())
        r = min(int(np.floor(np.float64(h["u"][m]) * float(total))), total - 1)
        out[m] = order[np.nonzero(np.cumsum(w) > r)[0][0]]
    return out
