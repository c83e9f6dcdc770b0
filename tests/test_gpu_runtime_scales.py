"""The operators with scales found at run time together: a small decoder generates
with them, each call checked against its definition on the inputs that it got, in
prompts, chunks and single tokens, eager and captured."""
import numpy as np
import pytest

from tests import runtime_scales as rs
from tests.test_gpu_attn_blocks import _compare
from tests.test_gpu_linear_tokens import _cuda, _weights

pytestmark = pytest.mark.gpu

TYPES = ["float32", "bfloat16", "float16"]
V, C, H, G, D, FF, LAYERS = 500, 128, 4, 2, 32, 264, 2
PAGE, BLOCK, PAGES, LONGEST = 32, 16, 40, 256


class Decoder:
    """gain: of the weights (at 1 values grow from layer to layer past fp16, logits past 1e7);
    checked: every call against its definition (None: nothing that waits)."""

    def __init__(self, type, gain, checked):
        import torch

        import paper_2408_13933_amd as mq
        rng = np.random.default_rng(1)
        self.dt, self.type, self.checked = getattr(torch, type), type, checked
        self.embed = torch.from_numpy(rng.standard_normal((V, C)).astype(np.float32)).to(self.dt)
        self.embed = self.embed.cuda()

        def weights(N, K, bits, asym, bias):
            w, s, zp = _weights(rng, N, K, bits, asym)
            s *= np.float32(gain * (0.1 if bits == 8 else 1.0))
            b = rng.standard_normal(N).astype(np.float32) if bias else None
            return (w, s, zp, b), (_cuda(rs.pack4(w) if bits == 4 else w), bits, _cuda(s),
                                   _cuda(zp), _cuda(b))
        self.layers = [(weights((H + 2 * G) * D, C, 4, False, True),
                        weights(C, H * D, 8, True, False), weights(FF, C, 8, False, False),
                        weights(C, FF, 4, True, True)) for _ in range(LAYERS)]
        self.head = weights(V, C, 8, False, False)
        self.caches = [[torch.zeros(s, dtype=t, device="cuda") for s, t in (
            ((PAGES, G, PAGE, D), torch.int8), ((PAGES, G, PAGE // BLOCK), torch.float32),
            ((PAGES, G, PAGE // 16, D, 16), torch.int8),
            ((PAGES, G, PAGE // BLOCK), torch.float32))] for _ in range(LAYERS)]
        self.table = mq.mq_rope_table(LONGEST, D)

    def linear(self, x, w):
        import torch

        import paper_2408_13933_amd as mq
        (wn, sn, zn, bn), (wq, bits, s, zp, b) = w
        y = mq.mq_linear_tokens(x, wq, bits, s, w_zp=zp, bias=b)
        if self.checked:
            codes, scale, _ = rs.quantize_tokens(x.float().cpu().numpy())
            want = torch.from_numpy(rs.linear(codes, scale, wn, sn, zn, bn)).to(self.dt)
            assert torch.equal(y.cpu(), want)
        return y

    def attention(self, qkv, cache, starts, lens, pages):
        """Rows of one tensor for queries, keys and values."""
        import torch

        import paper_2408_13933_amd as mq
        q, k, v = qkv[:, :H * D], qkv[:, H * D:(H + G) * D], qkv[:, (H + G) * D:]
        before = [a.cpu().numpy() for a in cache] if self.checked else None
        rot = mq.mq_rope_append_blocks(q, k, v, *cache, starts, lens, pages, table=self.table)
        out = mq.mq_paged_attn_blocks(rot, *cache, starts, lens, pages, D ** -0.5)
        if self.checked:
            at = [a.cpu().numpy() for a in (starts, lens, pages)]
            kc, ks, vc, vs = before
            vc, want = rs.v_rows(vc), np.zeros(tuple(q.shape), np.float32)
            rs.append_blocks(*[a.float().cpu().numpy() for a in (q, k, v)], kc, ks, vc, vs, *at,
                             self.table.cpu().numpy().reshape(LONGEST, D // 2, 2), want)
            assert torch.equal(rot.cpu(), torch.from_numpy(want).to(self.dt))
            for a, b in zip(cache, (kc, ks, rs.v_layout(vc), vs)):
                assert np.array_equal(a.cpu().numpy(), b)
            _compare(out.float().cpu().numpy(), rot.float().cpu().numpy(), (kc, ks, vc, vs), at,
                     float(np.float32(D ** -0.5)), self.type, D, 0, 0)
        return out

    def hidden(self, ids, starts, lens, pages):
        x = self.embed.index_select(0, ids)
        for (qkv, o, up, down), cache in zip(self.layers, self.caches):
            y = self.attention(self.linear(x, qkv), cache, starts, lens, pages)
            x = x + self.linear(y, o)
            x = x + self.linear(self.linear(x, up).relu(), down)
        return x

    def draw(self, x, history, held, prompts, settings, u):
        import torch

        import paper_2408_13933_amd as mq
        logits = self.linear(x, self.head)
        before = logits.clone()
        mq.mq_adjust_logits(logits, history=history, hist_lens=held, prompt_lens=prompts,
                            **settings)
        if self.checked:
            n = {k: v.cpu().numpy() if torch.is_tensor(v) else
                 tuple(a.cpu().numpy() for a in v) for k, v in settings.items()}
            want = rs.adjust_logits(before.float().cpu().numpy(), history=history.cpu().numpy(),
                                    lens=held.cpu().numpy(), prompts=prompts.cpu().numpy(), **n)
            assert torch.equal(logits.cpu(), torch.from_numpy(want).to(self.dt))
        next = mq.mq_sample(logits.float(), u)
        if self.checked is not None:
            at = next.cpu().long()  # (a row without any word gives -1)
            assert ((at >= 0) & (at < V)).all()
            assert (logits.cpu().gather(1, at[:, None]) > -np.inf).all()
        return next.clamp(0, V - 1)


def _settings(B):
    import torch
    rng = np.random.default_rng(2)
    bits = rng.random((B, -(-V // 32) * 32)) < 0.8
    bits[:, :4] = True
    f = [torch.from_numpy(rng.uniform(a, b, B).astype(np.float32)).cuda()
         for a, b in ((1.0, 1.5), (0, 1), (0, 0.5))]
    bias = (np.arange(B + 1, dtype=np.int32) * 3, rng.integers(0, V, 3 * B).astype(np.int32),
            rng.standard_normal(3 * B).astype(np.float32))
    return dict(repetition=f[0], presence=f[1], frequency=f[2], bias=tuple(_cuda(a) for a in bias),
                mask=_cuda(np.packbits(bits, axis=1, bitorder="little").view(np.int32)))


class Batch:
    """Prompts of 37, 5 and 64 words, their histories, pages for 100 words each."""

    def __init__(self):
        import torch
        rng = np.random.default_rng(3)
        self.prompts = [rng.integers(0, V, n) for n in (37, 5, 64)]
        self.B = len(self.prompts)
        self.pages = _cuda(rng.permutation(PAGES)[:4 * self.B].reshape(self.B, 4).astype(np.int32))
        self.history = torch.zeros(self.B, 100, dtype=torch.int32, device="cuda")
        for b, p in enumerate(self.prompts):
            self.history[b, :len(p)] = _cuda(p.astype(np.int32))
        self.held = _cuda(np.array([len(p) for p in self.prompts], np.int32))
        self.first = self.held.clone()
        self.settings = _settings(self.B)

    def fed(self, parts):
        """ids, starts, lens of calls that feed the prompts in parts of at most that many
        words, the sequences' last words with the last call."""
        n = max(-(-len(p) // parts) for p in self.prompts)
        done = [0] * self.B
        for c in range(n):
            ids, starts = [], [0]
            for b, p in enumerate(self.prompts):
                left = n - c - 1
                take = max(0, min(parts, len(p) - done[b] - left)) if parts == 1 or left == 0 or \
                    len(p) - done[b] > parts * left else 0
                ids += list(p[done[b]:done[b] + take])
                done[b] += take
                starts.append(len(ids))
            yield [_cuda(np.array(a, t)) for a, t in ((ids, np.int64), (starts, np.int32),
                                                      (done, np.int32))]


def _generate(model, batch, steps, parts):
    """The hidden rows of the prompts' last words and the words drawn."""
    import torch
    for ids, starts, lens in batch.fed(parts):
        x = model.hidden(ids, starts, lens, batch.pages)
    x = x[starts[1:].long() - 1]
    first = x.clone()
    u = torch.rand(steps, batch.B, generator=torch.Generator().manual_seed(5)).cuda()
    held, history, words = batch.held.clone(), batch.history.clone(), []
    one = torch.arange(batch.B + 1, dtype=torch.int32, device="cuda")
    for i in range(steps):
        next = model.draw(x, history, held, batch.first, batch.settings, u[i])
        words.append(next)
        history.scatter_(1, held.long()[:, None], next[:, None])
        held += 1
        x = model.hidden(next.long(), one, held, batch.pages)
    return first, torch.stack(words)


@pytest.mark.parametrize("type,gain", [("float32", 1.0), ("bfloat16", 1.0), ("float32", 0.05),
                                       ("bfloat16", 0.05), ("float16", 0.05)])
@pytest.mark.parametrize("parts", [64, 16, 7, 1])
def test_generation_step_by_step(type, gain, parts):
    _generate(Decoder(type, gain, True), Batch(), 6, parts)


@pytest.mark.parametrize("type", TYPES)
def test_chunks_of_whole_blocks_fill_the_cache_like_one_prompt(type):
    """The first layer's codes and scales, which no attention is before, bit for bit."""
    import torch
    caches = []
    for parts in (64, 32, 16):
        model, batch = Decoder(type, 0.05, False), Batch()
        batch.prompts = [p[:len(p) // 16 * 16] for p in batch.prompts[::2]]
        batch.B, batch.pages = 2, batch.pages[::2].contiguous()
        for ids, starts, lens in batch.fed(parts):
            model.hidden(ids, starts, lens, batch.pages)
        caches.append(model.caches[0])
    for other in caches[1:]:
        assert all(torch.equal(a, b) for a, b in zip(caches[0], other))


@pytest.mark.parametrize("type", TYPES)
def test_captured_generation(type):
    """A step with its draw as a graph, replayed with eager calls between, and on another
    stream: the words of the eager run."""
    import torch
    steps = 8
    _, want = _generate(Decoder(type, 0.05, False), Batch(), steps, 64)
    model, batch = Decoder(type, 0.05, None), Batch()
    for ids, starts, lens in batch.fed(64):
        x = model.hidden(ids, starts, lens, batch.pages)
    x = x[starts[1:].long() - 1].clone()
    us = torch.rand(steps, batch.B, generator=torch.Generator().manual_seed(5)).cuda()
    u, held, history = us[0].clone(), batch.held.clone(), batch.history.clone()
    one = torch.arange(batch.B + 1, dtype=torch.int32, device="cuda")
    word = torch.empty(batch.B, dtype=torch.int32, device="cuda")

    def step():
        word.copy_(model.draw(x, history, held, batch.first, batch.settings, u))
        history.scatter_(1, held.long()[:, None], word[:, None])
        held.add_(1)
        x.copy_(model.hidden(word.long(), one, held, batch.pages))

    start = [a.clone() for a in (x, held, history)]
    caches = [[a.clone() for a in c] for c in model.caches]

    def back():
        for a, b in zip((x, held, history), start):
            a.copy_(b)
        for c, d in zip(model.caches, caches):
            for a, b in zip(c, d):
                a.copy_(b)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = []
        for i in range(steps):
            u.copy_(us[i])
            step()
            got.append(word.clone())
    torch.cuda.synchronize()
    assert torch.equal(torch.stack(got), want)
    back()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        back()
        for i in range(steps):
            u.copy_(us[i])
            if i % 4 == 3:
                step()
            else:
                graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(word, want[i])
