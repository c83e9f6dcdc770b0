"""The cache, the attention over it and the draw of a token run together, as a
serving program runs them: prompts in one piece, in chunks and token by token
give the same tokens; a decoding step captured into a graph; streams other
than the current one."""
import numpy as np
import pytest

from tests import generation as gen

pytestmark = pytest.mark.gpu

H, G, D, HID, V, PAGE = 8, 2, 64, 256, 3000, 32
QF, KF, VF = (6.0e-5, 40), (6.0e-5, -25), (0.016, 3)
QO, KO = (6.2e-5, -10), (0.016, 2)
OF = (0.011, -4)
LF = (1.5e-4, 0)  # logits before their dequantization
XF = (0.03, 1)


class Model:
    """One attention layer between an embedding and a vocabulary, in codes."""

    def __init__(self, B, max_len, positions=4096):
        import torch

        import paper_2408_13933_amd as mq
        self.mq, self.torch, self.B = mq, torch, B
        g = torch.Generator().manual_seed(7)
        self.embed = torch.randint(-127, 128, (V, HID), generator=g, dtype=torch.int8).cuda()
        w = lambda n, k: mq.mq_pack_weights((torch.randn(n, k, generator=g) * 0.03).cuda(), 8)
        self.wq, self.wk, self.wv, self.wo = (w(H * D, HID), w(G * D, HID), w(G * D, HID),
                                              w(V, H * D))
        self.table = mq.mq_rope_table(positions, D)
        per = -(-max_len // PAGE)
        self.max_len = per * PAGE
        perm = torch.randperm(B * per + 2, generator=g)[:B * per].to(torch.int32)
        self.pages = perm.reshape(B, per).cuda()
        n = B * per + 2
        self.kc = torch.zeros((n, G, PAGE, D), dtype=torch.int8, device="cuda")
        self.vc = torch.zeros((n, G, D, PAGE), dtype=torch.int8, device="cuda")
        self.temperature = torch.tensor([0.0, 0.7, 1.0, 1.3] * B, device="cuda")[:B]
        self.top_k = torch.tensor([0, 40, 0, 5] * B, dtype=torch.int32, device="cuda")[:B]
        self.top_p = torch.tensor([1.0, 0.9, 0.95, 1.0] * B, device="cuda")[:B]
        self.min_p = torch.tensor([0.0, 0.0, 0.01, 0.0] * B, device="cuda")[:B]

    def context(self, tokens, starts, lens, kc=None, vc=None, ws=None, **kw):
        """Appends tokens [T] and returns their q codes and contexts."""
        mq = self.mq
        kc, vc = (self.kc, self.vc) if kc is None else (kc, vc)
        x = self.embed[tokens]
        q = mq.mq_qlinear(x, *self._w(self.wq), *XF, *QF, 16)
        k = mq.mq_qlinear(x, *self._w(self.wk), *XF, *KF, 16)
        v = mq.mq_qlinear(x, *self._w(self.wv), *XF, *VF, 8)
        qr = mq.mq_rope_append(q, k, v, *QF, *QO, *KF, *KO, kc, vc, starts, lens, self.pages,
                               table=self.table)
        c = mq.mq_paged_attn(qr, *QO, kc, KO[0], vc, *VF, starts, lens, self.pages, D ** -0.5,
                             *OF, 8, max_len=self.max_len, workspace=ws, **kw)
        return (q, k, v), c

    @staticmethod
    def _w(packed):
        wq, ws, cs = packed
        return wq, 8, ws, cs

    def draw(self, c, u, ws=None):
        logits = self.mq.mq_qlinear_dequant(c, *self._w(self.wo), *OF, *LF, 16)
        return logits, self.mq.mq_sample(logits, u, self.temperature, self.top_k, self.top_p,
                                         self.min_p, workspace=ws)


def _prompts(B, seed):
    rng = np.random.default_rng(seed)
    return [rng.integers(0, V, n).astype(np.int64) for n in rng.integers(1, 300, B)]


def _run(model, prompts, chunk, steps, us):
    """Prompts in pieces of `chunk` tokens (None: whole), then `steps` drawn
    tokens per sequence; the contexts of all prompt tokens and the tokens."""
    torch = model.torch
    B = len(prompts)
    i32 = dict(dtype=torch.int32, device="cuda")
    done = [0] * B
    ctx = [[] for _ in range(B)]
    last = [None] * B
    while any(done[b] < len(p) for b, p in enumerate(prompts)):
        new = [min(chunk or 10 ** 9, len(p) - done[b]) for b, p in enumerate(prompts)]
        toks = np.concatenate([p[done[b]:done[b] + new[b]] for b, p in enumerate(prompts)])
        starts = np.concatenate(([0], np.cumsum(new)))
        done = [d + n for d, n in zip(done, new)]
        _, c = model.context(torch.from_numpy(toks).cuda(), torch.tensor(starts, **i32),
                             torch.tensor(done, **i32))
        for b in range(B):
            if new[b]:
                ctx[b].append(c[starts[b]:starts[b + 1]])
                last[b] = c[starts[b + 1] - 1]
    out = []
    c = torch.stack(last)
    starts = torch.arange(B + 1, **i32)
    for s in range(steps):
        _, tok = model.draw(c, us[s])
        out.append(tok)
        done = [d + 1 for d in done]
        _, c = model.context(tok.long(), starts, torch.tensor(done, **i32))
    return [torch.cat(x).cpu().numpy() for x in ctx], torch.stack(out).cpu().numpy()


def test_prompts_whole_in_chunks_and_token_by_token():
    """The contexts do not depend on how the keys came into the cache or on
    how many rows are attended at once, but for a rounding tie of a join in
    fp64; so neither do the tokens."""
    import torch
    B, steps = 6, 12
    prompts = _prompts(B, 3)
    us = torch.rand(steps, B, generator=torch.Generator().manual_seed(5)).cuda()
    runs = [_run(Model(B, 330), prompts, chunk, steps, us) for chunk in (None, 37, 1)]
    for ctx, tokens in runs[1:]:
        for a, b in zip(ctx, runs[0][0]):
            assert np.array_equal(a, b)
        assert np.array_equal(tokens, runs[0][1])
    assert (runs[0][1] >= 0).all() and (runs[0][1] < V).all()
    assert len(np.unique(runs[0][1][:, 1:])) > steps  # not one token over and over


def test_run_against_plain_forms():
    """A prompt and three steps: cache, contexts and tokens against the plain
    forms, from the codes of the projections."""
    import torch
    B = 4
    model = Model(B, 320)
    i32 = dict(dtype=torch.int32, device="cuda")
    prompts = _prompts(B, 4)
    lens = np.array([len(p) for p in prompts])
    starts = np.concatenate(([0], np.cumsum(lens)))
    kc, vc = model.kc.cpu().numpy(), model.vc.cpu().numpy()
    pages = model.pages.cpu().numpy()
    angles = model.table.cpu().numpy().reshape(-1, D // 2, 2)
    tokens = torch.from_numpy(np.concatenate(prompts)).cuda()
    u = torch.rand(4, B, generator=torch.Generator().manual_seed(6)).cuda()
    for s in range(4):
        (q, k, v), c = model.context(tokens, torch.tensor(starts, **i32),
                                     torch.tensor(lens, **i32))
        qr = np.zeros(q.shape, np.int16)
        gen.rope_append(q.cpu().numpy(), k.cpu().numpy(), v.cpu().numpy(), QF, QO, KF, KO, kc, vc,
                        starts, lens, pages, angles, qr)
        assert np.array_equal(model.kc.cpu().numpy(), kc)
        assert np.array_equal(model.vc.cpu().numpy(), vc)
        real = gen.paged_attn(qr, QO, kc, KO[0], vc, VF, starts, lens, pages, D ** -0.5, 0, 0)
        slack = 255 * VF[0] / gen.ONE / OF[0] + 1e-9
        gen.assert_codes(c.cpu().numpy(), real, *OF, 8, slack)
        last = c[torch.from_numpy(starts[1:] - 1).cuda()].contiguous()
        logits, tok = model.draw(last, u[s])
        x = logits.cpu().numpy().astype(np.float64)
        f = lambda t: t.cpu().numpy().astype(np.float64)
        want = [gen.sample_row(x[b], f(u[s])[b], f(model.temperature)[b], int(model.top_k[b]),
                               f(model.top_p)[b], f(model.min_p)[b]) for b in range(B)]
        assert tok.tolist() == want
        tokens = tok.long()
        lens = lens + 1
        starts = np.arange(B + 1)


def _captured(step):
    import torch
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            step()
    torch.cuda.current_stream().wait_stream(s)
    return g


def test_captured_steps_share_workspaces():
    """A decoding step captured twice, over two caches and with the same
    workspaces, replayed in turn while lengths, tokens and random numbers
    change in place, with eager steps between: every token is the eager run's."""
    import torch
    B, steps, long = 4, 6, 700
    model = Model(B, long + 40)
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(9)
    fill = lambda t: t.random_(-100, 101, generator=g)
    caches = [(fill(torch.empty_like(model.kc)), fill(torch.empty_like(model.vc)))
              for _ in range(2)]
    mq = model.mq
    ws = torch.empty(mq.mq_paged_attn_workspace_bytes(B, B, H, G, D, model.max_len),
                     dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0
    ws2 = torch.empty(mq.mq_sample_workspace_bytes(B, V), dtype=torch.uint8, device="cuda")
    starts = torch.arange(B + 1, **i32)
    first = torch.tensor([long, 3, 129, 1], **i32)
    u = torch.rand(steps, B, generator=g, device="cuda")
    lens, tok, us = first.clone(), torch.zeros(B, dtype=torch.int64, device="cuda"), u[0].clone()

    def step(kc, vc, ws, ws2):
        _, c = model.context(tok, starts, lens, kc, vc, ws)
        return model.draw(c, us, ws2)[1]

    def start():
        lens.copy_(first)
        tok.copy_(torch.arange(B))

    saved = [tuple(t.clone() for t in c) for c in caches]
    want = []
    for c in caches:
        start()
        run = []
        for s in range(steps):
            us.copy_(u[s])
            new = step(*c, None, None)
            run.append(new.tolist())
            tok.copy_(new)
            lens.add_(1)
        want.append(run)
    assert want[0] != want[1]
    for c, old in zip(caches, saved):
        for t, o in zip(c, old):
            t.copy_(o)
    outs = [None, None]

    def body(i):
        outs[i] = step(*caches[i], ws, ws2)

    start()
    torch.cuda.synchronize()
    graphs = [_captured(lambda i=i: body(i)) for i in range(2)]
    state = [(first.clone(), torch.arange(B, device="cuda")) for _ in range(2)]
    for s in range(steps):
        us.copy_(u[s])
        for i in range(2):
            lens.copy_(state[i][0])
            tok.copy_(state[i][1])
            graphs[i].replay()
            torch.cuda.synchronize()
            assert outs[i].tolist() == want[i][s], (s, i)
            state[i] = (state[i][0] + 1, outs[i].long())
            # eager work in the same workspaces between replays
            lens.fill_(1)
            step(*saved[i], ws, ws2)
            torch.cuda.synchronize()


def test_stream_other_than_the_current_one():
    """Workspaces and outputs of a call on another stream are not memory that
    the current one still writes."""
    import torch

    import paper_2408_13933_amd as mq
    B = 3
    model = Model(B, 700)
    i32 = dict(dtype=torch.int32, device="cuda")
    gc = torch.Generator(device="cuda").manual_seed(1)
    model.kc.random_(-100, 101, generator=gc)
    model.vc.random_(-100, 101, generator=gc)
    q = torch.randint(-9000, 9000, (B, H * D), generator=gc, device="cuda", dtype=torch.int16)
    x = torch.randn(B, 50000, generator=gc, device="cuda")
    u = torch.rand(B, generator=gc, device="cuda")
    p = torch.full_like(u, 0.9)
    starts, lens = torch.arange(B + 1, **i32), torch.tensor([700, 5, 333], **i32)

    def attend(stream=None):
        return mq.mq_paged_attn(q, *QO, model.kc, KO[0], model.vc, *VF, starts, lens, model.pages,
                                D ** -0.5, *OF, 8, max_len=model.max_len, stream=stream)

    def sample(stream=None):
        return mq.mq_sample(x, u, top_p=p, stream=stream)

    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    for call, n in ((attend, mq.mq_paged_attn_workspace_bytes(B, B, H, G, D, model.max_len)),
                    (sample, mq.mq_sample_workspace_bytes(B, 50000))):
        want = call()
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(8):
            big @ big
        busy = torch.empty(n, dtype=torch.uint8, device="cuda")
        busy.fill_(1)  # after the products; the block is then free for this stream
        del busy
        got = call(side)
        side.synchronize()
        assert torch.equal(got, want)
        torch.cuda.synchronize()


def test_binding_refuses():
    """Tensors of another type, shape, layout or device, and streams of another
    device, are refused before anything is launched."""
    import types

    import torch
    model = Model(2, 64)
    mq = model.mq
    i32 = dict(dtype=torch.int32, device="cuda")
    base = dict(q=torch.zeros((3, H * D), dtype=torch.int16, device="cuda"),
                k=torch.zeros((3, G * D), dtype=torch.int16, device="cuda"),
                v=torch.zeros((3, G * D), dtype=torch.int8, device="cuda"), kc=model.kc,
                vc=model.vc, starts=torch.tensor([0, 1, 3], **i32),
                lens=torch.tensor([5, 9], **i32), pages=model.pages, table=model.table, out=None,
                stream=None, ws=None, logits=torch.zeros((2, 50), device="cuda"),
                u=torch.zeros(2, device="cuda"), t=None, k0=None, tok=None)

    def append(a):
        return mq.mq_rope_append(a.q, a.k, a.v, *QF, *QO, *KF, *KO, a.kc, a.vc, a.starts, a.lens,
                                 a.pages, table=a.table, out=a.out, stream=a.stream)

    def attend(a):
        return mq.mq_paged_attn(a.q, *QO, a.kc, KO[0], a.vc, *VF, a.starts, a.lens, a.pages, 0.125,
                                *OF, 16, out=a.out, workspace=a.ws, stream=a.stream)

    def sample(a):
        return mq.mq_sample(a.logits, a.u, temperature=a.t, top_k=a.k0, out=a.tok,
                            workspace=a.ws, stream=a.stream)

    cuda = dict(device="cuda")
    other = types.SimpleNamespace(device_index=torch.cuda.current_device() + 1, cuda_stream=0)
    both = [dict(q=base["q"].cpu()), dict(q=None), dict(q=base["q"].float()), dict(q=base["q"][0]),
            dict(q=base["q"][:, :-1]), dict(q=base["q"].t().contiguous().t()),
            dict(kc=base["kc"].cpu()), dict(kc=base["kc"].to(torch.int16)),
            dict(kc=base["kc"].transpose(2, 3)), dict(vc=model.kc), dict(vc=None),
            dict(starts=base["starts"][:2]), dict(starts=base["starts"].long()),
            dict(lens=base["starts"]), dict(lens=[5, 9]), dict(pages=base["pages"][:1]),
            dict(pages=base["pages"].t()), dict(out=base["q"][:2]), dict(out=base["v"]),
            dict(stream=other)]
    cases = {append: both + [dict(k=base["q"]), dict(v=base["k"]), dict(v=base["v"].cpu()),
                             dict(table=base["table"].float()), dict(table=base["table"].cpu())],
             attend: both + [dict(ws=torch.zeros(512, **cuda)),
                             dict(ws=torch.zeros(512, dtype=torch.uint8))],
             sample: [dict(logits=base["logits"].cpu()), dict(logits=base["logits"].half()),
                      dict(logits=base["logits"][0]), dict(logits=base["logits"].t()),
                      dict(u=base["u"][:1]), dict(u=base["u"].double()), dict(u=None),
                      dict(t=torch.zeros(3, **cuda)), dict(k0=torch.zeros(2, **cuda)),
                      dict(k0=torch.zeros(2, dtype=torch.int64, **cuda)),
                      dict(tok=torch.zeros(2, dtype=torch.int64, **cuda)),
                      dict(tok=torch.zeros(2, dtype=torch.int32)),
                      dict(ws=torch.zeros(512, **cuda)), dict(stream=other)]}
    for call, wrong in cases.items():
        call(types.SimpleNamespace(**base))
        for kw in wrong:
            with pytest.raises(ValueError):
                call(types.SimpleNamespace(**{**base, **kw}))
    small = torch.zeros(512, dtype=torch.uint8, **cuda)
    with pytest.raises(mq.MQError):  # less than a row's
        sample(types.SimpleNamespace(**{**base, "ws": small}))
    torch.cuda.synchronize()
