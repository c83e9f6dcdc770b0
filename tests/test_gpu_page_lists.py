"""Page lists that end with a sequence's last page: the entries after it are
not read.  The last sequence's list is the end of an allocation, so a read of
them would be a read past it; the outputs are those of whole lists."""
import struct

import pytest

pytestmark = pytest.mark.gpu

QF, KF, QO, KO = (3.1e-4, 700), (2.4e-4, -1500), (3.3e-4, -1600), (0.0667, -7)
VF, OF = (0.031, 5), (1.2e-4, -11)
MEMORY = 32 << 20  # bytes; an allocation of its own


def _ends_with(entries):
    """int32 entries as the last ones of an allocation."""
    import torch
    m = torch.empty(MEMORY // 4, dtype=torch.int32, device="cuda")
    at = m[MEMORY // 4 - entries.numel():]
    at.copy_(entries)
    return at


@pytest.mark.parametrize("H,G,D", [(8, 2, 64), (4, 1, 128), (2, 1, 256)])
@pytest.mark.parametrize("page", [16, 32, 64])
@pytest.mark.parametrize("new,lens", [(1, (200, 1)), (1, (9, 17)), (1, (700, 383)), (9, (400, 130)),
                                      (40, (300, 257)), (70, (90, 900))])
def test_list_ends_with_the_last_page(H, G, D, page, new, lens):
    import torch

    import paper_2408_13933_amd as mq
    B, ld = 2, 80
    n = [min(new, x) for x in lens]
    T = sum(n)
    g = torch.Generator(device="cuda").manual_seed(page + new)
    i16, i8 = dict(dtype=torch.int16, device="cuda"), dict(dtype=torch.int8, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    q, k = (torch.randint(-9000, 9001, (T, h * D), generator=g, **i16) for h in (H, G))
    v = torch.randint(-100, 101, (T, G * D), generator=g, **i8)
    need = [-(-x // page) for x in lens]
    pool = sum(need) + 2
    cache = [torch.randint(-100, 101, s, generator=g, **i8)
             for s in ((pool, G, page, D), (pool, G, D, page))]
    perm = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    pages = torch.zeros((B, ld), **i32)
    pages[0, :need[0]] = perm[:need[0]]
    pages[1, :need[1]] = perm[need[0]:sum(need)]
    starts, ls = torch.tensor([0, n[0], T], **i32), torch.tensor(lens, **i32)
    table = mq.mq_rope_table(max(lens), D)
    short = _ends_with(pages.flatten()[:ld + need[1]])
    ws = torch.empty(mq.mq_paged_attn_workspace_bytes(T, B, H, G, D, max(lens)),
                     dtype=torch.uint8, device="cuda")
    cached = [c.clone() for c in cache]
    out, y = torch.empty_like(q), torch.empty((T, H * D), **i16)
    c = struct.pack("qqqiii4x", *(t.data_ptr() for t in cached), pool, page, G, D)
    b = struct.pack("qqqqq", starts.data_ptr(), ls.data_ptr(), short.data_ptr(), B, ld)
    stream = torch.cuda.current_stream().cuda_stream
    for window, sinks in ((0, 0), (50, 3)):
        want_q = mq.mq_rope_append(q, k, v, *QF, *QO, *KF, *KO, *cache, starts, ls, pages,
                                   table=table)
        want = mq.mq_paged_attn(want_q, *QO, cache[0], KO[0], cache[1], *VF, starts, ls, pages,
                                D ** -0.5, *OF, 16, window=window, sinks=sinks, max_len=max(lens),
                                workspace=ws)
        assert mq.lib().mq_rope_append(q.data_ptr(), H * D, k.data_ptr(), G * D, v.data_ptr(), G * D,
                                       T, H, *QF, *QO, *KF, *KO, table.data_ptr(), max(lens), c, b,
                                       out.data_ptr(), H * D, stream) == 0
        assert mq.lib().mq_paged_attn(out.data_ptr(), H * D, T, H, *QO, c, KO[0], *VF, b, D ** -0.5,
                                      window, sinks, *OF, 16, y.data_ptr(), H * D, max(lens),
                                      ws.data_ptr(), ws.numel(), stream) == 0
        assert torch.equal(out, want_q) and torch.equal(y, want)
        assert torch.equal(cached[0], cache[0]) and torch.equal(cached[1], cache[1])
