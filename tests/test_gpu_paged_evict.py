"""Eviction of sequences that lie in pages, as a program does it: a sequence's rows are
gathered by its table, evicted as a contiguous cache, and the kept rows written back into
the first of its pages; the others go back to the stack, from which the next sequence
takes its own."""

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_paged import DEV, DT, _dense, _i32, _pool
from test_gpu_prefix import check_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["heads", "rows", "side"])
@pytest.mark.parametrize("dtype,page,G", [("bf16", 8, 2), ("f32", 5, 1), ("bf16", 16, 4)])
def test_evicted_sequences_give_pages_back(dtype, page, G, layout):
    B, H, D, L, P, LAYERS = 4, 2, 64, 240, 6, 2
    g = torch.Generator().manual_seed(page)
    dt, HQ, entries = DT[dtype], H * G, -(-L // page)
    lens = [200, 77, 131, 0]
    budget = {0: 40, 2: 33}  # of the sequences that are evicted
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 2
    perm = torch.randperm(n_pages, generator=g).int().tolist()
    table = torch.full((B, entries), -1, dtype=torch.int32)
    for b in range(B):
        table[b, :need[b]] = torch.tensor(perm[sum(need[:b]):sum(need[:b + 1])], dtype=torch.int32)
    table, lens, held = table.to(DEV), _i32(lens), _i32(need)
    free, n_free = _i32(perm[sum(need):] + [-7] * sum(need)), _i32([2])
    pools = [_pool(g, n_pages, H, page, D, dtype, layout) for _ in range(LAYERS)]
    prob = nacl.Problem(B, H, L, D, dtype, [0], q_group=G)
    rotation = nacl.Rotation(prob)  # of nothing: kept rows are turned already

    for b, C in budget.items():
        n = int(lens[b])
        # The kept rows' slots: the sequence starts again with C new tokens, the others get none.
        start, new = lens.clone(), torch.zeros_like(lens)
        start[b], new[b] = 0, C
        step = nacl.Step(prob, C, lens=start, n_new=new)
        kept = []
        shape = nacl.Problem(1, H, n, D, dtype, list(range(n - P, n)), q_group=G)
        for layer, (k, v) in enumerate(pools):
            kc, vc = (_dense(x, table[b:b + 1], n).contiguous() for x in (k, v))
            q = torch.randn((1, HQ, n, D), generator=g).to(dt).to(DEV)
            _, keep, ko, vo = nacl.evict(shape, q, kc, vc, C, 8, seed=3, layer=layer)
            for x, y in ((kc, ko), (vc, vo)):
                assert torch.equal(y, x.gather(2, keep.long()[..., None].expand(-1, -1, -1, D)))
            kept.append((ko, vo))
        _, _, slots, missing = nacl.pages_assign(step, page, table, held, free, n_free, held_out=held, n_free_out=n_free)
        assert int(missing) == 0
        for (k, v), (ko, vo) in zip(pools, kept):
            kn, vn = (torch.zeros((B, H, C, D), dtype=dt, device=DEV) for _ in range(2))
            kn[b], vn[b] = ko[0], vo[0]
            unused = torch.empty((B, HQ, C, D), dtype=dt, device=DEV)
            nacl.paged_append(prob, step, rotation, None, unused, kn, vn, nacl.Pages(prob, k, v, table), slots, q_out=unused)
        lens[b] = C
        for (k, v), (ko, vo) in zip(pools, kept):
            assert torch.equal(_dense(k, table, L)[b, :, :C], ko[0]) and torch.equal(_dense(v, table, L)[b, :, :C], vo[0])
    used = [-(-int(n) // page) for n in lens]
    assert held.tolist() == used and int(n_free) == n_pages - sum(used)

    # The freed pages take a new sequence's prompt, and all attend to what they hold.
    T = int(n_free) * page - page  # (the others' next tokens may take a page each)
    T = min(T, L)
    new = _i32([1, 1, 1, T])
    step = nacl.Step(prob, T, lens=lens, n_new=new)
    before = [[x.clone() for x in (_dense(k, table, L), _dense(v, table, L))] for k, v in pools]
    _, _, slots, missing = nacl.pages_assign(step, page, table, held, free, n_free, held_out=held, n_free_out=n_free)
    ok = [b for b in range(B) if (slots[b, :int(new[b])] >= 0).all()]
    assert len(ok) >= 3 and (int(missing) == 0) == (len(ok) == B)
    pages_now = [e for b in range(B) for e in table[b, :int(held[b])].tolist()] + free[:int(n_free)].tolist()
    assert sorted(pages_now) == list(range(n_pages))
    for (k, v), (kb, vb) in zip(pools, before):
        q, kn, vn = (torch.randn((B, h, T, D), generator=g).to(dt).to(DEV) for h in (HQ, H, H))
        pages = nacl.Pages(prob, k, v, table)
        q = nacl.paged_append(prob, step, rotation, None, q, kn, vn, pages, slots)
        out, lse = nacl.paged_attention(prob, step, q, pages)
        torch.cuda.synchronize()
        kd, vd = _dense(k, table, L), _dense(v, table, L)
        for b in ok:
            n = int(lens[b])
            assert torch.equal(kd[b, :, :n], kb[b, :, :n]) and torch.equal(vd[b, :, :n], vb[b, :, :n])
            assert torch.equal(kd[b, :, n:n + int(new[b])], kn[b, :, :int(new[b])])
        check_rows(q, kd, vd, None, None, lens.tolist(), None, out, lse, prob.c.sm_scale,
                   [(b, h, t) for b in ok for h in range(HQ) for t in {0, int(new[b]) - 1}], n_new=new.tolist())
