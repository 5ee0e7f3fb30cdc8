"""nacl_paged_attention where the table is wider than the sequences: as many
work-groups at work as under a table of the sequences' own width, and splits that go
several times round a sequence's blocks of keys."""

import math

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_paged import _attend_case, _check_seen, _dense
from test_gpu_prefix import DEV, DT, _rows, check_rows

pytestmark = pytest.mark.gpu


def _parts(B, H, G, T, D, page, dtype, n, width):
    """Partial results per query row of sequences of n rows under a table of `width`
    rows: what a call leaves of the numbers that its workspace was filled with."""
    entries, own = -(-width // page), -(-n // page)
    k = torch.zeros((own, H, page, D), dtype=DT[dtype], device=DEV)
    table = torch.full((B, entries), -1, dtype=torch.int32, device=DEV)
    table[:, :own] = torch.arange(own, dtype=torch.int32, device=DEV)  # (pages may be shared)
    q = torch.zeros((B, H * G, T, D), dtype=DT[dtype], device=DEV)
    prob = nacl.Problem(B, H, width, D, dtype, [0], q_group=G)
    step = nacl.Step(prob, T, lens=torch.full((B,), n - T, dtype=torch.int32, device=DEV))
    pages = nacl.Pages(prob, k, k, table)
    ws = nacl.paged_workspace(prob, step, pages)
    if ws.numel() <= 256:
        return 1.0  # one part, the output itself
    words = ws.view(torch.int32)
    words.fill_(-1)
    nacl.paged_attention(prob, step, q, pages, ws=ws)
    torch.cuda.synchronize()
    return int((words != -1).sum()) / (B * H * G * T * (D + 2))


@pytest.mark.parametrize("B,H,G,T,D,page,dtype,n", [
    (1, 8, 4, 1, 128, 16, "bf16", 2112), (8, 8, 4, 1, 128, 16, "bf16", 4000), (32, 8, 4, 1, 128, 64, "bf16", 600),
    (6, 4, 2, 5, 64, 27, "f32", 1999), (4, 8, 4, 8, 64, 16, "bf16", 8000), (1, 8, 4, 128, 128, 16, "bf16", 4096),
    (1, 2, 2, 100, 64, 33, "f32", 1000),
])
def test_work_follows_the_lengths(B, H, G, T, D, page, dtype, n):
    own = _parts(B, H, G, T, D, page, dtype, n, n)
    for width in (8 * n, 131072):
        assert _parts(B, H, G, T, D, page, dtype, n, width) >= 0.75 * own


#        B   H  G  T   L      D    page dtype  layout
WIDE = [
    (9, 8, 4, 1, 4500, 128, 16, "bf16", "heads"),
    (9, 8, 4, 1, 4500, 64, 37, "f32", "rows"),
    (5, 8, 3, 5, 3000, 64, 27, "f32", "side"),
    (5, 8, 4, 3, 6000, 128, 16, "bf16", "rows"),
    (4, 8, 4, 6, 5000, 128, 16, "bf16", "heads"),
    (3, 8, 2, 50, 3000, 64, 5, "bf16", "one"),
    (3, 8, 4, 70, 3000, 128, 64, "bf16", "heads"),
    (2, 8, 2, 40, 2500, 128, 16, "f32", "heads"),
]


@pytest.mark.parametrize("case", WIDE, ids=str)
def test_sequences_of_every_length_under_one_table(case):
    """From none to all of the table's rows: several rounds of a split's blocks, splits
    without any, last blocks of a part."""
    B, H, G, T, L, D, page, dtype, layout = case
    q, k, v, table, lens = _attend_case(*case, seed=L)
    for i, n in enumerate((L - T, 0, L // 2 + 1, 127, 640)[:B]):
        lens[i] = n
    n_new = torch.full((B,), T, dtype=torch.int32)
    n_new[-1] = T // 2
    prob = nacl.Problem(B, H, L, D, dtype, [0], q_group=G)
    step = nacl.Step(prob, T, lens=lens.to(DEV), n_new=n_new.to(DEV))
    pages = nacl.Pages(prob, k, v, table)
    ws = nacl.paged_workspace(prob, step, pages)
    ws.fill_(255)  # NaN
    out, lse = nacl.paged_attention(prob, step, q, pages, ws=ws)
    torch.cuda.synchronize()
    check_rows(q, _dense(k, table, L), _dense(v, table, L), None, None, lens, None, out, lse, prob.c.sm_scale,
               _rows(B, H * G, T, 60), n_new=n_new.tolist())


@pytest.mark.parametrize("dtype,G,T,page", [("bf16", 2, 3, 16), ("bf16", 4, 6, 27), ("bf16", 4, 60, 16), ("f32", 2, 6, 16)])
def test_hidden_rows_of_long_sequences(dtype, G, T, page):
    """Later tokens' rows with NaN and infinities, which the tokens before do not see,
    where the splits go several times round the blocks."""
    B, H, L, D = 4, 8, 9000, 64
    q, k, v, table, lens = _attend_case(B, H, G, T, L, D, page, dtype, seed=page)
    lens[:] = torch.tensor([L - T, 4000, 127, 1000 - T])
    for b in range(B):
        at = int(lens[b]) + 1  # the row of token 1
        k[int(table[b, at // page]), :, at % page] = math.nan
        v[int(table[b, at // page]), :, at % page] = -math.inf
    prob = nacl.Problem(B, H, L, D, dtype, [0], q_group=G)
    out, lse = nacl.paged_attention(prob, nacl.Step(prob, T, lens=lens.to(DEV)), q, nacl.Pages(prob, k, v, table))
    torch.cuda.synchronize()
    check_rows(q, _dense(k, table, L), _dense(v, table, L), None, None, lens, None, out, lse, prob.c.sm_scale,
               [(b, h, 0) for b in range(B) for h in range(H * G)])
    assert torch.isnan(out[:, :, 1:]).any(dim=3).all()


@pytest.mark.parametrize("dtype,G,T", [("bf16", 3, 1), ("bf16", 4, 5), ("bf16", 4, 60), ("f32", 3, 4), ("f32", 2, 12)])
def test_far_pools_and_long_sequences(dtype, G, T):
    """Pools past 4 GiB, pages outside the pool, several rounds."""
    B, H, D, page = 8, 8, 64, 1100
    g = torch.Generator().manual_seed(T)
    size = 1500 * 2 ** 20
    wide = [torch.zeros(4 * size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    k, v = (torch.as_strided(x.view(DT[dtype]), (4, H, page, D), (size // DT[dtype].itemsize, page * D, D, 1)) for x in wide)
    for x in (k, v):
        x.copy_(torch.randn((4, H, page, D), generator=g).to(DT[dtype]))
    q = torch.randn((B, H * G, T, D), generator=g).to(DT[dtype]).to(DEV)
    table = torch.stack([torch.randperm(4, generator=g) for _ in range(B)]).int()
    table[3, 1], table[4, 3] = -1, 4
    lens = torch.tensor([4400 - T, 0, 2000, 3300, 4000, 129, 1100, 700], dtype=torch.int32)
    prob = nacl.Problem(B, H, 4400, D, dtype, [0], q_group=G)
    step = nacl.Step(prob, T, lens=lens.to(DEV))
    out, lse = nacl.paged_attention(prob, step, q, nacl.Pages(prob, k, v, table.to(DEV)))
    torch.cuda.synchronize()
    _check_seen(q, k, v, table.to(DEV), lens, out, lse, prob.c.sm_scale)
