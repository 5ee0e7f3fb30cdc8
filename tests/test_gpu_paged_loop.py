"""Paged decoding with beams, as a program uses it: prompts whose full pages a
group's beams share, then steps that take pages, write the new tokens, attend, pick
the best continuations and let the beams take over what their parents hold, in two
layers.  Every step against references, and captured steps against eager ones."""

import numpy as np
import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from oracle.step import rotate
from test_gpu_beam import _check as check_beams
from test_gpu_paged import DEV, _dense, _f64
from test_gpu_prefix import check_rows

pytestmark = pytest.mark.gpu
GROUPS, W, H, G, D, V = 2, 3, 2, 2, 64, 400
B, HQ, PAGE, SHARED, TAIL, STEPS = GROUPS * W, H * G, 8, 4, 5, 7
ENTRIES = SHARED + 3
L, N_PAGES, LAYERS = ENTRIES * PAGE, GROUPS * SHARED + B * 3 + 1, 2


class Program:
    """Random weights: each token's projections come from a table, the logits from
    the layers' attention."""

    def __init__(self, seed=0):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).to(DEV)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        self.embed = r(LAYERS, V, HQ + 2 * H, D)
        self.head = r(LAYERS * HQ * D, V) * 0.1
        self.wq, self.wk = (1 + 0.2 * r(D) for _ in range(2))
        self.inv_freq = (10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float().to(DEV)
        self.prompt = torch.randint(0, V, (GROUPS, SHARED * PAGE + TAIL), generator=g).to(DEV)
        self.pools = [(r(N_PAGES, H, PAGE, D), r(N_PAGES, H, PAGE, D)) for _ in range(LAYERS)]
        # The groups' shared pages, then a stack of the others.
        perm = torch.randperm(N_PAGES, generator=g).int().to(DEV)
        self.table = torch.full((B, ENTRIES), -1, dtype=torch.int32, device=DEV)
        self.table[:, :SHARED] = perm[:GROUPS * SHARED].view(GROUPS, SHARED).repeat_interleave(W, dim=0)
        self.free = torch.zeros(N_PAGES, dtype=torch.int32, device=DEV)
        self.n_free = i32([N_PAGES - GROUPS * SHARED])
        self.free[:int(self.n_free)] = perm[GROUPS * SHARED:]
        self.lens, self.held = i32([SHARED * PAGE] * B), i32([SHARED] * B)
        self.shared = i32([0] + [SHARED] * (W - 1)).repeat(GROUPS)
        self.scores = torch.full((GROUPS, W), -float("inf"), device=DEV)
        self.scores[:, 0] = 0.0
        self.ended = torch.zeros((GROUPS, W), dtype=torch.int32, device=DEV)
        self.token = self.prompt[:, -1].repeat_interleave(W).clone()
        self.prob = nacl.Problem(B, H, L, D, "bf16", [0], q_group=G)
        self.step = nacl.Step(self.prob, 1, lens=self.lens)
        self.rotation = nacl.Rotation(self.prob, self.inv_freq, self.wq, self.wk)
        self.pages = [nacl.Pages(self.prob, k, v, self.table) for k, v in self.pools]
        self.out = [(torch.empty((B, HQ, 1, D), dtype=torch.bfloat16, device=DEV), torch.empty((B, HQ, 1), device=DEV))
                    for _ in range(LAYERS)]
        self.q = [torch.empty((B, HQ, 1, D), dtype=torch.bfloat16, device=DEV) for _ in range(LAYERS)]
        self.slots, self.missing = torch.empty((B, 1), dtype=torch.int32, device=DEV), i32([0])
        self.ws = nacl.paged_workspace(self.prob, self.step, self.pages[0])
        self.bws = nacl.beam_workspace(GROUPS, W, V, W, DEV)
        self.best = [torch.empty((GROUPS, W), dtype=t, device=DEV) for t in (torch.int32, torch.int32, torch.float32)]
        self.next = [torch.empty_like(t) for t in (self.table, self.lens, self.held)]

    def split(self, layer, tokens):
        x = self.embed[layer][tokens].permute(0, 2, 1, 3)
        return x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]

    def prefill(self):
        """The prompts' full pages by one beam of each group, then what is left by all."""
        n = SHARED * PAGE
        for tokens, rows, slots in ((self.prompt[:, :n], slice(0, B, W), None),
                                    (self.prompt[:, n:].repeat_interleave(W, dim=0), slice(0, B), self.slots)):
            T, b = tokens.shape[1], len(range(B)[rows])
            prob = nacl.Problem(b, H, L, D, "bf16", [0], q_group=G)
            lens = torch.full((b,), 0 if slots is None else n, dtype=torch.int32, device=DEV)
            step = nacl.Step(prob, T, lens=lens)
            table = self.table[rows].contiguous() if slots is None else self.table
            if slots is None:
                j = torch.arange(T, device=DEV)
                at = (table[:, j // PAGE] * PAGE + j % PAGE).int()
            else:
                _, _, at, missing = nacl.pages_assign(step, PAGE, table, self.held, self.free, self.n_free, shared=self.shared,
                                                      held_out=self.held, n_free_out=self.n_free)
                assert int(missing) == 0
            pos = (torch.arange(T, device=DEV) + int(lens[0])).int()
            for layer, (k, v) in enumerate(self.pools):
                pages = nacl.Pages(prob, k, v, table)
                q = nacl.paged_append(prob, step, nacl.Rotation(prob, self.inv_freq, self.wq, self.wk), pos,
                                      *self.split(layer, tokens), pages, at)
                out, lse = nacl.paged_attention(prob, step, q, pages)
                torch.cuda.synchronize()
                check_rows(q, _dense(k, table, L), _dense(v, table, L), None, None, lens.tolist(), None, out, lse,
                           prob.c.sm_scale, [(i, h, t) for i in range(b) for h in range(HQ) for t in (0, T - 1)])
        self.lens += TAIL

    def one(self):
        nacl.pages_assign(self.step, PAGE, self.table, self.held, self.free, self.n_free, shared=self.shared, held_out=self.held,
                          n_free_out=self.n_free, slots=self.slots, missing=self.missing)
        for layer, pages in enumerate(self.pages):
            q, kn, vn = self.split(layer, self.token[:, None])
            nacl.paged_append(self.prob, self.step, self.rotation, self.lens[:, None], q, kn, vn, pages, self.slots, q_out=self.q[layer])
            nacl.paged_attention(self.prob, self.step, self.q[layer], pages, out=self.out[layer][0], lse=self.out[layer][1], ws=self.ws)
        self.logits = torch.cat([o.view(B, HQ * D) for o, _ in self.out], dim=1) @ self.head
        nacl.beam_select(self.logits, self.scores, W, ended=self.ended, end_token=7, parents=self.best[0], tokens=self.best[1],
                         out=self.best[2], ws=self.bws)
        self.lens += 1

    def take_over(self):
        table, lens, held = self.next
        for pages in self.pages:
            nacl.beam_reorder(self.prob, pages, self.best[0], self.lens, held=self.held, table_out=table, lens_out=lens, held_out=held)
        for old, new in ((self.table, table), (self.lens, lens), (self.held, held), (self.scores, self.best[2])):
            old.copy_(new)
        self.ended.copy_(self.ended.gather(1, self.best[0].long()) | (self.best[1] == 7))
        self.token.copy_(self.best[1].view(-1))


def _rows(p, layer, b):
    """What sequence b holds, from its pages."""
    n = int(p.lens[b])
    return [x[b, :, :n].clone() for x in (_dense(p.pools[layer][0], p.table, L), _dense(p.pools[layer][1], p.table, L))]


def _pages_are_dealt_once(p):
    free = p.free[:int(p.n_free)].tolist()
    own = [e for b in range(B) for e in p.table[b, SHARED:int(p.held[b])].tolist()]
    shared = [e for b in range(0, B, W) for e in p.table[b, :SHARED].tolist()]
    assert sorted(free + own + shared) == list(range(N_PAGES))
    for b in range(B):
        assert p.table[b, :SHARED].tolist() == p.table[b // W * W, :SHARED].tolist()


def test_steps_against_references():
    p = Program()
    p.prefill()
    _pages_are_dealt_once(p)
    for _ in range(STEPS):
        before = [[_rows(p, layer, b) for b in range(B)] for layer in range(LAYERS)]
        token, lens, scores, ended = p.token.clone(), p.lens.clone(), p.scores.clone(), p.ended.clone()
        p.one()
        torch.cuda.synchronize()
        assert int(p.missing) == 0
        _pages_are_dealt_once(p)
        for layer in range(LAYERS):
            q, kn, vn = p.split(layer, token[:, None])
            for b in range(B):
                n = int(lens[b])
                k, v = _rows(p, layer, b)
                assert torch.equal(k[:, :n], before[layer][b][0]) and torch.equal(v[:, :n], before[layer][b][1])
                assert torch.equal(v[:, n], vn[b, :, 0])
                for h in range(H):
                    ref = rotate(_f64(kn[b, h]), [n], p.inv_freq.cpu().numpy(), _f64(p.wk), 1e-6)[0]
                    size = np.abs(ref) + np.abs(np.roll(ref, D // 2))
                    assert (np.abs(_f64(k[h, n]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * size).all()
            check_rows(p.q[layer], _dense(p.pools[layer][0], p.table, L), _dense(p.pools[layer][1], p.table, L), None, None,
                       lens.tolist(), None, *p.out[layer], p.prob.c.sm_scale, [(b, h, 0) for b in range(B) for h in range(HQ)])
        check_beams(p.logits, scores, W, p.best, ended, 7)
        held = [[_rows(p, layer, b) for b in range(B)] for layer in range(LAYERS)]
        source = (torch.arange(GROUPS, device=DEV)[:, None] * W + p.best[0]).view(-1).tolist()
        p.take_over()
        torch.cuda.synchronize()
        _pages_are_dealt_once(p)
        for layer in range(LAYERS):
            for b in range(B):
                for x, y in zip(_rows(p, layer, b), held[layer][source[b]]):
                    assert torch.equal(x, y)
    # The end: all pages go back, the shared ones once.
    p.lens.zero_()
    nacl.pages_assign(p.step, PAGE, p.table, p.held, p.free, p.n_free, shared=p.shared, held_out=p.held, n_free_out=p.n_free)
    p.held.zero_()
    step = nacl.Step(p.prob, 1, n_new=torch.zeros(B, dtype=torch.int32, device=DEV))
    p.held.fill_(1)
    nacl.pages_assign(step, PAGE, p.table, p.held, p.free, p.n_free, shared=p.shared, held_out=p.held, n_free_out=p.n_free)
    assert sorted(p.free.tolist()) == list(range(N_PAGES)) and int(p.n_free) == N_PAGES


STATE = ("table", "free", "n_free", "lens", "held", "scores", "ended", "token")


def test_captured_steps_equal_eager_ones():
    """A captured step replayed, with the program's own eager work between."""
    eager, captured = Program(1), Program(1)
    for p in (eager, captured):
        p.prefill()
    state = [getattr(captured, x) for x in STATE] + [t for kv in captured.pools for t in kv]
    saved = [t.clone() for t in state]

    def whole():
        captured.one()
        captured.take_over()

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        whole()  # allocations and library handles before the capture
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        whole()
    for t, s in zip(state, saved):
        t.copy_(s)
    for i in range(STEPS):
        eager.one()
        eager.take_over()
        graph.replay()
        torch.cuda.synchronize()
        for x in STATE:
            assert torch.equal(getattr(eager, x), getattr(captured, x)), (i, x)
        for x, y in zip(eager.pools, captured.pools):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
        assert all(torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) for x, y in zip(eager.out, captured.out))


def test_two_programs_on_two_streams():
    """Two programs under way at once, each on a stream and with workspaces of its own."""
    def run(p):
        p.one()
        p.take_over()
        return [getattr(p, x).clone() for x in STATE] + [t.clone() for o in p.out for t in o]

    def made(seed):
        p = Program(seed)
        p.prefill()
        return p

    alone = [[run(p) for _ in range(STEPS)] for p in (made(1), made(2))]
    programs, streams, logs = [made(1), made(2)], [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(STEPS):
        for p, st, log in zip(programs, streams, logs):
            with torch.cuda.stream(st):
                log.append(run(p))
    torch.cuda.synchronize()
    for log, ref in zip(logs, alone):
        for got, want in zip(log, ref):
            assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_pages_follow_their_tensors():
    """Pools and a table that get another storage between two calls are read where they are then."""
    p = Program(3)
    p.prefill()
    k, v = p.pools[0]
    want = [t.clone() for t in nacl.paged_attention(p.prob, p.step, p.q[0].fill_(1), p.pages[0])]
    for t in (k, v, p.table):
        t.data = t.data.clone()
    for t, y in zip(nacl.paged_attention(p.prob, p.step, p.q[0], p.pages[0]), want):
        assert torch.equal(t, y)
    k.data = k.data[:, :, :PAGE // 2].contiguous()
    with pytest.raises(ValueError):
        nacl.paged_attention(p.prob, p.step, p.q[0], p.pages[0])


def test_ended_beams_need_an_end_token():
    x, scores, ended = torch.zeros((2, 50), device=DEV), torch.zeros((1, 2), device=DEV), torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    for token in (None, -1, 50):
        with pytest.raises(ValueError, match="end_token"):
            nacl.beam_select(x, scores, 2, ended=ended, end_token=token)


@pytest.mark.parametrize("name", ["shared", "missing", "lse", "ended", "held", "held_out"])
def test_an_optional_tensor_without_memory_is_refused(name):
    """Its null address would mean that it was not given."""
    p = Program(5)
    t = dict(shared=p.shared, missing=p.missing, lse=p.out[0][1], ended=p.ended, held=p.held.clone(), held_out=p.next[2])[name]
    t.untyped_storage().resize_(0)
    with pytest.raises(ValueError, match="no memory"):
        if name in ("shared", "missing"):
            nacl.pages_assign(p.step, PAGE, p.table, p.held, p.free, p.n_free, **{name: t})
        elif name == "lse":
            nacl.paged_attention(p.prob, p.step, p.q[0], p.pages[0], lse=t)
        elif name == "ended":
            nacl.beam_select(torch.zeros((B, V), device=DEV), p.scores, W, ended=t, end_token=7)
        else:
            nacl.beam_reorder(p.prob, p.pages[0], p.best[0].zero_(), p.lens, **{"held": p.held, name: t})


def test_a_used_workspace_of_any_contents():
    p = Program(4)
    p.prefill()
    want = [t.clone() for t in nacl.paged_attention(p.prob, p.step, p.q[0].fill_(1), p.pages[0])]
    x = torch.randn((B, V), device=DEV)
    best = [t.clone() for t in nacl.beam_select(x, p.scores, W)]
    for fill in (0, 255, 127):
        p.ws.fill_(fill)
        p.bws.fill_(fill)
        for t, y in zip(nacl.paged_attention(p.prob, p.step, p.q[0], p.pages[0], ws=p.ws), want):
            assert torch.equal(t, y)
        for t, y in zip(nacl.beam_select(x, p.scores, W, ws=p.bws), best):
            assert torch.equal(t, y)
