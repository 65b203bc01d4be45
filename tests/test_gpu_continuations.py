"""The operators for several continuations as they are used together: steps of beam search, steps with drafted tokens, captured into graphs, on streams of their own."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Searcher:
    """Beam search with one attention layer.  What the projections and the output layer would give are tables: a token's q, k and v by its number, the next token's logits
    by the token before it, so that the choice can be followed exactly and each attention checked against its definition."""

    def __init__(self, prompts, K, V, steps, H, H_kv, d, page, dtype, rot, seed, end_token=-1, spare=0):
        self.K, self.V, self.H, self.H_kv, self.d, self.page, self.dtype, self.end_token = K, V, H, H_kv, d, page, dtype, end_token
        gen = torch.Generator().manual_seed(seed)
        self.prompts = [torch.randint(V, (n,), generator=gen).tolist() for n in prompts]
        self.q_of, self.k_of, self.v_of = (sv.normal(V, h, d, seed=seed + i, dtype=dtype) for i, h in ((1, H), (2, H_kv), (3, H_kv)))
        self.logits_of = sv.normal(V, V, seed=seed + 4, dtype=torch.float32, std=2.0)
        self.freq = sv.frequencies(rot) if rot else None
        B = len(prompts)
        self.B = B
        wide = -(-(max(prompts) + steps + 1) // page)
        n_pages = sum(-(-n // page) for n in prompts) + B * K * (-(-steps // page) + 2) + spare
        self.kc, self.vc = (torch.full((n_pages, page, H_kv, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
        self.wide, self.n_pages = wide, n_pages
        self.gpu = [x.cuda() for x in (self.q_of, self.k_of, self.v_of, self.logits_of)]
        self.gpu_freq = None if self.freq is None else self.freq.cuda()

    def start(self):
        # pages for the prompts out of nothing, and their tokens into them
        table, lengths, missing = lss.lss_paged_fork(self.kc, self.vc, torch.empty(0, self.wide, dtype=torch.int32, device="cuda"), _i32([]), _i32([-1] * self.B),
                                                     room=_i32([len(p) for p in self.prompts]))
        assert int(missing) == 0 and lengths.tolist() == [len(p) for p in self.prompts]
        at = torch.tensor(sum(self.prompts, []), device="cuda")
        cu = sv.starts([len(p) for p in self.prompts]).cuda()
        lss.lss_paged_append(self.gpu[1][at], self.gpu[2][at], self.kc, self.vc, table, lengths, cu, q=self.gpu[0][at], inv_freq=self.gpu_freq)
        # every beam is its prompt at first, only one of them is alive
        self.table, self.lengths, missing = lss.lss_paged_fork(self.kc, self.vc, table, lengths, _i32([b for b in range(self.B) for _ in range(self.K)]),
                                                               room=_i32([0] * (self.B * self.K)))
        assert int(missing) == 0
        self.scores = torch.full((self.B, self.K), -math.inf, device="cuda")
        self.scores[:, 0] = 0.0
        self.finished = torch.zeros(self.B, self.K, dtype=torch.bool, device="cuda")
        self.tokens = torch.tensor([p[-1] for p in self.prompts for _ in range(self.K)], device="cuda").view(self.B, self.K)

    def step(self):
        """One step; returns the attention's (out, lse) of the tokens that were chosen"""
        logits = self.gpu[3][self.tokens.flatten().clamp(min=0).long()]
        ended = dict(finished=self.finished, end_token=self.end_token) if self.end_token >= 0 else {}
        self.scores, self.parents, self.tokens, fin = lss.lss_beam_select(logits, self.scores, **ended)
        if fin is not None:
            self.finished = fin
        self.table, self.lengths, self.missing = lss.lss_paged_fork(self.kc, self.vc, self.table, self.lengths, self.parents)
        at = self.tokens.flatten().long()
        q, _ = lss.lss_paged_append(self.gpu[1][at], self.gpu[2][at], self.kc, self.vc, self.table, self.lengths, q=self.gpu[0][at], inv_freq=self.gpu_freq)
        return lss.lss_paged_attn_decode(q, self.kc, self.vc, self.table, self.lengths)

    def rows(self, tokens):
        p = torch.arange(len(tokens))
        q, k = (sv.rotate(x[tokens], p, self.freq, False)[0].to(self.dtype) for x in (self.q_of, self.k_of))
        return q, k, self.v_of[tokens]


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("K,H,H_kv,d,page,rot,end_token", [(4, 8, 2, 64, 16, 0, -1), (3, 4, 4, 128, 32, 0, 5), (8, 6, 1, 64, 16, 0, 11)])
def test_beam_search(dtype, K, H, H_kv, d, page, rot, end_token):
    s = Searcher([5, 16, 33, 1], K, 40, 40, H, H_kv, d, page, dtype, rot, seed=1, end_token=end_token)
    s.start()
    histories = [[list(p) for _ in range(K)] for p in s.prompts]
    scores = torch.full((s.B, K), -math.inf)
    scores[:, 0] = 0.0
    finished = torch.zeros(s.B, K, dtype=torch.bool)
    for step in range(40):
        out, lse = s.step()
        # the choice, from the scores that the kernel left (its own rounding of them to 32 bits is not what is meant here)
        logits = s.logits_of[[h[-1] for hs in histories for h in hs]]
        want = co.select(logits, scores, K, finished if end_token >= 0 else None, end_token)
        parents, tokens = s.parents.cpu().long(), s.tokens.cpu().long()
        if want[4] > 2 * co.LSE_BOUND:
            assert torch.equal(parents, want[1]) and torch.equal(tokens, want[2]), step
        else:
            # (totals of two beams nearer than what they may be off by: either order; the choice is as good as the best within that, nothing is chosen twice)
            for b in range(s.B):
                chosen = list(zip(parents[b].tolist(), tokens[b].tolist()))
                assert len(set(chosen)) == K
                for i, (p, v) in enumerate(chosen):
                    ended = end_token >= 0 and bool(finished[b, p - b * K])
                    total = float(scores[b, p - b * K]) + (0.0 if ended else float(torch.log_softmax(logits[p].double(), 0)[v]))
                    assert (not ended or v == end_token) and abs(total - float(want[0][b, i])) <= 2 * co.LSE_BOUND
        sv.check(s.scores, want[0], 3 * co.LSE_BOUND + 2.0 ** -24 * want[0].abs(), "scores")
        scores = s.scores.cpu()
        if end_token >= 0:
            finished = s.finished.cpu()
            assert torch.equal(finished, tokens == end_token)
        histories = [[histories[b][int(parents[b, i]) - b * K] + [int(tokens[b, i])] for i in range(K)] for b in range(s.B)]
        # the pages: each beam's cache holds its history, whatever the others wrote
        assert int(s.missing) == 0
        flat = [h for hs in histories for h in hs]
        assert s.lengths.tolist() == [len(h) for h in flat]
        if step % 13 == 12 or step < 3:
            for i, h in enumerate(flat):
                q, k, v = s.rows(h)
                for head in range(H):
                    g = head // (H // H_kv)
                    o, l, ob, lb = sv.attention(q[-1:, head], k[:, g], v[:, g], torch.tensor([len(h)]), dtype)
                    sv.check(out[i:i + 1, head], o, ob, f"out of beam {i}")
                    sv.check(lse[i:i + 1, head], l, lb, f"lse of beam {i}")
    # no page is lost: those that the tables name and no others are in use
    used = {int(x) for row in s.table.tolist() for x in row if x >= 0}
    assert len(used) < s.n_pages


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("H,H_kv,d,page,rot", [(8, 2, 64, 16, 64), (4, 4, 128, 32, 64), (12, 1, 64, 16, 48)])
def test_drafted_trees(dtype, H, H_kv, d, page, rot):
    # a path of every step's tree is accepted; then the cache holds what appending the path's tokens one by one would have put there, bit for bit, and every drafted token's
    # attention was that over its own path
    gen = torch.Generator().manual_seed(3)
    V, prompts, drafts = 50, [7, 30, 16, 1], [9, 1, 20, 6]
    q_of, k_of, v_of = (sv.normal(V, h, d, seed=20 + i, dtype=dtype) for i, h in ((1, H), (2, H_kv), (3, H_kv)))
    gpu = [x.cuda() for x in (q_of, k_of, v_of)]
    freq = sv.frequencies(rot)
    wide = -(-(max(prompts) + 6 * max(drafts)) // page)
    n_pages = 4 * wide
    kc, vc = (torch.full((n_pages, page, H_kv, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    table = torch.randperm(n_pages, generator=gen).to(torch.int32).view(4, wide).cuda()
    texts = [torch.randint(V, (n,), generator=gen).tolist() for n in prompts]
    lengths = _i32(prompts)
    at = torch.tensor(sum(texts, []), device="cuda")
    lss.lss_paged_append(gpu[1][at], gpu[2][at], kc, vc, table, lengths, sv.starts(prompts).cuda(), q=gpu[0][at], inv_freq=freq.cuda())
    for step in range(5):
        new = [max(1, n - step) for n in drafts]
        cu = sv.starts(new)
        bits, depth, tokens, paths = [], [], [], []
        for b, n in enumerate(new):
            parents = [-1] + [int(torch.randint(-1, i, (), generator=gen)) for i in range(1, n)]
            seen, deep, path = [], [], []
            for i, p in enumerate(parents):
                seen.append((1 << i) | (seen[p] if p >= 0 else 0))
                deep.append(deep[p] + 1 if p >= 0 else 0)
                path.append((path[p] if p >= 0 else []) + [i])
            bits += seen
            depth += [len(texts[b]) + x for x in deep]
            tokens.append(torch.randint(V, (n,), generator=gen).tolist())
            paths.append(path)
        flat = torch.tensor(sum(tokens, []), device="cuda")
        lengths = lengths + _i32(new)
        q, _ = lss.lss_paged_append(gpu[1][flat], gpu[2][flat], kc, vc, table, lengths, cu.cuda(), q=gpu[0][flat], inv_freq=freq.cuda(), positions=_i32(depth))
        out, lse = lss.lss_paged_attn_tree(q, kc, vc, table, lengths, cu.cuda(), tree=co.to_bits(bits, 1).cuda())
        for b, n in enumerate(new):
            for i in range(n):
                history = texts[b] + [tokens[b][j] for j in paths[b][i]]
                p = torch.arange(len(history))
                k = sv.rotate(k_of[history], p, freq, False)[0].to(dtype)
                qr = q[int(cu[b]) + i].cpu()                # (checked by itself elsewhere: rotated by the token's depth)
                for head in range(H):
                    g = head // (H // H_kv)
                    o, l, ob, lb = sv.attention(qr[None, head], k[:, g], v_of[history][:, g], torch.tensor([len(history)]), dtype)
                    # (a rotated key next to a border may be kept as its other neighbour: the slack of test_gpu_serving.test_prompts_then_tokens)
                    few = 16 * sv.HALF[dtype] * (q_of.double().abs().amax() * k_of.double().abs().amax()) * (8 if dtype == torch.float32 else 1) / d ** 0.5
                    sv.check(out[int(cu[b]) + i:int(cu[b]) + i + 1, head], o, ob + 2 * few * v_of.double().abs().amax(), f"out of drafted token {i} of sequence {b}")
                    sv.check(lse[int(cu[b]) + i:int(cu[b]) + i + 1, head], l, lb + few, f"lse of drafted token {i} of sequence {b}")
        # the deepest path is accepted, of one sequence none of it
        kept = [max(path, key=len) if b != step % 4 else [] for b, path in enumerate(paths)]
        lists = torch.zeros(4, max(map(len, kept)), dtype=torch.int32)
        for b, path in enumerate(kept):
            lists[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
            texts[b] = texts[b] + [tokens[b][j] for j in path]
        lengths = lss.lss_paged_compact(kc, vc, table, lengths, cu.cuda(), lists.cuda(), _i32([len(x) for x in kept]))
        assert lengths.tolist() == [len(t) for t in texts]
        # one by one into another cache
        k2, v2 = torch.full_like(kc, math.nan), torch.full_like(vc, math.nan)
        at = torch.tensor(sum(texts, []), device="cuda")
        lss.lss_paged_append(gpu[1][at], gpu[2][at], k2, v2, table, lengths, sv.starts([len(t) for t in texts]).cuda(), inv_freq=freq.cuda())
        for b, t in enumerate(texts):
            rows = torch.tensor([int(table[b, p // page]) * page + p % page for p in range(len(t))], device="cuda")
            for x, y in ((kc, k2), (vc, v2)):
                assert torch.equal(sv.bits(x.view(-1, H_kv, d)[rows]), sv.bits(y.view(-1, H_kv, d)[rows])), (step, b)


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_positions_of_appended_tokens(dtype):
    # positions of their own, in any order, far and below 0; rows of no sequence; places as ever
    new, lengths, rows = [3, 0, 5, 1], [3, 9, 40, 17], 11
    table, n_pages = sv.tables(lengths, 16, 5, extra=1)
    k, v, q = (sv.normal(rows, h, 64, seed=6 + h, dtype=dtype) for h in (2, 3, 4))
    v = sv.normal(rows, 2, 64, seed=60, dtype=dtype)
    positions = torch.tensor([7, 0, 2 ** 20 - 3, -5, 3, 3, 100, 2, 2 ** 31 - 1, -2 ** 31, 1], dtype=torch.int32)
    freq = sv.frequencies(64)
    kc, vc = (torch.full((n_pages, 16, 2, 64), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    q_rot, k_rot = (torch.full(x.shape, 7.0, dtype=dtype, device="cuda") for x in (q, k))
    cu = sv.starts(new)
    args = (table.cuda(), _i32(lengths), cu.cuda())
    lss.lss_paged_append(k.cuda(), v.cuda(), kc, vc, *args, q=q.cuda(), inv_freq=freq.cuda(), q_rot=q_rot, k_rot=k_rot, positions=positions.cuda())
    # angles of far positions: the argument is taken in 64 bits, as for places
    for x, got in ((q, q_rot), (k, k_rot)):
        want, slack = sv.rotate(x[:9], positions[:9], freq, False)
        sv.check(got[:9], want, slack + sv.HALF[dtype] * want.abs(), "rotated")
        assert bool((got[9:] == 7.0).all())
    at = 0
    for b, n in enumerate(new):
        for i in range(n):
            p = lengths[b] - n + i
            place = int(table[b, p // 16]), p % 16
            assert torch.equal(sv.bits(kc[place]), sv.bits(k_rot[at])) and torch.equal(sv.bits(vc[place]), sv.bits(v[at]))
            at += 1
    with pytest.raises(ValueError, match="positions must have one entry"):
        lss.lss_paged_append(k.cuda(), v.cuda(), kc, vc, *args, positions=positions[:5].cuda())
    # the places themselves are what there is without positions
    own = torch.cat([torch.arange(n - m, n) for m, n in zip(new, lengths)] + [torch.zeros(2, dtype=torch.long)]).int()
    a = lss.lss_paged_append(k.cuda(), v.cuda(), kc, vc, *args, q=q.cuda(), inv_freq=freq.cuda(), k_rot=torch.empty_like(k_rot), positions=own.cuda())
    b = lss.lss_paged_append(k.cuda(), v.cuda(), kc, vc, *args, q=q.cuda(), inv_freq=freq.cuda(), k_rot=torch.empty_like(k_rot))
    assert torch.equal(sv.bits(a[0][:9]), sv.bits(b[0][:9])) and torch.equal(sv.bits(a[1][:9]), sv.bits(b[1][:9]))


def test_captured_steps_of_beam_search():
    # two graphs of different shapes, each a whole step on tables that its replay leaves for the next, share what scratch the binding keeps; against eager steps on copies
    made = []
    for seed, (prompts, K, V, H, H_kv, d, page) in enumerate((([300, 20, 700], 4, 300, 8, 2, 64, 16), ([1, 90], 8, 9000, 4, 4, 128, 32))):
        s, e = (Searcher(prompts, K, V, 30, H, H_kv, d, page, torch.bfloat16, 64, seed=30 + seed, end_token=3) for _ in range(2))
        s.start(), e.start()
        names = ("table", "lengths", "scores", "finished", "tokens")
        kept = {n: getattr(s, n).clone() for n in names}
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):               # (a step ahead of the capture, then everything as it was)
            s.step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        s.kc.copy_(e.kc), s.vc.copy_(e.vc)
        for n in names:
            setattr(s, n, kept[n])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = s.step()
            after = {n: getattr(s, n) for n in names}
            for n in names:                         # what the next replay begins with
                kept[n].copy_(after[n])
        made.append((s, e, graph, kept, out, lse))
    for _ in range(7):
        for s, e, graph, kept, out, lse in made:
            out.fill_(3.0), lse.fill_(3.0)
            graph.replay()
            want = e.step()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            for n, x in kept.items():
                assert torch.equal(x, getattr(e, n)), n
            assert torch.equal(sv.bits(s.kc), sv.bits(e.kc)) and torch.equal(sv.bits(s.vc), sv.bits(e.vc))


def test_captured_steps_with_drafted_tokens():
    # append, attention and compaction in a graph, trees and lengths new for each replay; both kernels of the attention
    for dtype, H, H_kv, n in ((torch.bfloat16, 16, 2, 24), (torch.float32, 4, 4, 6)):
        B, d, page, wide = 5, 64, 16, 80
        gen = torch.Generator().manual_seed(7)
        state = {}
        for name in "se":
            kc, vc = (sv.normal(B * wide, page, H_kv, d, seed=i, dtype=dtype).cuda() for i in (1, 2))
            state[name] = (kc, vc)
        table = torch.randperm(B * wide, generator=gen).to(torch.int32).view(B, wide).cuda()
        cu = sv.starts([n] * B).cuda()
        q, k, v = (sv.normal(B * n, h, d, seed=5 + h, dtype=dtype).cuda() for h in (H, H_kv, H_kv))
        lengths, bits, positions = _i32([n + 5] * B), torch.zeros(B * n, 1, dtype=torch.int64, device="cuda"), _i32([0] * (B * n))
        kept, n_kept = _i32([[0] * 4] * B), _i32([0] * B)
        freq = sv.frequencies(64).cuda()

        def step(kc, vc):
            qr, _ = lss.lss_paged_append(k, v, kc, vc, table, lengths, cu, q=q, inv_freq=freq, positions=positions)
            out, lse = lss.lss_paged_attn_tree(qr, kc, vc, table, lengths, cu, tree=bits)
            return out, lse, lss.lss_paged_compact(kc, vc, table, lengths, cu, kept, n_kept)

        step(*state["s"])
        state["s"][0].copy_(state["e"][0]), state["s"][1].copy_(state["e"][1])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step(*state["s"])
        for i in range(6):
            lens = torch.randint(n, 1200 if i % 2 else 60, (B,), generator=gen)
            lengths.copy_(lens)
            bits.copy_(torch.cat([co.random_tree(n, 1, gen) for _ in range(B)]))
            positions.copy_(torch.randint(0, 3000, (B * n,), generator=gen))
            kept.copy_(torch.stack([torch.randperm(n, generator=gen)[:4].sort()[0] for _ in range(B)]))
            n_kept.copy_(torch.randint(0, 5, (B,), generator=gen))
            q.copy_(sv.normal(B * n, H, d, seed=50 + i, dtype=dtype))
            for x in got:
                x.fill_(3)
            graph.replay()
            want = step(*state["e"])
            torch.cuda.synchronize()
            for x, y in zip((*got, *state["s"]), (*want, *state["e"])):
                assert torch.equal(x, y)


def test_streams_of_their_own():
    s, e = (Searcher([200, 31], 4, 200, 10, 4, 2, 64, 16, torch.bfloat16, 64, seed=50) for _ in range(2))
    e.start()
    want = [e.step() for _ in range(3)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.start()
        got = [s.step() for _ in range(3)]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(s.table, e.table) and torch.equal(s.scores, e.scores)
    # ... and one that is passed instead of the current one, for each of them
    logits = torch.randn(8, 5000, device="cuda")
    scores = torch.zeros(2, 4, device="cuda")
    q = sv.normal(16, 4, 64, seed=60).cuda()
    cu, parents = _i32([0, 2, 4, 6, 8, 10, 12, 14, 16]), _i32([0, 0, 1, 2, 4, 4, 4, 7])
    lists, counts = _i32([[1]] * 8), _i32([1] * 8)
    torch.cuda.synchronize()
    for x in (s, e):
        x.got = []
        kw = dict(stream=side) if x is s else {}
        x.got += lss.lss_beam_select(logits, scores, **kw)[:3]
        x.got += lss.lss_paged_attn_tree(q, x.kc, x.vc, x.table, x.lengths, cu, **kw)
        x.got += lss.lss_paged_fork(x.kc, x.vc, x.table, x.lengths, parents, **kw)
        x.got.append(lss.lss_paged_compact(x.kc, x.vc, x.table, x.lengths, cu, lists, counts, **kw))
        side.synchronize()
        torch.cuda.synchronize()
    for a, b in zip((*s.got, s.kc, s.vc), (*e.got, e.kc, e.vc)):
        assert torch.equal(a.nan_to_num() if a.is_floating_point() else a, b.nan_to_num() if b.is_floating_point() else b)


def test_two_calls_at_once_with_scratch_of_their_own():
    q, table, cu = sv.normal(40, 16, 128, seed=70).cuda(), torch.randperm(200, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(2, 100).cuda(), _i32([0, 15, 40])
    kc, vc = (sv.normal(200, 16, 2, 128, seed=71 + i).cuda() for i in (0, 1))
    n = _i32([1500, 1333])
    logits, scores = torch.randn(64, 30011, device="cuda").bfloat16(), torch.zeros(8, 8, device="cuda")
    want = (*lss.lss_paged_attn_tree(q, kc, vc, table, n, cu), *lss.lss_beam_select(logits, scores)[:3])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for st in streams:
            ws = [torch.empty(max(16, b), dtype=torch.uint8, device="cuda") for b in (lss.lss_paged_attn_tree_workspace_bytes(40, 2, 16, 2, 128, 1600), lss.lss_beam_select_workspace_bytes(8, 8, 30011, 8))]
            outs = [torch.empty_like(x) for x in want]
            torch.cuda.synchronize()
            got.append((st, ws, outs))
        for st, ws, outs in got:
            lss.lss_paged_attn_tree(q, kc, vc, table, n, cu, out=outs[0], lse=outs[1], stream=st, workspace=ws[0])
            lss.lss_beam_select(logits, scores, scores_out=outs[2], parents=outs[3], tokens=outs[4], stream=st, workspace=ws[1])
        torch.cuda.synchronize()
        for _, _, outs in got:
            for a, b in zip(outs, want):
                assert torch.equal(a, b)
