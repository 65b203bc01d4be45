"""The serving operators as they are used together, captured into graphs, and on streams of their own."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _serving as sv

pytestmark = pytest.mark.gpu


class Server:
    """One attention layer of a model that answers several prompts: what a program keeps between its calls"""

    def __init__(self, prompts, steps, H, H_kv, d, page, dtype, rot, seed):
        self.B, self.H, self.H_kv, self.d, self.steps, self.prompts = len(prompts), H, H_kv, d, steps, prompts
        total = [n + steps for n in prompts]
        self.table, n_pages = sv.tables(total, page, seed)
        gpu = dict(dtype=dtype, device="cuda")
        self.k_cache, self.v_cache = (torch.full((n_pages, page, H_kv, d), float("nan"), **gpu) for _ in range(2))
        # what the projections would give, for every token of every sequence
        self.q, self.k, self.v = ([sv.normal(n, h, d, seed=seed + 10 * b + i, dtype=dtype) for b, n in enumerate(total)] for i, h in ((1, H), (2, H_kv), (3, H_kv)))
        self.freq = sv.frequencies(rot) if rot else None
        self.lengths = torch.tensor(prompts, dtype=torch.int32, device="cuda")
        self.cu, self.gpu_table = sv.starts(prompts).cuda(), self.table.cuda()
        self.gpu_freq = None if self.freq is None else self.freq.cuda()

    def prompt(self):
        q, k, v = (torch.cat([x[:n] for x, n in zip(xs, self.prompts)]).cuda() for xs in (self.q, self.k, self.v))
        k_rot = torch.empty_like(k)
        q_rot, _ = lss.lss_paged_append(k, v, self.k_cache, self.v_cache, self.gpu_table, self.lengths, self.cu, q=q, inv_freq=self.gpu_freq, k_rot=k_rot)
        return lss.lss_packed_attn_fwd(q_rot, k_rot, v, self.cu)

    def tokens(self, i):
        return [torch.stack([x[n + i] for x, n in zip(xs, self.prompts)]).cuda() for xs in (self.q, self.k, self.v)]

    def step(self, q, k, v):
        self.lengths += 1
        q_rot, _ = lss.lss_paged_append(k, v, self.k_cache, self.v_cache, self.gpu_table, self.lengths, q=q, inv_freq=self.gpu_freq)
        return lss.lss_paged_attn_decode(q_rot, self.k_cache, self.v_cache, self.gpu_table, self.lengths)

    def want(self, b):
        """Attention of sequence b over all its tokens in 64 bits; the rotated rows rounded to the type, as they are kept"""
        p = torch.arange(len(self.q[b]))
        q, k = (sv.rotate(x[b], p, self.freq, False)[0].to(x[b].dtype) for x in (self.q, self.k))
        per_head = [sv.attention(q[:, h], k[:, h // (self.H // self.H_kv)], self.v[b][:, h // (self.H // self.H_kv)], p + 1, q.dtype) for h in range(self.H)]
        return [torch.stack(x, 1) for x in zip(*per_head)]


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("H,H_kv,d,page,rot", [(8, 2, 64, 16, 64), (4, 4, 128, 32, 64), (6, 1, 64, 64, 0)])
def test_prompts_then_tokens(dtype, H, H_kv, d, page, rot):
    steps = 20
    s = Server([33, 1, 140, 64], steps, H, H_kv, d, page, dtype, rot, seed=1)
    out, lse = s.prompt()
    got = [[out[int(s.cu[b]):int(s.cu[b + 1])]] for b in range(s.B)]
    got_lse = [[lse[:, int(s.cu[b]):int(s.cu[b + 1])].T] for b in range(s.B)]
    for i in range(steps):
        out, lse = s.step(*s.tokens(i))
        for b in range(s.B):
            got[b].append(out[b:b + 1])
            got_lse[b].append(lse[b:b + 1])
    for b in range(s.B):
        want, want_lse, ob, lb = s.want(b)
        # a rotated element next to a border may be kept as the type's value on its other side (a step): up to 2 half steps of it in q and k
        # each, in a score at most 4 half steps of the sum of its products' sizes -- seen for an element in 10^4 or so (float: 2^-24 against 2^-22)
        q, k = s.q[b].double(), s.k[b].double()
        if rot:
            few = 4 * sv.HALF[dtype] * (q.abs().amax() * k.abs().amax()) * (8 if dtype == torch.float32 else 1) / d ** 0.5
            slack = few * 4
        else:
            slack = 0.0
        sv.check(torch.cat(got[b]), want, ob + 2 * slack * s.v[b].double().abs().amax(), f"out of sequence {b}")
        sv.check(torch.cat(got_lse[b]), want_lse, lb + slack, f"lse of sequence {b}")


def test_captured_steps_follow_the_lengths():
    # one token per replay: the graph holds the increment of the lengths, the append and the attention; each replay against eager calls on a
    # copy of everything, with eager work of the process between the replays.  Two graphs of different shapes share what scratch the binding keeps
    steps = 7
    graphs = []
    for seed, (prompts, H, H_kv, d) in enumerate((([300, 20, 1500], 8, 2, 64), ([1, 90], 4, 4, 128))):
        s, e = (Server(prompts, steps + 1, H, H_kv, d, 16, torch.bfloat16, 64, seed=10 + seed) for _ in range(2))
        s.prompt(), e.prompt()
        inputs = s.tokens(0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.step(*inputs)
        torch.cuda.current_stream().wait_stream(side)
        e.step(*e.tokens(0))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out, lse = s.step(*inputs)
        graphs.append((s, e, inputs, graph, out, lse))
    for i in range(1, steps):
        for s, e, inputs, graph, out, lse in graphs:
            for x, y in zip(inputs, s.tokens(i)):
                x.copy_(y)
            out.fill_(3.0), lse.fill_(3.0)
            graph.replay()
            want = e.step(*e.tokens(i))
            torch.cuda.synchronize()
            for a, b in zip((out, lse, s.lengths), (*want, e.lengths)):
                assert torch.equal(a, b) and torch.isfinite(a.float()).all()


def test_captured_prompts_follow_the_starts():
    gen = lambda seed, *shape: sv.normal(*shape, seed=seed).cuda()
    rows, H, H_kv, d = 500, 4, 2, 64
    q, k, v, cu = gen(1, rows, H, d), gen(2, rows, H_kv, d), gen(3, rows, H_kv, d), sv.starts([100, 300, 100]).cuda()
    lss.lss_packed_attn_fwd(q, k, v, cu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = lss.lss_packed_attn_fwd(q, k, v, cu)
    for i, n in enumerate(([100, 300, 100], [500, 0, 0], [1, 1, 498], [130, 240, 130])):
        cu.copy_(sv.starts(n))
        q.copy_(gen(10 + i, rows, H, d))
        out.fill_(3.0), lse.fill_(3.0)
        graph.replay()
        want = lss.lss_packed_attn_fwd(q, k, v, cu)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_a_stream_of_its_own():
    s = Server([200, 31], 1, 4, 2, 64, 16, torch.bfloat16, 64, seed=30)
    e = Server([200, 31], 1, 4, 2, 64, 16, torch.bfloat16, 64, seed=30)
    want = [*e.prompt(), *e.step(*e.tokens(0))]
    tokens = s.tokens(0)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = [*s.prompt(), *s.step(*tokens)]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # ... and one that is passed instead of the current one
    q = e.q[0][:2].cuda()
    out, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    torch.cuda.synchronize()
    got = lss.lss_paged_attn_decode(q, e.k_cache, e.v_cache, e.gpu_table, e.lengths, out=out, lse=lse, stream=side)
    side.synchronize()
    for a, b in zip(got, lss.lss_paged_attn_decode(q, e.k_cache, e.v_cache, e.gpu_table, e.lengths)):
        assert torch.equal(a, b)


def test_refusals_of_the_binding():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    kc, table, lengths = z(2, 16, 2, 64), i32(1, 2), i32(1)
    with pytest.raises(ValueError, match="q must be \\[B, H, d\\]"):
        lss.lss_paged_attn_decode(z(2, 4, 64), kc, kc, table, lengths)
    with pytest.raises(ValueError, match="q must be \\[B, H, d\\]"):
        lss.lss_paged_attn_decode(z(1, 4, 64, dt=torch.float32), kc, kc, table, lengths)
    with pytest.raises(ValueError, match="block_table must be a contiguous torch.int32"):
        lss.lss_paged_attn_decode(z(1, 4, 64), kc, kc, table.long(), lengths)
    with pytest.raises(ValueError, match="disagree"):
        lss.lss_paged_attn_decode(z(1, 4, 64), kc, kc, table, i32(2))
    with pytest.raises(ValueError, match="current GPU"):
        lss.lss_paged_attn_decode(torch.zeros(1, 4, 64, dtype=torch.bfloat16), kc, kc, table, lengths)
    with pytest.raises(ValueError, match="output has shape"):
        lss.lss_paged_attn_decode(z(1, 4, 64), kc, kc, table, lengths, out=z(1, 4, 128))
    with pytest.raises(lss.LssError, match="LSS_ERR_SHAPE"):
        lss.lss_paged_attn_decode(z(1, 3, 64), kc, kc, table, lengths)
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_paged_attn_decode(z(1, 4, 64), kc, kc, table, lengths, max_len=33)
    with pytest.raises(lss.LssError, match="LSS_ERR_UNSUPPORTED_D"):
        lss.lss_paged_attn_decode(z(1, 4, 32), z(2, 16, 2, 32), z(2, 16, 2, 32), table, lengths)
    with pytest.raises(ValueError, match="one row for every sequence"):
        lss.lss_paged_append(z(2, 2, 64), z(2, 2, 64), kc, kc.clone(), table, lengths)
    with pytest.raises(ValueError, match="q_rot without q"):
        lss.lss_paged_append(z(1, 2, 64), z(1, 2, 64), kc, kc.clone(), table, lengths, q_rot=z(1, 4, 64))
    with pytest.raises(ValueError, match="inv_freq must be"):
        lss.lss_paged_append(z(1, 2, 64), z(1, 2, 64), kc, kc.clone(), table, lengths, inv_freq=z(32, dt=torch.float32))
    with pytest.raises(lss.LssError, match="rot_dim = 24"):
        lss.lss_paged_append(z(1, 2, 64), z(1, 2, 64), kc, kc.clone(), table, lengths, inv_freq=z(12, dt=torch.float64))
    with pytest.raises(ValueError, match="heads of a row of k"):
        lss.lss_paged_append(z(1, 64, 2).transpose(1, 2), z(1, 2, 64), kc, kc.clone(), table, lengths)
    with pytest.raises(ValueError, match="one entry more"):
        lss.lss_packed_attn_fwd(z(3, 4, 64), z(3, 2, 64), z(3, 2, 64), i32(2), i32(3))
    with pytest.raises(lss.LssError, match="LSS_ERR_ALIGN"):
        lss.lss_packed_attn_fwd(z(3, 4 * 64 + 4)[:, :256].unflatten(1, (4, 64)), z(3, 2, 64), z(3, 2, 64), i32(2))
