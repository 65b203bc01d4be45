"""Attention of packed sequences with groups of heads, against its definition in 64 bits."""
import pytest
import torch

from paper_2311_02382_amd import lss
import _serving as sv

pytestmark = pytest.mark.gpu


def _want(q, k, v, cu_q, cu_k, causal):
    """The definition, where q, k and v are"""
    rows, H, d = q.shape
    H_kv = k.shape[1]
    out, lse, ob, lb = (torch.zeros(s, dtype=torch.float64, device=q.device) for s in ((rows, H, d), (H, rows), (rows, H, d), (H, rows)))
    for b in range(len(cu_q) - 1):
        mq, mk = slice(int(cu_q[b]), int(cu_q[b + 1])), slice(int(cu_k[b]), int(cu_k[b + 1]))
        n_q, n_k = mq.stop - mq.start, mk.stop - mk.start
        seen = ((n_k - n_q + 1 + torch.arange(n_q)).clamp(0, n_k) if causal else torch.full((n_q,), n_k)).to(q.device)
        for h in range(H):
            g = h // (H // H_kv)
            out[mq, h], lse[h, mq], ob[mq, h], lb[h, mq] = sv.attention(q[mq, h], k[mk, g], v[mk, g], seen, q.dtype)
    return out, lse, ob, lb


def _tensors(n_q, n_k, H, H_kv, d, dtype, seed):
    return [sv.normal(sum(n), h, d, seed=seed + i, dtype=dtype) for i, (n, h) in enumerate(((n_q, H), (n_k, H_kv), (n_k, H_kv)))]


def _run(n_q, H, H_kv, d, dtype=torch.bfloat16, n_k=None, causal=True, seed=1):
    q, k, v = _tensors(n_q, n_k or n_q, H, H_kv, d, dtype, seed)
    cu_q, cu_k = sv.starts(n_q), sv.starts(n_k or n_q)
    out, lse = lss.lss_packed_attn_fwd(q.cuda(), k.cuda(), v.cuda(), cu_q.cuda(), None if n_k is None else cu_k.cuda(), causal=causal)
    torch.cuda.synchronize()
    want, want_lse, ob, lb = _want(q, k, v, cu_q, cu_k, causal)
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_around_every_tile(dtype, d, causal):
    _run([0, 1, 2, 15, 16, 17, 31, 0, 0, 32, 33, 63, 64, 65, 127, 128, 129, 0], 2, 1, d, dtype, causal=causal, seed=10)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("H,H_kv", [(1, 1), (3, 3), (8, 1), (6, 2), (10, 2), (16, 16)])
def test_groups_of_heads(dtype, H, H_kv):
    _run([40, 150, 7], H, H_kv, 64, dtype, seed=20 + H)
    _run([70, 1], H, H_kv, 128, dtype, seed=40 + H)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("n_q,H,H_kv,d", [([1500], 2, 2, 64), ([1025], 2, 1, 128), ([700, 1, 300, 257], 4, 2, 128), ([513, 800], 3, 1, 64)])
def test_longer_prompts(dtype, n_q, H, H_kv, d):
    _run(n_q, H, H_kv, d, dtype, seed=60)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_behind_keys_that_are_there_and_rows_that_see_none(dtype, causal, d):
    # continued prompts; more rows than keys: the first rows see no key; no keys at all; keys without rows
    _run([1, 5, 130, 70, 90, 12, 0, 64], 4, 2, d, dtype, n_k=[300, 69, 131, 500, 40, 0, 77, 64], causal=causal, seed=80)


def _some(n, B, seed):
    return [int(x) for x in torch.randint(n // 2, n + n // 2, (B,), generator=torch.Generator().manual_seed(seed))]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("form,n_q,old,H,H_kv,d", [
    ((4, 1), _some(200, 40, 1), 0, 16, 8, 64), ((4, 2), [500, 701], 3700, 32, 8, 64), ((2, 1), _some(100, 5, 2), 0, 4, 2, 64), ((1, 4), [700], 33, 2, 2, 64),
    ((2, 4), [1301], 1234, 8, 8, 64), ((2, 2), [600, 901, 700], 0, 8, 4, 64), ((4, 1), _some(200, 40, 3), 0, 16, 8, 128), ((8, 1), [4203], 0, 32, 8, 128),
    ((4, 2), [500, 701], 3700, 32, 8, 128), ((2, 2), [300, 901], 100, 6, 2, 128), ((4, 1), _some(100, 70, 4), 0, 5, 1, 64)])
def test_every_form_of_workgroup(form, n_q, old, H, H_kv, d, causal):
    n_k = [n + old for n in n_q]
    assert sv.packed_plan(sum(n_q), sum(n_k), len(n_q), H, H_kv, d)[:2] == form
    q, k, v = (x.cuda() for x in _tensors(n_q, n_k, H, H_kv, d, torch.bfloat16, 150))
    cu_q, cu_k = sv.starts(n_q), sv.starts(n_k)
    out, lse = lss.lss_packed_attn_fwd(q, k, v, cu_q.cuda(), cu_k.cuda(), causal=causal)
    want, want_lse, ob, lb = (x.cpu() for x in _want(q, k, v, cu_q, cu_k, causal))
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")
    # a value that is not finite in the last sequence's middle: the rows in front of it
    at = sum(n_k) - n_k[-1] + old + n_q[-1] // 2
    v[at] = float("nan")
    again, lse_again = lss.lss_packed_attn_fwd(q, k, v, cu_q.cuda(), cu_k.cuda(), causal=causal)
    sees = sum(n_q) - n_q[-1] + (n_q[-1] // 2 if causal else 0)
    sv.check(again[:sees], want[:sees], ob[:sees], "out in front")
    sv.check(lse_again, want_lse, lb, "lse with it")
    assert bool(torch.isnan(again[sees:]).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,n_q,n_k,H,H_kv,d,splits", [
    (torch.bfloat16, [64], [4100], 8, 2, 64, 8), (torch.bfloat16, [1, 3, 0], [2500, 3, 5000], 6, 1, 64, 8), (torch.bfloat16, [300], [9001], 8, 4, 64, 6),
    (torch.bfloat16, [33, 70], [4100, 2100], 4, 4, 128, 8), (torch.bfloat16, [513], [3000], 8, 4, 128, 3), (torch.float32, [700], [700], 2, 2, 64, 5),
    (torch.float32, [1, 40, 9], [900, 40, 1], 5, 1, 64, 2), (torch.float32, [130, 260], [1000, 260], 4, 2, 128, 4), (torch.float32, [300], [9001], 2, 1, 128, 16)])
def test_key_splits(dtype, n_q, n_k, H, H_kv, d, splits, causal):
    assert sv.packed_plan(sum(n_q), sum(n_k), len(n_q), H, H_kv, d, dtype)[2] == splits
    q, k, v = (x.cuda() for x in _tensors(n_q, n_k, H, H_kv, d, dtype, 160))
    cu_q, cu_k = sv.starts(n_q), sv.starts(n_k)
    need = lss.lss_packed_attn_workspace_bytes(sum(n_q), sum(n_k), len(n_q), H, H_kv, d, dtype.itemsize)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    run = lambda: lss.lss_packed_attn_fwd(q, k, v, cu_q.cuda(), cu_k.cuda(), causal=causal, workspace=ws)
    out, lse = run()
    want, want_lse, ob, lb = (x.cpu() for x in _want(q, k, v, cu_q, cu_k, causal))
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")
    assert all(torch.equal(sv.bits(a), sv.bits(b)) for a, b in zip(run(), (out, lse)))
    # values that are not finite where the first sequence's last row alone sees them
    v[n_k[0] - 1, :, 3] = float("inf")
    again, _ = run()
    if causal:
        at = n_q[0] - 1
        keep = torch.arange(sum(n_q)) != at
        sv.check(again[keep.cuda()], want[keep], ob[keep], "the other rows")
        assert not bool(torch.isfinite(again[at, :, 3]).any()) and bool(torch.isfinite(again[at, :, :3]).all())
    with pytest.raises(ValueError, match="workspace of"):
        lss.lss_packed_attn_fwd(q, k, v, cu_q.cuda(), cu_k.cuda(), workspace=ws[:-16])


def test_many_sequences():
    _run([(7 * b) % 23 for b in range(400)], 4, 1, 64, seed=90)
    _run([1] * 1000, 2, 2, 64, n_k=[1 + b % 70 for b in range(1000)], seed=91)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_no_sequence_are_left_and_never_read(dtype, d):
    n_q, n_k = [70, 33], [70, 150]
    q, k, v = _tensors([5] + n_q + [40], [9] + n_k + [50], 4, 2, d, dtype, 100)
    cu_q, cu_k = sv.starts(n_q) + 5, sv.starts(n_k) + 9
    for x, cu in ((q, cu_q), (k, cu_k), (v, cu_k)):
        x[:int(cu[0])], x[int(cu[-1]):] = float("nan"), float("nan")
    out, lse = torch.full(q.shape, 7.0, dtype=dtype, device="cuda"), torch.full((4, len(q)), 7.0, device="cuda")
    r = lss.lss_packed_attn_fwd(q.cuda(), k.cuda(), v.cuda(), cu_q.cuda(), cu_k.cuda(), out=out, lse=lse)
    assert r[0] is out and r[1] is lse
    want, want_lse, ob, lb = _want(q, k, v, cu_q, cu_k, True)
    want[:5], want[5 + 103:], want_lse[:, :5], want_lse[:, 5 + 103:] = 7.0, 7.0, 7.0, 7.0
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [(40,), (129, 200), (0,)])
def test_a_key_that_is_not_seen_does_not_reach_a_row(dtype, d, value, at):
    # values (and keys) that are not finite in the middle of a sequence: the rows in front of them have the bits they have without
    n = [10, 260, 30]
    q, k, v = _tensors(n, n, 4, 2, d, dtype, 110)
    cu = sv.starts(n).cuda()
    clean = lss.lss_packed_attn_fwd(q.cuda(), k.cuda(), v.cuda(), cu)
    for i, j in enumerate(at):
        v[10 + j, :, 5:9] = value
        if i:
            k[10 + j] = value
    got = lss.lss_packed_attn_fwd(q.cuda(), k.cuda(), v.cuda(), cu)
    first = 10 + at[0]
    want, want_lse, ob, lb = _want(q[:first], k[:first], v[:first], torch.tensor([0, 10, first]), torch.tensor([0, 10, first]), True)
    sv.check(got[0][:first], want, ob, "out")
    sv.check(got[1][:, :first], want_lse, lb, "lse")
    for a, b in zip((got[0][270:], got[1][:, 270:], got[0][:10]), (clean[0][270:], clean[1][:, 270:], clean[0][:10])):
        assert torch.equal(sv.bits(a), sv.bits(b))
    assert not bool(torch.isfinite(got[0][first, :, 5:9]).any())            # the first row that sees it


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_slices_of_a_wider_product(dtype):
    n, H, H_kv, d = [100, 61], 4, 2, 64
    q, k, v = _tensors(n, n, H, H_kv, d, dtype, 120)
    wide = torch.cat([x.flatten(1) for x in (q, k, v)], 1).cuda()
    parts = [x.unflatten(1, (-1, d)) for x in wide.split([H * d, H_kv * d, H_kv * d], 1)]
    cu = sv.starts(n)
    got = lss.lss_packed_attn_fwd(*parts, cu.cuda())
    for a, b in zip(got, lss.lss_packed_attn_fwd(q.cuda(), k.cuda(), v.cuda(), cu.cuda())):
        assert torch.equal(sv.bits(a), sv.bits(b))


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_scores_from_far_apart(dtype):
    n = [300, 40]
    q, k, v = _tensors(n, n, 2, 1, 64, dtype, 130)
    k *= torch.linspace(0.1, 3.0, len(k))[:, None, None].to(dtype)
    k[7] = (4.0 * q[200, 0]).to(dtype)
    cu = sv.starts(n)
    out, lse = lss.lss_packed_attn_fwd(q.cuda(), k.cuda(), v.cuda(), cu.cuda())
    want, want_lse, ob, lb = _want(q, k, v, cu, cu, True)
    sv.check(out, want, ob, "out")
    sv.check(lse, want_lse, lb, "lse")


@pytest.mark.parametrize("dtype", sv.DTYPES)
def test_one_sequence_is_the_segment_call(dtype):
    # one sequence whose rows are a segment of it: what lss_segment_attn_fwd computes
    q, k, v = _tensors([200], [500], 4, 4, 64, dtype, 140)
    cu_q, cu_k = sv.starts([200]), sv.starts([500])
    _, _, ob, lb = _want(q, k, v, cu_q, cu_k, True)
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    got = lss.lss_packed_attn_fwd(q, k, v, cu_q.cuda(), cu_k.cuda())
    want = lss.lss_segment_attn_fwd(q[None], k[None], v[None], 300)
    # (either is as far from the definition as the bounds say at most)
    sv.check(got[0], want[0][0].double().cpu(), 2 * ob, "out")
    sv.check(got[1], want[1][0].double().cpu(), 2 * lb, "lse")


def test_nothing_to_do():
    empty = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    out, lse = lss.lss_packed_attn_fwd(empty(0, 4, 64), empty(0, 2, 64), empty(0, 2, 64), sv.starts([0, 0]).cuda())
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0)
    out, lse = lss.lss_packed_attn_fwd(torch.ones(3, 4, 64, dtype=torch.bfloat16, device="cuda"), empty(0, 2, 64), empty(0, 2, 64), sv.starts([1, 2]).cuda(),
                                       sv.starts([0, 0]).cuda())
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
