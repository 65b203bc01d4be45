"""Beam search's choice, against its definition: parents and tokens exactly, totals within the bound of a row's log-sum-exp."""
import math

import pytest
import torch

from paper_2311_02382_amd import lss
import _continuations as co
import _serving as sv

pytestmark = pytest.mark.gpu


def _check(logits, scores, n_out, finished=None, end_token=-1, gpu_logits=None):
    want = co.select(logits, scores, n_out, finished, end_token)
    # (two totals nearer than what they may be off by could be told apart neither way: these inputs have none)
    assert want[4] > 2 * co.LSE_BOUND + 2.0 ** -40
    got = lss.lss_beam_select(logits.cuda() if gpu_logits is None else gpu_logits, scores.cuda(), n_out, finished=None if finished is None else finished.cuda(), end_token=end_token)
    torch.cuda.synchronize()
    assert torch.equal(got[1].cpu().long(), want[1]) and torch.equal(got[2].cpu().long(), want[2])
    sv.check(got[0], want[0], co.LSE_BOUND + 2.0 ** -24 * want[0].abs().nan_to_num(posinf=0.0), "scores_out")
    if end_token < 0:
        assert got[3] is None
    else:
        assert torch.equal(got[3].cpu(), want[3])
    return got


def _inputs(B, K, V, dtype, seed, spread=3.0):
    return sv.normal(B * K, V, seed=seed, dtype=torch.float32, std=spread).to(dtype), -20 * torch.rand(B, K, generator=torch.Generator().manual_seed(seed + 1))


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 256, 1000, 2047, 2048, 2049, 4095, 4096, 4097, 5000, 32001])
@pytest.mark.parametrize("K,n_out", [(1, 1), (4, 4), (3, 7)])
def test_vocabularies(dtype, V, K, n_out):
    _check(*_inputs(2, K, V, dtype, seed=V + K), n_out)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("K,n_out", [(1, 64), (2, 1), (5, 10), (16, 32), (17, 3), (64, 64), (33, 64)])
@pytest.mark.parametrize("V", [300, 9001])
def test_beams(dtype, K, n_out, V):
    _check(*_inputs(2, K, V, dtype, seed=1000 + K + V, spread=6.0), n_out)


def test_many_prompts_and_a_large_vocabulary():
    _check(*_inputs(150, 2, 3001, torch.bfloat16, seed=3), 4)
    _check(*_inputs(1, 2, 300007, torch.float32, seed=4), 8)
    _check(*_inputs(1, 1, 2000003, torch.bfloat16, seed=5, spread=8.0), 8)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("V", [500, 20000])
def test_equal_logits_go_to_the_lower_token(dtype, V):
    # few different values; all alike; beams whose totals are exactly alike; both zeros
    gen = torch.Generator().manual_seed(6)
    logits = torch.randint(-3, 4, (4, V), generator=gen).to(dtype)
    scores = torch.tensor([[-1.0, -1.0 - 5.5], [-2.0, -30.0]])
    for n_out in (1, 5, 64):
        _check(logits, scores, n_out)
        alike = torch.zeros(2, V, dtype=dtype)
        got = _check(alike, torch.tensor([[0.0, 0.0]]), n_out)
        assert got[2].tolist()[0] == list(range(n_out)) and set(got[1].tolist()[0]) == {0}
    signs = torch.full((1, V), -4.0, dtype=dtype)
    signs[0, 3], signs[0, 5], signs[0, V - 1] = 0.0, -0.0, 0.0
    assert _check(signs, torch.zeros(1, 1), 4)[2].tolist() == [[3, 5, V - 1, 0]]


@pytest.mark.parametrize("V", [130, 9000])
@pytest.mark.parametrize("K", [8, 20, 64])
def test_more_alike_than_are_wanted(K, V):
    # all beams alike: the lowest beam's lowest tokens; totals that 32 bits cannot tell apart: the best of them all the same
    alike = torch.zeros(K, V)
    for n_out in (33, 64):
        got = _check(alike, torch.full((1, K), -3.0), n_out)
        assert got[2].tolist()[0] == list(range(n_out)) and set(got[1].tolist()[0]) == {0}
    _check(torch.randn(K, V, generator=torch.Generator().manual_seed(65)).mul(0.25), torch.full((1, K), -1.0e9), 50)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("V", [700, 12000])
def test_ascending_and_descending_logits(dtype, V):
    # candidates in the worst order: each beats all before it
    rising = (torch.arange(V, dtype=torch.float32) * (16.0 / V)).to(dtype)
    for n_out in (3, 64):
        _check(torch.stack([rising, rising.flip(0)]), torch.tensor([[0.0, -0.75]]), n_out)


@pytest.mark.parametrize("V", [90, 9000])
def test_beams_that_have_ended(V):
    for seed in range(3):
        logits, scores = _inputs(5, 4, V, torch.bfloat16, seed=20 + seed)
        finished = torch.rand(5, 4, generator=torch.Generator().manual_seed(seed)) < 0.4
        finished[4] = True                          # a prompt all of whose beams have: fewer continuations than are wanted
        logits[finished.flatten()] = math.nan        # (their logits are not looked at)
        scores[0] = torch.tensor([-1.0, -2.0, -50.0, -3.0])
        _check(logits, scores, 6, finished, end_token=V - 1)
        _check(logits, scores, 6, finished, end_token=0)
    logits, scores = _inputs(2, 3, V, torch.float32, seed=30)
    logits[:, 7] = 30.0                              # all go to the end
    assert bool(_check(logits, scores, 2, None, end_token=7)[3].all())


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("V", [200, 9000])
def test_what_is_not_finite(dtype, V):
    logits, scores = _inputs(4, 5, V, dtype, seed=40)
    logits[0, V // 2] = math.nan                     # prompt 0: rows of NaN and infinity, a dead beam, nothing but -inf; one good beam
    logits[1, 3] = math.inf
    scores[0, 2] = -math.inf
    logits[3] = -math.inf
    scores[1, 0], scores[1, 1] = math.nan, math.inf
    logits[11, 5:] = -math.inf                       # prompt 2: five tokens allowed, one, none but -inf elsewhere
    logits[12, 1:] = -math.inf
    logits[13], logits[14], logits[10] = -math.inf, -math.inf, -math.inf
    scores[3] = -math.inf                            # prompt 3: nothing at all
    logits[19] = torch.finfo(dtype).min
    got = _check(logits, scores, 9, None, end_token=1)
    assert got[1][3].tolist() == [-1] * 9 and bool((got[0][3] == -math.inf).all()) and bool(got[3][3].all())
    assert got[1][2].tolist().count(-1) == 3
    # the first step: all beams of a prompt are alike, one is alive
    first = torch.full((4, 5), -math.inf)
    first[:, 0] = 0.0
    clean, _ = _inputs(4, 5, V, dtype, seed=41)
    _check(clean, first, 5)


def test_the_types_lowest_and_highest_values():
    logits = torch.full((2, 300), -3.4028234663852886e38)
    logits[0, 7], logits[1, 9] = 3.0e38, -3.3e38
    _check(logits, torch.zeros(1, 2), 3)


@pytest.mark.parametrize("dtype", sv.DTYPES)
@pytest.mark.parametrize("V", [333, 8191])
def test_rows_that_lie_apart_and_anywhere(dtype, V):
    logits, scores = _inputs(3, 2, V, dtype, seed=50)
    for shift in (0, 1, 3, 5):
        wide = torch.full((6, V + 19), math.inf, dtype=dtype, device="cuda")
        wide[:, shift:shift + V] = logits.cuda()
        _check(logits, scores, 5, gpu_logits=wide[:, shift:shift + V])


def test_given_outputs_and_the_same_bits_every_time():
    logits, scores = (x.cuda() for x in _inputs(8, 4, 50001, torch.bfloat16, seed=60))
    finished = torch.zeros(8, 4, dtype=torch.bool, device="cuda")
    outs = [torch.empty(8, 8, device="cuda"), *(torch.empty(8, 8, dtype=torch.int32, device="cuda") for _ in range(2)), torch.empty(8, 8, dtype=torch.bool, device="cuda")]
    ws = torch.empty(lss.lss_beam_select_workspace_bytes(8, 4, 50001, 8), dtype=torch.uint8, device="cuda")
    call = lambda: lss.lss_beam_select(logits, scores, 8, finished=finished, end_token=2, scores_out=outs[0], parents=outs[1], tokens=outs[2], finished_out=outs[3], workspace=ws)
    r = call()
    assert all(a is b for a, b in zip(r, outs))
    first = [x.clone() for x in outs]
    for fill in (0, 255, 127):
        ws.fill_(fill)                               # scratch that holds anything
        call()
        assert all(torch.equal(a, b) for a, b in zip(outs, first))


def test_refusals_of_the_binding():
    x, s = torch.zeros(4, 50, device="cuda"), torch.zeros(2, 2, device="cuda")
    with pytest.raises(ValueError, match="logits must be"):
        lss.lss_beam_select(x[:3], s)
    with pytest.raises(ValueError, match="logits must be"):
        lss.lss_beam_select(x.half(), s)
    with pytest.raises(ValueError, match="logits must be"):
        lss.lss_beam_select(x.T.contiguous().T, s)
    with pytest.raises(ValueError, match="scores must be"):
        lss.lss_beam_select(x, s.double())
    with pytest.raises(ValueError, match="finished must be"):
        lss.lss_beam_select(x, s, finished=torch.zeros(4, dtype=torch.bool, device="cuda"), end_token=1)
    with pytest.raises(ValueError, match="torch.int32"):
        lss.lss_beam_select(x, s, parents=torch.zeros(2, 2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="output has shape"):
        lss.lss_beam_select(x, s, 3, tokens=torch.zeros(2, 2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="torch.bool device tensor"):
        lss.lss_beam_select(x, s, end_token=1, finished_out=torch.zeros(2, 2, dtype=torch.bool))
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_beam_select(x, s, finished=torch.zeros(2, 2, dtype=torch.bool, device="cuda"))
    with pytest.raises(lss.LssError, match="LSS_ERR_SHAPE"):
        lss.lss_beam_select(x, s, 65)
    with pytest.raises(lss.LssError, match="LSS_ERR_RANGE"):
        lss.lss_beam_select(x, s, scores_out=s)


@pytest.mark.parametrize("V", [1454, 20000])
def test_wide_beams_captured(V):
    # more shared memory than a launch has without asking; a graph follows its inputs
    inputs = [_inputs(3, 32, V, torch.bfloat16, seed=90 + i) for i in range(3)]
    logits, scores = (x.cuda() for x in inputs[0])
    eager = [tuple(x.clone() for x in lss.lss_beam_select(l.cuda(), s.cuda(), 64)[:3]) for l, s in inputs]
    ws = torch.empty(lss.lss_beam_select_workspace_bytes(3, 32, V, 64), dtype=torch.uint8, device="cuda")
    outs = torch.empty(3, 64, device="cuda"), torch.empty(3, 64, dtype=torch.int32, device="cuda"), torch.empty(3, 64, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lss.lss_beam_select(logits, scores, 64, scores_out=outs[0], parents=outs[1], tokens=outs[2], workspace=ws)
    for i in (0, 1, 2, 1):
        logits.copy_(inputs[i][0]), scores.copy_(inputs[i][1])
        for x in outs:
            x.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, eager[i]))
