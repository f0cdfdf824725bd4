"""GPU: beam search's selection against the plain 64-bit form.

A row's sum of exponentials: each term within 3 u |x - max| + 2 u (subtraction, product, the constant, the
exponential; u = 2^-24, |x - max| under 20 where terms count), at most vocab / 256 + 8 terms of a lane in a row with a
rescaling every 8: so ln of the sum is within (62 + 1.5 (vocab / 256 + 8)) u.  The score is then rounded to float32.
"""
import numpy as np
import pytest
import torch

import _kv_forms as forms
import paper_2608_07971_amd as esp
from paper_2608_07971_amd import kv

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)


def _randn(seed, *shape, dtype=torch.float32, gain=2.5):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype).cuda()


def _check(logits, scores, width, ended=None, pad=0):
    out, parents, tokens = (t.cpu().numpy() for t in kv.select_beams(logits, scores, width, ended=ended, pad=pad))
    G, B, V = logits.shape
    x = logits.double().cpu().numpy()
    e = None if ended is None else ended.cpu().numpy()
    totals = forms.beam_totals(x, scores.cpu().numpy(), e, pad)
    off = (62 + 1.5 * (V / 256 + 8)) * U
    assert out.shape == parents.shape == tokens.shape == (G, width) and parents.dtype == tokens.dtype == np.int32
    for g in range(G):
        all_of = np.sort(totals[g].reshape(-1))[::-1]
        n = min(width, int((all_of > -np.inf).sum()))
        assert (parents[g, n:] == -1).all() and (tokens[g, n:] == -1).all() and (out[g, n:] == -np.inf).all()
        beam, token = parents[g, :n] - g * B, tokens[g, :n]
        assert ((beam >= 0) & (beam < B) & (token >= 0) & (token < V)).all()
        got = totals[g, beam, token]
        assert len({*zip(beam.tolist(), token.tolist())}) == n
        assert (np.abs(out[g, :n] - got) <= U * np.abs(got) + off * 1.01).all()
        assert (np.abs(got - all_of[:n]) <= 2 * off).all()       # each as good as the one of its rank
        for b in set(beam.tolist()):                              # one beam's in the order of its logits, then of its tokens
            if e is None or not e[g, b]:
                mine = token[beam == b]
                assert (mine == np.lexsort((np.arange(V), -x[g, b]))[:len(mine)]).all()
    return out, parents, tokens


CASES = [
    (1, 1, 1, 1, torch.float32), (1, 1, 2, 3, torch.bfloat16), (2, 3, 7, 40, torch.float16), (3, 4, 63, 4, torch.float32), (1, 4, 500, 4, torch.bfloat16),
    (2, 16, 2047, 32, torch.float16), (1, 5, 2049, 64, torch.float32), (9, 5, 50261, 10, torch.float32), (1, 1, 262143, 1, torch.bfloat16),
    (2, 8, 131072, 8, torch.bfloat16), (70, 2, 3001, 2, torch.float16), (1, 100, 1234, 7, torch.bfloat16), (1200, 1, 65, 5, torch.float32),
]


@pytest.mark.parametrize("groups,beams,vocab,width,dtype", CASES)
def test_select_beams(groups, beams, vocab, width, dtype):
    _say(f"select {groups}x{beams}x{vocab} width={width} {dtype}")
    logits = _randn(1, groups, beams, vocab, dtype=dtype)
    scores = -5.0 - _randn(2, groups, beams, gain=1.0).abs() * 3
    first = _check(logits, scores, width)
    again = _check(logits, scores, width)
    assert all((a == b).all() for a, b in zip(first, again))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_banned_tokens_ended_beams_and_the_first_step(dtype):
    G, B, V, W = 6, 5, 5003, 10
    logits, scores = _randn(3, G, B, V, dtype=dtype), -_randn(4, G, B, gain=4.0).abs()
    gen = torch.Generator().manual_seed(5)
    logits[(torch.rand(G, 1, V, generator=gen) < 0.7).expand(G, B, V).cuda()] = -float("inf")
    logits[1, 2] = -float("inf")                                  # a beam that may not go on
    logits[2, :, 4:] = -float("inf")                              # fewer tokens than beams asked for
    logits[3] = -float("inf")                                     # nothing at all
    ended = (torch.rand(G, B, generator=gen) < 0.3).cuda()
    ended[3, :] = False
    ended[3, 1] = True                                            # all that is left
    ended[4, :] = True
    _check(logits, scores, W, ended, pad=V - 1)
    _check(logits, scores, W, ended, pad=2)
    scores[:, 1:] = -float("inf")                                 # one beam of each counts
    scores[5, 0] = float("nan")
    scores[5, 1] = float("inf")
    _check(logits, scores, W, ended, pad=0)
    _check(logits, scores, W)


def test_beams_with_nan_or_infinity_have_no_candidates():
    logits, scores = _randn(6, 2, 4, 999), -_randn(7, 2, 4, gain=1.0).abs()
    logits[0, 1, 998], logits[0, 2, 0], logits[1, 0, 500] = float("nan"), float("inf"), -float("nan")
    _, parents, _ = _check(logits, scores, 6)
    assert set(parents[0].tolist()) <= {0, 3} and set(parents[1].tolist()) <= {5, 6, 7}


@pytest.mark.parametrize("vocab", [3, 700, 4097, 40001])
def test_ties_go_to_the_lower_beam_then_the_lower_token(vocab):
    B, W = 4, 9
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        same = torch.full((2, B, vocab), 1.5, dtype=dtype, device="cuda")
        same[1] = -0.0
        same[1, :, ::2] = 0.0                                     # equal numbers
        scores = torch.full((2, B), -3.0, device="cuda")
        out, parents, tokens = kv.select_beams(same, scores, W)
        n = min(vocab, W)
        assert tokens[:, :n].tolist() == [list(range(n))] * 2 and parents[:, :n].tolist() == [[0] * n, [B] * n]
        # beams that are copies of each other, whatever place their rows have in memory
        rows = torch.randn(vocab, generator=torch.Generator().manual_seed(vocab)).to(dtype).cuda().expand(2, B, vocab).contiguous()
        out, parents, tokens = kv.select_beams(rows, scores, W)
        order = np.lexsort((np.arange(vocab), -rows[0, 0].double().cpu().numpy()))
        x = rows[0, 0].double().cpu().numpy()[order]
        want = []
        for v in dict.fromkeys(x.tolist()):                       # equal logits: by beam, then by token
            want += [(b, t) for b in range(B) for t in order[x == v]]
        want = want[:W]
        for g in range(2):
            assert tokens[g, :len(want)].tolist() == [t for _, t in want] and parents[g, :len(want)].tolist() == [g * B + b for b, _ in want]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [2, 300, 20000])
def test_logits_whose_sums_round_to_the_same(vocab, dtype):
    """One beam's tokens go by their logits, also where these differ by less than their sums in binary64 can show."""
    _say(f"select, sums that are equal and logits that are not, {vocab} {dtype}")
    B, gen = 3, torch.Generator().manual_seed(vocab)
    small = (torch.rand(2, B, vocab, generator=gen) * 1e-20).to(dtype).cuda()     # beside a sum of logarithms above 0.6
    small[:, :, 0] = 0.0
    scores = torch.tensor([[-1.0, -1.0, -3.0], [-2.0, -2.5, -2.0]], device="cuda")
    x = small.double().cpu().numpy()
    totals = forms.beam_totals(x, scores.cpu().numpy(), None, 0)
    assert (totals == totals[..., :1]).all()
    for width in (1, 2, 7, 64):
        _, parents, tokens = _check(small, scores, width)
        n = min(width, B * vocab)
        for g in range(2):
            # beams of equal rows of sums: the better score, then the lower beam; sums of rows differ by 1e-20 at most
            best = np.lexsort((np.arange(B), -totals[g, :, 0]))
            want = [(g * B + b, t) for b in best for t in np.lexsort((np.arange(vocab), -x[g, b]))[:width]][:n]
            assert [*zip(parents[g, :n].tolist(), tokens[g, :n].tolist())] == want
        first = kv.select_beams(small, scores, 1)
        assert torch.equal(first[2].cpu(), torch.tensor(tokens[:, :1]))


def test_logits_in_any_order_and_at_any_place():
    V, W = 30011, 16
    up = torch.linspace(-9, 9, V).expand(1, 3, V)
    for x in (up, up.flip(-1)):                                   # every batch has better ones than all before, or none
        _check(x.contiguous().cuda(), torch.tensor([[-1.0, -1.5, -2.0]], device="cuda"), W)
    scores = -_randn(8, 3, 4, gain=1.0).abs()
    for dtype in (torch.bfloat16, torch.float32):
        wide = _randn(9, 3, 5, V + 5, dtype=dtype)                # a vocabulary that is padded
        _check(wide[:, 1:, 3:V], scores, W)
        _check(wide.transpose(0, 1).contiguous().transpose(0, 1)[:, :4, 1:V], scores, W)
        _check(wide[:, :1, :V].expand(3, 4, V), scores, W)        # all beams read one row


def test_select_in_a_graph_and_on_another_stream():
    G, B, V, W, side = 3, 4, 20001, 8, torch.cuda.Stream()
    logits, scores = torch.zeros(G, B, V, dtype=torch.bfloat16, device="cuda"), torch.zeros(G, B, device="cuda")
    kv.select_beams(logits, scores, W)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = kv.select_beams(logits, scores, W)
    for i in range(5):
        _say(f"replay {i}")
        logits.copy_(_randn(i, G, B, V))
        scores.copy_(-_randn(50 + i, G, B).abs())
        graph.replay()
        torch.cuda.synchronize()
        want = kv.select_beams(logits, scores, W)
        torch.cuda.synchronize()
        other = kv.select_beams(logits, scores, W, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(got, want, other))


def test_what_does_not_fit_is_refused():
    logits, scores = _randn(1, 2, 3, 50), torch.zeros(2, 3, device="cuda")
    ended = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    call = lambda x=logits, s=scores, w=4, **more: kv.select_beams(x, s, w, **more)  # noqa: E731
    for bad in (dict(x=logits.double()), dict(x=logits[0]), dict(x=logits.transpose(1, 2)), dict(s=scores.double()), dict(s=scores[:, :2]), dict(s=scores.cpu()),
                dict(ended=ended.int()), dict(ended=ended[:1]), dict(x=logits.cpu(), s=scores.cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(w=0), dict(w=65), dict(ended=ended, pad=50), dict(ended=ended, pad=-1), dict(x=torch.zeros(1, 1025, 4, device="cuda"), s=torch.zeros(1, 1025, device="cuda"))):
        with pytest.raises(esp.EspError):
            call(**bad)
    out = call(x=torch.zeros(0, 3, 50, device="cuda"), s=scores[:0])
    assert [t.shape for t in out] == [(0, 4)] * 3
    lost = call(x=logits.clone().requires_grad_())[0]
    with pytest.raises(RuntimeError, match="no gradient"):
        lost.sum().backward()
