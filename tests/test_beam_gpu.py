"""Beam selection against a candidate-by-candidate 64-bit form, whole numbers equal; reordering against indexing."""
import math

import pytest
import torch

import layer_reference as ref
import paper_2401_04658_amd as la2

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
INF = math.inf


def check(logits, scores, finished=None, eos=-1):
    got = la2.la2_beam_select(logits.cuda(), scores.cuda(), None if finished is None else finished.cuda(), eos=eos)
    want, closest = ref.select(logits, scores, finished, eos)
    assert closest == 0 or closest > 2e-5   # of the inputs: an order that the bound on the scores does not leave open
    out, parent, token, done = (t.cpu() for t in got)
    for b, row in enumerate(want):
        for j, (s, i, t, f) in enumerate(row):
            at = (b, j)
            assert (int(parent[at]), int(token[at]), bool(done[at])) == (i, t, f), (at, row[j], int(parent[at]), int(token[at]), bool(done[at]))
            # the sum of exp is off by 2^-20 at most (2^-22 an exponential, arguments rounded to fp32), the score is rounded once
            assert float(out[at]) == s or abs(float(out[at]) - s) <= 2 ** -20 + 2 ** -23 * abs(s), (at, float(out[at]), s)


def make(batch, beams, vocab, dtype, seed, scale=3.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    full = torch.full((batch, beams, vocab + pad), INF)
    full[..., :vocab] = torch.randn(batch, beams, vocab, generator=g) * scale
    scores = (-6 * torch.rand(batch, beams, generator=g)).sort(1, descending=True).values
    return full.to(dtype)[..., :vocab], scores, torch.rand(batch, beams, generator=g) < 0.25


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 64, 255, 1000, 4095, 4096, 4097, 8191, 8193, 32000, 50021])
def test_vocabularies(vocab, dtype):
    for beams in (1, 4):
        logits, scores, finished = make(3, beams, vocab, dtype, seed=1000 + vocab + beams)
        check(logits, scores)
        check(logits, scores, finished, eos=vocab // 2)


@pytest.mark.parametrize("beams", [1, 2, 3, 5, 8, 13, 16, 31, 32])
def test_beams(beams):
    logits, scores, finished = make(2, beams, 9001, torch.float32, seed=2000 + beams)
    check(logits, scores, finished, eos=2)
    check(*make(1, beams, 70000, torch.float32, seed=2100 + beams)[:2])


def test_many_rows_take_large_pieces():
    logits, scores, finished = make(70, 16, 8500, torch.float32, seed=31)
    check(logits, scores, finished, eos=0)


def test_largest_vocabulary():
    logits, scores, _ = make(1, 3, 1 << 20, torch.float32, seed=41)
    check(logits, scores)
    logits, scores, _ = make(1, 32, 300001, torch.float32, seed=42)
    check(logits, scores)


@pytest.mark.parametrize("dtype", DTYPES)
def test_equal_logits_go_to_the_lowest_token(dtype):
    for vocab in (5, 1000, 20001):
        logits = torch.zeros(2, 4, vocab, dtype=dtype)
        logits[0, 1, vocab // 2:] = 1.0
        logits[0, 2, ::3] = 2.0
        scores = torch.tensor([[0.0, -1.0, -30.0, -50.0], [-9.0, -2.0, -1.0, -0.5]])
        check(logits, scores)
        logits[1] = -0.0
        logits[1, :, 1::2] = 0.0   # the two zeros are equal
        check(logits, scores)


def test_equal_beams_go_to_the_lowest_beam():
    """The same logits in every beam, rows at every alignment: their sums have the same bits."""
    for vocab in (999, 4097, 12345):
        g = torch.Generator().manual_seed(vocab)
        logits = (torch.randn(1, 1, vocab, generator=g) * 3).to(torch.bfloat16).expand(2, 6, vocab).contiguous()
        check(logits, torch.full((2, 6), -1.5))


@pytest.mark.parametrize("dtype", DTYPES)
def test_all_the_best_in_one_place(dtype):
    """The best tokens next to one another (one thread's share) and spread over one piece; the rest far below."""
    for vocab, at in ((8192, 4000), (40000, 39960), (40000, 0)):
        logits = torch.full((1, 32, vocab), -20.0, dtype=dtype)
        logits[0, 3, at:at + 40] = torch.linspace(1, 5, 40).to(dtype)
        check(logits, torch.arange(32).float().mul(-100).view(1, 32).contiguous())


def test_masked_tokens_and_beams_without_any():
    logits, scores, _ = make(4, 4, 5000, torch.float32, seed=51)
    logits[0, :, 10:] = -INF                 # ten tokens a beam
    logits[1, 1] = -INF                      # a beam without tokens
    logits[2, :] = -INF                      # a row without candidates
    logits[3, :, 1:] = -INF                  # one candidate a beam
    check(logits, scores)
    logits[3, 1:] = -INF                     # one candidate in all
    check(logits, scores, torch.zeros(4, 4, dtype=torch.bool), eos=7)
    logits[0, 0, 3], logits[0, 2, 4096] = float("nan"), float("nan")
    logits[3, 0, 1:] = float("nan")
    check(logits, scores)


def test_first_step_dead_and_finished_beams():
    logits, scores, _ = make(5, 4, 3001, torch.bfloat16, seed=61)
    scores[0] = torch.tensor([0.0, -INF, -INF, -INF])
    scores[1] = torch.tensor([-INF, float("nan"), -2.0, -INF])
    scores[2] = -INF
    check(logits, scores)
    finished = torch.tensor([[0, 0, 0, 0], [1, 1, 1, 1], [1, 0, 0, 0], [1, 1, 1, 1], [0, 1, 0, 1]], dtype=torch.bool)
    scores[3], scores[4] = torch.tensor([-4.0, -1.0, -1.0, -3.0]), torch.tensor([-50.0, -0.1, -60.0, -55.0])
    check(logits, scores, finished, eos=0)
    check(logits, scores, finished, eos=3000)


def test_infinite_logits_count_as_the_largest_number():
    logits, scores, _ = make(2, 2, 4000, torch.float32, seed=71)
    logits[0, 0, 77], logits[1, 1, 5], logits[1, 1, 3900] = INF, INF, INF
    check(logits, scores)
    logits, scores, _ = make(1, 2, 100, torch.float32, seed=72, scale=1e30)
    check(logits, scores)


def test_rows_at_a_distance_in_place_and_on_another_stream():
    logits, scores, finished = make(3, 5, 1001, torch.float16, seed=82, pad=6)   # +inf between the rows
    check(logits, scores, finished, eos=1)
    x, s, f = logits.cuda(), scores.cuda(), finished.cuda()
    want = la2.la2_beam_select(x, s, f, eos=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = la2.la2_beam_select(x, s, f, eos=1)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- reordering
def moved(states, parent):
    batch, beams = parent.shape
    p = parent.clone()
    own = torch.arange(beams).expand(batch, beams)
    p = torch.where((p < 0) | (p >= beams), own.to(p.dtype), p).long()
    rows = (p + beams * torch.arange(batch)[:, None]).reshape(-1)
    return [s[rows] for s in states]


@pytest.mark.parametrize("beams", [1, 2, 3, 4, 5, 8, 9, 16, 17, 32])
def test_reorder(beams):
    g = torch.Generator().manual_seed(beams)
    for batch, shape in ((1, (4,)), (3, (2, 64, 64)), (2, (1037, 4))):
        states = [torch.randn(batch * beams, *shape, generator=g) for _ in range(3)]
        for parent in (torch.randint(0, beams, (batch, beams), generator=g, dtype=torch.int32), torch.zeros(batch, beams, dtype=torch.int32),
                       torch.arange(beams - 1, -1, -1, dtype=torch.int32).expand(batch, beams).contiguous(),
                       torch.arange(beams, dtype=torch.int32).roll(1).expand(batch, beams).contiguous(),
                       torch.arange(beams, dtype=torch.int32).expand(batch, beams).contiguous(),
                       torch.randint(-3, beams + 3, (batch, beams), generator=g, dtype=torch.int32)):
            on = [s.cuda() for s in states]
            back = la2.la2_beam_reorder(on, parent.cuda())
            assert back is on
            for got, want in zip(on, moved(states, parent)):
                assert torch.equal(got.cpu(), want)


def test_reorder_one_tensor_many_tensors_and_other_types():
    parent = torch.tensor([[1, 1, 0], [2, 0, 2]], dtype=torch.int32)
    one = torch.randn(6, 2, 96, 96)
    on = one.cuda()
    assert la2.la2_beam_reorder(on, parent.cuda()) is on and torch.equal(on.cpu(), moved([one], parent)[0])
    many = [torch.randn(6, 8) for _ in range(131)]   # more than one launch takes
    on = [s.cuda() for s in many]
    la2.la2_beam_reorder(tuple(on), parent.cuda())
    assert all(torch.equal(a.cpu(), b) for a, b in zip(on, moved(many, parent)))
    half = torch.randn(6, 16).bfloat16()
    on = half.cuda()
    la2.la2_beam_reorder(on, parent.cuda())
    assert torch.equal(on.cpu(), moved([half], parent)[0])
    la2.la2_beam_reorder([], parent.cuda())
    la2.la2_beam_reorder(torch.empty(0, 4, device="cuda"), parent[:0].cuda())


def test_search_as_a_program_runs_it():
    """Three steps of selection, reordering and decoding against a search that keeps every beam's own tokens and replays them."""
    batch, beams, heads, d, vocab = 2, 3, 2, 64, 50
    g = torch.Generator().manual_seed(9)
    table = torch.randn(vocab, 3, heads, d, generator=g).bfloat16().cuda()     # a token's q, k, v
    head = (torch.randn(vocab, heads * d, generator=g) * 0.3).bfloat16().cuda()
    lam = torch.tensor([0.9, 0.8], device="cuda")

    def step(kv, token):
        q, k, v = (table[token.reshape(-1).long(), i].contiguous() for i in range(3))
        o = la2.la2_decode_step(q, k, v, lam, kv)
        return la2.la2_linear_fwd(o.view(batch * beams, heads * d), head)[0].view(batch, beams, vocab)

    kv = torch.zeros(batch * beams, heads, d, d, device="cuda")
    token = torch.zeros(batch, beams, dtype=torch.int32, device="cuda")
    scores = torch.tensor([0.0, -INF, -INF], device="cuda").repeat(batch, 1)
    finished = torch.zeros(batch, beams, dtype=torch.bool, device="cuda")
    said = [[[0] for _ in range(beams)] for _ in range(batch)]
    for _ in range(3):
        logits = step(kv, token)
        scores, parent, token, finished = la2.la2_beam_select(logits, scores, finished, eos=1)
        la2.la2_beam_reorder(kv, parent)
        p, t = parent.tolist(), token.tolist()
        said = [[said[b][p[b][i]] + [t[b][i]] for i in range(beams)] for b in range(batch)]
    again = torch.zeros_like(kv)   # every beam's tokens from the start: the same state
    for n in range(3):
        step(again, torch.tensor([[said[b][i][n] for i in range(beams)] for b in range(batch)], device="cuda"))
    assert torch.equal(again, kv)


def test_states_beyond_32_bits():
    """128 beams of 36 MiB: a state buffer of more than 4 GiB; and logits of more."""
    batch, beams, floats = 4, 32, 9 << 20
    s = torch.empty(batch * beams, floats, device="cuda").normal_()
    parent = torch.randint(0, beams, (batch, beams), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    rows = (parent.long() + beams * torch.arange(batch)[:, None]).reshape(-1).cuda()
    want = s.view(batch * beams, -1, 4096)[:, ::97].index_select(0, rows)
    la2.la2_beam_reorder(s, parent.cuda())
    assert torch.equal(s.view(batch * beams, -1, 4096)[:, ::97], want)
    del s, want
    batch, beams, vocab = 1100, 8, 262144
    logits = torch.empty(batch, beams, vocab, dtype=torch.bfloat16, device="cuda").normal_()
    scores = torch.zeros(batch, beams, device="cuda")
    got = la2.la2_beam_select(logits, scores)
    tail = la2.la2_beam_select(logits[-3:], scores[-3:])
    assert all(torch.equal(a[-3:], b) for a, b in zip(got[1:], tail[1:]))
    # the rows alone are cut otherwise than the whole batch: sums of exp in another order, 2^-20
    assert float((got[0][-3:] - tail[0]).abs().max()) <= 2 ** -19
