"""How exact the chunk and window operators are, at bounds near what their arithmetic gives, and where windows end.

A score is D / 16 steps of the tensor core (one more where it subtracts the log-sum-exp), each of which adds 17 terms after
cutting them off one bit below the last place of the largest: q = 2^-18 for partial sums below 128, which is where the
inputs here lie.  An error of up to q in each term is q sqrt(17 / 3) in the root mean square, and up to q / 2 a step on one side;
with D = 128, 9 steps, that is (sqrt(9 * 17 / 3) + 4.5) q = 4.4e-5, times the scale 3.9e-6; D = 64 gives 3.7e-6.  The
log-sum-exp's own rounding (2^-21 below 16), the exponential and the sums add less than 1e-6.  So 5e-6 in the root mean square
covers it, while a missing piece of the log-sum-exp (4e-5) or a pair more or less in a window of 4000 (2.5e-4) does not fit in.
"""
import pytest
import torch

import chunk_ref as ref
from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu
RMS = 5e-6


def rms(x):
    return float(x.double().square().mean().sqrt())


@pytest.mark.parametrize("D,g", [(64, 2), (128, 4)])
@pytest.mark.parametrize("n,T", [(572, 128), (1500, 300), (300, 9)])
@pytest.mark.parametrize("window", [0, 400])
def test_features_to_the_accuracy_of_the_scores(D, g, n, T, window):
    c = Case(2, g, D, [n], seed=3)
    k, v, q = c.chunk([T])
    c.cache.append_chunk(0, k, v, [T])
    c.extend(k, v, [T])
    pos = c.seqs[0].pos[0]
    ok = ref.seen(pos, torch.arange(n, n + T, device="cuda"), pos[n:], window, 4)
    lse = torch.empty((T, 2 * g), dtype=torch.float64, device="cuda")
    want = []
    for hq in range(2 * g):
        z = q[:, hq].double() @ c.seqs[0].k[hq // g].double().T * D ** -0.5
        lse[:, hq] = torch.logsumexp(torch.where(ok, z, -torch.inf), 1)
        p = torch.where(ok, torch.exp(z - lse[:, hq:hq + 1].float().double()), 0.0)   # (of the log-sum-exp as it is handed over)
        want.append(ref.features(torch.zeros((n + T, 6), device="cuda"), p, T))
    c.cache.set_features(0, 0, torch.zeros((2, n + T, 6 * g), device="cuda"))
    c.cache.chunk_features(0, q, lse.float(), [T], window=window, sinks=4)
    got = c.cache.export_features(0, 0).double()
    for hq in range(2 * g):
        x, w = got[hq // g][:, 6 * (hq % g):6 * (hq % g) + 6], want[hq]
        for i in range(6):
            on = w[:, i] > 1e-30
            assert rms(x[on, i] / w[on, i] - 1) <= RMS, (hq, i, rms(x[on, i] / w[on, i] - 1))


@pytest.mark.parametrize("D,g", [(64, 2), (128, 4)])
@pytest.mark.parametrize("n,T,window,gap", [(700, 128, 0, 1), (3, 300, 0, 1), (9000, 200, 4000, 1), (9000, 60, 4000, 2)])
def test_log_sum_exp_to_the_accuracy_of_the_scores(D, g, n, T, window, gap):
    c = Case(2, g, D, [n], seed=4, gap=gap)
    k, v, q = c.chunk([T])
    lse = torch.empty((T, 2 * g), device="cuda")
    c.cache.append_chunk_attn(0, k, v, q, [T], window=window, sinks=4, lse=lse)
    c.extend(k, v, [T])
    pos = c.seqs[0].pos[0]
    ok = ref.seen(pos, torch.arange(n, n + T, device="cuda"), pos[n:], window, 4)
    for hq in range(2 * g):
        z = q[:, hq].double() @ c.seqs[0].k[hq // g].double().T * D ** -0.5
        d = lse[:, hq].double() - torch.logsumexp(torch.where(ok, z, -torch.inf), 1)
        assert rms(d) <= RMS, (hq, rms(d))


def marked(c, D, s, sinks, at):
    """Values that show which pairs a query sees: all keys zero, so every seen pair weighs the same; channel i of the values
    marks one pair, half of them around slot `at`, half around the last sink.  Returns the pairs that are marked."""
    n = len(c.seqs[s])
    first = max(0, min(n - D // 2, at - D // 4))
    last = max(0, min(n - D // 2, sinks - D // 4))
    slots = torch.cat([torch.arange(first, first + D // 2), torch.arange(last, last + D // 2)]).cuda()
    v = torch.zeros((n, D), device="cuda")
    v[slots, torch.arange(D, device="cuda")] = 1.0
    for h in range(c.Hkv):
        c.seqs[s].k[h], c.seqs[s].v[h] = torch.zeros_like(c.seqs[s].k[h]), v.to(torch.bfloat16)
    return slots


def check_marked(out, ok, slots):
    """out [rows][D]: 1 / (pairs seen) where the channel's pair is seen, exactly 0 where it is not."""
    want = torch.where(ok[:, slots], 1.0 / ok.sum(1, keepdim=True).double(), 0.0)
    assert torch.equal(out != 0, want != 0)
    assert bool(((out.double() - want).abs() <= 2.0 ** -8 * want + 2.0 ** -20 * want).all())   # (rounded to bf16 once)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks,gap", [(4000, 4, 1), (4001, 0, 1), (3999, 50, 2), (1000, 333, 3), (33, 0, 1)])
def test_windows_end_where_they_should_at_any_length(D, window, sinks, gap):
    n, T, g = 6000, 100, 4
    c = Case(2, g, D, [n], gap=gap, sinks=sinks, cap=n + 64)
    pos = c.seqs[0].pos[0]
    edge = int(torch.searchsorted(pos, pos[n - T // 2] - window + 1))
    slots = marked(c, D, 0, sinks, edge)
    c.cache.append_chunk(0, None, None, [0], keep_lens=[0])
    c.cache.append_chunk(0, torch.stack(c.seqs[0].k, 1), torch.stack(c.seqs[0].v, 1), [n], pos=pos)
    q = c.rand(T, 2 * g)
    out = c.cache.chunk_attn(0, q, [T], window=window, sinks=sinks)
    ok = ref.seen(pos, torch.arange(n - T, n, device="cuda"), pos[n - T:], window, sinks)
    for hq in range(2 * g):
        check_marked(out[:, hq], ok, slots)
    # One token: at every position of the chunk in turn, then with a pair appended behind.
    for j in (*range(0, T, 7), T - 1):
        p = pos[n - T + j:n - T + j + 1]
        got = c.cache.decode_attn_window(0, q[:1], window, sinks, q_pos=p)
        one = ref.seen(pos, torch.tensor([n - 1], device="cuda"), p, window, sinks)
        for hq in range(2 * g):
            check_marked(got[:, hq], one, slots)
    zero = torch.zeros((1, 2, D), dtype=torch.bfloat16, device="cuda")
    for _ in range(20):
        got = c.cache.append_decode_attn_window(0, zero, zero, q[:1], window, sinks)
        pos = torch.cat([pos, pos[-1:] + 1])
        one = ref.seen(pos, torch.tensor([len(pos) - 1], device="cuda"), pos[-1:], window, sinks)
        for hq in range(2 * g):
            check_marked(got[:, hq], one, slots)
    assert c.status() == 0


@pytest.mark.parametrize("T", [5, 60, 200])
def test_a_sequence_alone_and_in_other_batches(T):
    """The pages of all items are cut into equal ranges, so the batch decides where a sequence's items are cut: other partial
    results, the same attention."""
    n, D, g = 3000, 128, 4
    alone = Case(2, g, D, [n], cap=n + 300)
    k, v, q = alone.chunk([T])
    lse = torch.empty((T, 2 * g), device="cuda")
    out = alone.cache.append_chunk_attn(0, k, v, q, [T], lse=lse)
    alone.extend(k, v, [T])
    alone.check_chunk(out, lse, q, [T])
    seq = alone.seqs[0]
    for others, lens in [([40], [3]), ([9000], [1]), ([100] * 30, [7] * 30), ([5000, 0, 17], [300, 64, 0])]:
        c = Case(2, g, D, [*others, 0], seed=9, cap=9700)
        c.cache.prefill(0, len(others), torch.stack([x[:n] for x in seq.k]), torch.stack([x[:n] for x in seq.v]))
        kk, vv, qq = c.chunk(lens)
        full = torch.empty((sum(lens) + T, 2 * g), device="cuda")
        both = c.cache.append_chunk_attn(0, torch.cat([kk, k]), torch.cat([vv, v]), torch.cat([qq, q]), [*lens, T], lse=full)
        alone.check_chunk(both[sum(lens):], full[sum(lens):], q, [T])
        assert rms(full[sum(lens):].double() - lse.double()) <= 2 * RMS
        assert c.status() == 0
