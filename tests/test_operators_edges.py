"""Attention of drafted tokens: NaN that a row sees, graphs that hold only a part of it, weights that add up to one, and its plainest calls: a token that
sees itself, a chain without bits, a denominator of 3e7 like terms.  Bounds are those of test_operators.py unless derived here."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2511_07427_amd.binding import TORCH_DTYPES, PackedCache, tree_scratch  # noqa: E402
from test_operators import D, DEV, HALF, U32, _bits, _check_tree, _drafts, _plain_tree, _random_tree, _retrieved  # noqa: E402

gpu = pytest.mark.gpu


def _filled(dt, bits, U, cap, gen, spoil=None):
    """A packed cache of `cap` random entries a unit, and the values that it holds; spoil(K, V) changes them before they are written."""
    K, V = (torch.randn(U, max(1, cap), D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    if spoil:
        spoil(K, V)
    c = PackedCache.zeros(U, max(1, cap), dt, bits, DEV)
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    return c, K[:, :cap], V[:, :cap]


def _check_with_nan(got, got_lse, ref, dt, L):
    """Rows whose definition is NaN are NaN throughout, the others right.  Returns how many are."""
    gone = ref[1].isnan()
    assert got[gone].isnan().all() and got_lse[gone].isnan().all()
    got, got_lse, ref = got.clone(), got_lse.clone(), [x.clone() for x in ref]
    for x in (got, got_lse, *ref):
        x[gone] = 0
    _check_tree(got, got_lse, ref, dt, L)
    return int(gone.sum())


def _chain(T):
    return torch.ones(T, T, dtype=torch.bool, device=DEV).tril()


# Calls whose rows are one group's, several groups' of a workgroup, several workgroups', and joined from few and from many pieces.
SHAPES = [(2, 1, 1, 0), (2, 1, 4, 33), (2, 5, 3, 700), (1, 9, 4, 6000), (1, 1, 2, 60000), (3, 40, 8, 900), (600, 1, 2, 70)]


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 8), ("bf16", 4), ("f32", 8)])
@pytest.mark.parametrize("U,T,G,cap", SHAPES)
def test_a_query_that_is_nan_gives_nan(dt, bits, U, T, G, cap):
    gen = torch.Generator(DEV).manual_seed(U + T + cap)
    c, K, V = _filled(dt, bits, U, cap, gen)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    Q[0, T - 1, G - 1, 3] = float("nan")
    c.dynakv_packed_attend(torch.full((U,), cap, dtype=torch.int32, device=DEV), Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV))
    for u in range(min(U, 3)):
        ref = _plain_tree(Q[u].double(), K[u].double(), V[u].double(), K1[u].double(), V1[u].double(), _chain(T), D ** -0.5)
        assert _check_with_nan(out[u], lse[u], ref, dt, cap + T) == (1 if u == 0 else 0)


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 4), ("bf16", 8), ("f32", 8)])
@pytest.mark.parametrize("T,G", [(1, 1), (3, 4), (30, 4)])
@pytest.mark.parametrize("cap,first,last", [(1, 0, 1), (33, 32, 33), (65, 64, 65), (65, 63, 64), (5000, 4999, 5000), (20000, 3000, 9000), (700, 0, 700)])
def test_keys_that_are_nan_reach_every_row(dt, bits, T, G, cap, first, last):
    # (one entry by itself in a tile, one at a tile's end, whole pieces, everything)
    gen = torch.Generator(DEV).manual_seed(cap + T)
    U = 2

    def spoil(K, V):
        K[0, first:last, 70] = float("nan")
    c, K, V = _filled(dt, bits, U, cap, gen, spoil)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    c.dynakv_packed_attend(None, Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV))
    assert out[0].isnan().all() and lse[0].isnan().all()
    ref = _plain_tree(Q[1].double(), K[1].double(), V[1].double(), K1[1].double(), V1[1].double(), _chain(T), D ** -0.5)
    _check_tree(out[1], lse[1], ref, dt, cap + T)


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 8), ("bf16", 4), ("f32", 8)])
@pytest.mark.parametrize("U,T,G,cap", SHAPES)
def test_drafted_keys_that_are_nan_reach_the_rows_that_see_them(dt, bits, U, T, G, cap):
    gen = torch.Generator(DEV).manual_seed(U + T + cap)
    c, K, V = _filled(dt, bits, U, cap, gen)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    K1[0, T - 1] = float("nan")
    seen = _random_tree(U, T, gen)
    seen[0, :, T - 1] = False
    seen[0, T - 1, T - 1] = True                                 # the last node sees itself, no other does
    if T > 1:
        seen[0, 0] = False
    c.dynakv_packed_attend(torch.full((U,), cap, dtype=torch.int32, device=DEV), Q, K1, V1, _bits(seen), out, lse, tree_scratch(U, T, G, DEV))
    for u in range(min(U, 3)):
        ref = _plain_tree(Q[u].double(), K[u].double(), V[u].double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
        assert _check_with_nan(out[u], lse[u], ref, dt, cap + T) == (G if u == 0 else 0)


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("U,T,G,budget", [(1, 1, 4, 20), (2, 6, 3, 300), (1, 40, 4, 900)])
def test_nan_over_a_retrieval(dt, U, T, G, budget):
    ix, K, V, at, gen, _, _ = _retrieved(dt, U, G, 1000, 100, budget, T)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    Q[0, 0, 0, 5] = float("nan")
    K1[U - 1, T - 1, 9] = float("nan")
    ix.dynakv_attend_tree(Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV))
    for u in range(U):
        ref = _plain_tree(Q[u].double(), K[u, at[u]].double(), V[u, at[u]].double(), K1[u].double(), V1[u].double(), _chain(T), D ** -0.5)
        gone = _check_with_nan(out[u], lse[u], ref, dt, len(at[u]) + T)
        assert gone == (G if u == U - 1 else 0) + (1 if u == 0 else 0) - (1 if u == 0 == U - 1 and T == 1 else 0)


@gpu
def test_a_retrieval_that_is_only_captured_lists_nothing_outside_its_graph():
    """Capturing a retrieval does not run it: attention over its list belongs into the same graph, and a graph's attention needs its own retrieval."""
    U, T, G, budget = 2, 3, 4, 100
    ix, K, V, at, gen, Q0, flat = _retrieved("f16", U, G, 300, 20, budget, 4)
    Q, K1, V1, out, lse = _drafts("f16", U, T, G, gen)
    scratch, side, other = tree_scratch(U, T, G, DEV), torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()

    def retrieve():
        ix.dynakv_retrieve_attend(Q0, budget, flat, None)

    def attend():
        ix.dynakv_attend_tree(Q, K1, V1, None, out, lse, scratch)

    def refused():
        out.fill_(3.0)
        with pytest.raises(RuntimeError, match="out of order"):
            attend()
        assert torch.cuda.is_current_stream_capturing() or bool((out == 3.0).all())
    # (the list of the eager retrieval before is there throughout: no call reads what was never written)
    before, alone, later, both = (torch.cuda.CUDAGraph() for _ in range(4))
    with torch.cuda.graph(before, stream=side):
        refused()                                                # the list is not this graph's
    attend()                                                     # nothing has changed for eager calls
    with torch.cuda.graph(alone, stream=side):
        retrieve()
    refused()                                                    # the retrieval has not run
    with torch.cuda.graph(later, stream=side):
        refused()                                                # it is another graph's
    with torch.cuda.graph(both, stream=side):
        retrieve()
        other.wait_stream(side)
        with torch.cuda.stream(other):
            attend()                                             # on a stream that joins the capture
        side.wait_stream(other)
    refused()
    for i in range(4):
        Q0.copy_(torch.randn(Q0.shape, generator=gen, device=DEV))
        out.fill_(9.0)
        both.replay()
        torch.cuda.synchronize()
        got = out.clone()
        retrieve()
        attend()
        assert torch.equal(out, got), i


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 8), ("f16", 4), ("bf16", 8), ("bf16", 4), ("f32", 8), ("f32", 4)])
@pytest.mark.parametrize("U,T,G,cap", [(3, 1, 1, 1), (2, 1, 8, 64), (2, 1, 3, 4097), (600, 1, 2, 50), (2, 2, 4, 33), (3, 33, 3, 300), (1, 64, 16, 700)])
def test_a_chain_without_bits(dt, bits, U, T, G, cap):
    # node i sees drafted tokens 0..i; one token: decoding, it sees the cache and itself
    gen = torch.Generator(DEV).manual_seed(U + T + cap)
    c, K, V = _filled(dt, bits, U, cap, gen)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    K1[:, T - 1] += Q[:, T - 1, 0]                               # a weight that counts
    scratch = tree_scratch(U, T, G, DEV)
    for lengths in (None, torch.zeros(U, dtype=torch.int32, device=DEV)):
        c.dynakv_packed_attend(lengths, Q, K1, V1, None, out, lse, scratch)
        n = cap if lengths is None else 0
        for u in range(min(U, 3)):
            ref = _plain_tree(Q[u].double(), K[u, :n].double(), V[u, :n].double(), K1[u].double(), V1[u].double(), _chain(T), D ** -0.5)
            _check_tree(out[u], lse[u], ref, dt, n + T)
        again, lse2 = torch.empty_like(out), torch.empty_like(lse)
        c.dynakv_packed_attend(lengths, Q, K1, V1, _bits(_chain(T).expand(U, T, T)), again, lse2, scratch)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("U,T,G,budget", [(2, 1, 4, 300), (1, 1, 7, 1), (3, 5, 2, 200)])
def test_a_chain_without_bits_over_a_retrieval(dt, U, T, G, budget):
    ix, K, V, at, gen, _, _ = _retrieved(dt, U, G, 900, 60, budget, T)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    ix.dynakv_attend_tree(Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV))
    for u in range(U):
        ref = _plain_tree(Q[u].double(), K[u, at[u]].double(), V[u, at[u]].double(), K1[u].double(), V1[u].double(), _chain(T), D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, len(at[u]) + T)


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_every_entry_beyond_32_bits_counts(dt):
    """2^25 + 77 entries, 4.3 GB of codes, of which 50 are random and the others are alike: key 0, value 1 in column 7.  With a largest logit near 16 both
    kinds have a share in the denominator, so an entry left out or taken twice for every few hundred shows."""
    cap, G = (1 << 25) + 77, 2
    gen = torch.Generator(DEV).manual_seed(3)
    c = PackedCache.zeros(1, cap, dt, 8, DEV)
    c.tensors[2][0, :, 7] = 1                                    # value codes and their block's scale, 2^0
    c.tensors[3][0, :, 0] = 127
    K, V = (torch.randn(1, 50, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    start = torch.tensor([cap - 50], dtype=torch.int32, device=DEV)
    c.dynakv_packed_write(K, V, start)
    k, v = torch.empty_like(K), torch.empty_like(V)
    c.dynakv_packed_read((start[:, None] + torch.arange(50, device=DEV, dtype=torch.int32)).contiguous(), k, v)
    Q = (k[:, :1, None, :].float() * (16 * D ** 0.5 / k[0, 0].float().square().sum())).to(K.dtype).expand(1, 1, G, D).contiguous()
    out, lse = torch.empty_like(Q), torch.empty(1, 1, G, device=DEV)
    c.dynakv_packed_attend(None, Q, None, None, None, out, lse, tree_scratch(1, 1, G, DEV))
    logit = (Q[0, 0].double() @ k[0].double().T) / D ** 0.5
    like, weight = float(cap - 50), logit.exp()
    den = weight.sum(-1) + like
    one = torch.zeros(D, dtype=torch.float64, device=DEV)
    one[7] = 1.0
    want, spread = (weight @ v[0].double() + like * one) / den[:, None], (weight @ v[0].double().abs() + like * one) / den[:, None]
    assert 0.05 < float(like / den[0]) < 0.95                    # (both kinds count)
    # The bound: one unit of few rows is shared by 256 workgroups or more, the entries of each by at least four wavefronts, 2^15 entries each; every addition of
    # such a sum is off by at most u of the sum so far: 2^15 u = 2^-9, for the denominator and for the weighted values.  The weights: the logits'
    # error and the exponential's, as in _check_tree, and h in 16 bits; float16's small weights are off by half a step of 2^-31 of the largest,
    # e^-16 of it or more here: 2^-32 e^16 = 0.0021 of each.  An output of float16 below 2^-14 is rounded to steps of 2^-24: off by 2^-25.
    delta = 132 * U32 * float((Q[0, 0].double().abs() @ k[0].double().abs().T).max()) / D ** 0.5
    sums = 2.0 ** -9 + 2 * delta + 2.0 ** -21
    weights = HALF[dt] if dt != "f32" else 0.0
    if dt == "f16":
        weights = weights + 2.0 ** -32 * float(logit.max().exp())
    bound = spread * (2 * sums + weights) * 1.01 + HALF[dt] * want.abs() + (2.0 ** -25 if dt == "f16" else 0.0)
    assert bool(((out[0, 0].double() - want).abs() <= bound).all())
    assert bool(((lse[0, 0].double() - den.log()).abs() <= 1.01 * sums + 64 * U32).all())


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("U,T,G,cap", [(300, 1, 16, 32), (20, 5, 16, 30), (2, 5, 3, 700), (1, 9, 4, 3000), (3, 40, 8, 900)])
def test_equal_values_come_out_as_they_are(dt, U, T, G, cap):
    """A mean of equal values, with equal weights but for one, so that all are rounded alike: whatever a weight is rounded to, the weights add up to one.  What
    is left are float32 sums, (3000 / 4 + 64) u = 5e-5 at most, which the output's rounding, half a step of 2^-12 or more of a value of 16 bits, takes back."""
    gen = torch.Generator(DEV).manual_seed(U + T + cap)
    value = torch.arange(D, device=DEV).remainder(32) + 96.0     # codes of 8 bits with scale 1

    def spoil(K, V):
        V[:], K[:, 2:] = value, K[:, 1:2].clone()
    c, K, V = _filled(dt, 8, U, cap, gen, spoil)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    V1[:], K1[:] = value, K[:, 1:2]
    c.dynakv_packed_attend(None, Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV))
    assert torch.equal(out.float(), value.expand_as(out))


@gpu
def test_the_largest_values_stay_finite():
    """32 drafted tokens with the largest value of float16, one with weight 1, the others with a weight whose rounding to 11 bits goes up by almost half a step,
    1/2 (1 + 0.51 2^-10).  Weights whose sum is taken before they are rounded would give 1.00045 times that value: infinity."""
    T = 32
    Q, K1 = (torch.zeros(1, T, *s, D, dtype=torch.float16, device=DEV) for s in ((1,), ()))
    logit = torch.log(torch.tensor(0.5 * (1 + 0.51 * 2.0 ** -10), dtype=torch.float64))
    Q[..., 0], Q[..., 1] = 1.0, 2.0 ** -11
    K1[:, 1:, 0] = logit.half().item()
    K1[:, 1:, 1] = (logit - logit.half().double()).item() * 2.0 ** 11
    V1 = torch.full_like(K1, torch.finfo(torch.float16).max)
    out, lse = torch.empty_like(Q), torch.empty(1, T, 1, device=DEV)
    c = PackedCache.zeros(1, 1, "f16", 8, DEV)
    c.dynakv_packed_attend(torch.zeros(1, dtype=torch.int32, device=DEV), Q, K1, V1, torch.full((1, T), -1, dtype=torch.int64, device=DEV), out, lse,
                           tree_scratch(1, T, 1, DEV), softmax_scale=1.0)
    assert torch.equal(out, V1[0, 0].expand_as(out))
