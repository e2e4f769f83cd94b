"""Operators beside the index: norm + rotation by unit, packed caches, attention of drafted tokens.

Every kernel against a plain float64 implementation.  Tolerances count roundings: h = half a step of the storage type
(2^-11 of float16, 2^-8 of bfloat16, 2^-24 of float32), u = 2^-24 for float32 arithmetic; each bound is written where it is used."""
import ctypes as C
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2511_07427_amd import binding  # noqa: E402
from paper_2511_07427_amd.binding import TORCH_DTYPES, PackedCache, dynakv_norm_rope, tree_scratch  # noqa: E402

DEV = "cuda:0"
D = 128
HALF = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U32 = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_07427_amd.build import build
        build()
    return binding.load()


# ------------------------------------------------------------------------------------------- refusals (no GPU needed)
FAKE = 1 << 20


def _heads(**kw):
    c = dict(dtype=1, n_seqs=2, n_tokens=3, n_kv_heads=2, group_size=4, head_dim=128, rotary_dim=128, interleaved=0, eps=1e-6,
             q_seq_stride=2048 * 8, q_token_stride=2048, k_seq_stride=2048, k_token_stride=256, v_seq_stride=2048, v_token_stride=256)
    c.update(kw)
    return binding._Heads(**c)


def test_norm_rope_refuses_what_it_does_not_take(lib):
    def call(c, q=FAKE, k=FAKE, v=FAKE, wq=FAKE, wk=None, freq=FAKE, pos=FAKE, Q=FAKE, K=FAKE, V=FAKE):
        return lib.dynakv_norm_rope(C.byref(c) if c is not None else None, q, k, v, wq, wk, freq, pos, Q, K, V, None)
    assert call(None) == 1
    for bad in (dict(dtype=3), dict(dtype=-1), dict(n_seqs=0), dict(n_tokens=0), dict(n_kv_heads=0), dict(group_size=0), dict(group_size=17),
                dict(head_dim=64), dict(rotary_dim=4), dict(rotary_dim=136), dict(rotary_dim=-8), dict(interleaved=2), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(q_token_stride=2052), dict(k_seq_stride=4), dict(v_token_stride=129),
                dict(n_seqs=1 << 20, n_tokens=1 << 20), dict(n_kv_heads=1 << 20)):
        assert call(_heads(**bad)) == 1, bad
    c = _heads()
    assert call(c, freq=None) == 1 and call(c, pos=None) == 1
    for one in (dict(q=None), dict(Q=None), dict(k=None), dict(K=None), dict(v=None), dict(V=None)):
        assert call(c, **one) == 1, one                       # an input without its output, an output without its input
    for one in (dict(q=FAKE + 8), dict(V=FAKE + 8), dict(wq=FAKE + 2), dict(pos=FAKE + 2)):
        assert call(c, **one) == 1, one
    assert call(_heads(dtype=0, q_token_stride=2052), q=None, Q=None, k=None, K=None, v=None, V=None) == 0     # nothing to do


def _packed(**kw):
    c = dict(n_units=2, capacity=64, head_dim=128, dtype=1, bits=8, k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE)
    c.update(kw)
    return binding._Packed(**c)


def test_packed_calls_refuse_what_they_do_not_take(lib):
    bad = (dict(n_units=0), dict(capacity=0), dict(capacity=(1 << 30) + 1), dict(head_dim=64), dict(dtype=3), dict(bits=2), dict(k_codes=None), dict(v_scales=None),
           dict(k_codes=FAKE + 8), dict(v_scales=FAKE + 2))
    for b in bad:
        c = C.byref(_packed(**b))
        assert lib.dynakv_packed_write(c, FAKE, FAKE, 1, None, None, None) == 1, b
        assert lib.dynakv_packed_read(c, None, 1, FAKE, FAKE, None) == 1, b
        assert lib.dynakv_packed_attend(c, None, FAKE, 1, 1, None, None, None, 0.0, FAKE, None, FAKE, 1 << 20, None) == 1, b
    c = C.byref(_packed())
    assert lib.dynakv_packed_write(None, FAKE, FAKE, 1, None, None, None) == 1
    for K, V, n in ((None, FAKE, 1), (FAKE, None, 1), (FAKE, FAKE, -1), (FAKE + 8, FAKE, 1), (FAKE, FAKE, 1 << 30)):
        assert lib.dynakv_packed_write(c, K, V, n, None, None, None) == 1
        assert lib.dynakv_packed_read(c, None, n, K, V, None) == 1
    assert lib.dynakv_packed_write(c, FAKE, FAKE, 1, FAKE + 2, None, None) == 1
    assert lib.dynakv_packed_write(c, FAKE, FAKE, 0, None, None, None) == 0
    assert lib.dynakv_packed_read(c, None, 0, FAKE, FAKE, None) == 0


def test_attentions_of_drafted_tokens_refuse_what_they_do_not_take(lib):
    assert lib.dynakv_tree_scratch_bytes(2, 3, 4) > 0
    for u, t, g in ((0, 1, 1), (1, 0, 1), (1, 65, 1), (1, 1, 0), (1, 1, 17), (-1, 1, 1)):
        assert lib.dynakv_tree_scratch_bytes(u, t, g) == 0
    c, need = C.byref(_packed()), lib.dynakv_tree_scratch_bytes(2, 5, 4)

    def call(Q=FAKE, T=5, G=4, k=FAKE, v=FAKE, tree=FAKE, scale=0.0, out=FAKE, lse=FAKE, scratch=FAKE, n=need, lengths=FAKE):
        return lib.dynakv_packed_attend(c, lengths, Q, T, G, k, v, tree, scale, out, lse, scratch, n, None)
    for bad in (dict(Q=None), dict(out=None), dict(scratch=None), dict(T=0), dict(T=65), dict(G=0), dict(G=17), dict(k=None), dict(v=None),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(Q=FAKE + 8), dict(out=FAKE + 8), dict(k=FAKE + 8),
                dict(tree=FAKE + 4), dict(lse=FAKE + 2), dict(scratch=FAKE + 8), dict(lengths=FAKE + 2)):
        assert call(**bad) == 1, bad
    assert call(n=need - 1) == 2
    # the index: a handle without a retrieval
    cfg = binding._cfg(binding.Config(2, 4, "f16", 8, 32, 256))
    h, size = C.c_void_p(), lib.dynakv_workspace_bytes(C.byref(cfg))
    assert lib.dynakv_create(C.byref(cfg), FAKE, size, C.byref(h)) == 0
    assert lib.dynakv_attend_tree(h, FAKE, 5, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, None) == 3
    assert lib.dynakv_attend_tree(None, FAKE, 5, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, None) == 1
    assert lib.dynakv_attend_tree(h, FAKE, 65, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need, None) == 1
    assert lib.dynakv_attend_tree(h, FAKE, 5, FAKE, None, FAKE, FAKE, FAKE, FAKE, need, None) == 1
    assert lib.dynakv_attend_tree(h, FAKE, 5, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need - 1, None) == 2
    assert lib.dynakv_destroy(h) == 0


def test_sizes_beyond_what_one_launch_holds_are_refused(lib):
    """Fewer than 2^32 work-items to a launch."""
    def heads(B, T, H, G):
        c = _heads(n_seqs=B, n_tokens=T, n_kv_heads=H, group_size=G)
        return lib.dynakv_norm_rope(C.byref(c), FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, None)
    assert heads(1, (1 << 27) // 3 + 1, 1, 1) == 1 and heads(1 << 13, 1 << 13, 1, 2) == 1
    c = C.byref(_packed(n_units=4, capacity=1 << 30))
    assert lib.dynakv_packed_write(c, FAKE, FAKE, 1 << 26, None, None, None) == 1
    assert lib.dynakv_packed_read(c, None, 1 << 26, FAKE, FAKE, None) == 1
    for U, T, G in ((1 << 22, 1, 1), (1 << 18, 64, 16)):
        assert lib.dynakv_tree_scratch_bytes(U, T, G) == 0
        c = C.byref(_packed(n_units=U, capacity=1))
        assert lib.dynakv_packed_attend(c, None, FAKE, T, G, None, None, None, 0.0, FAKE, None, FAKE, 1 << 62, None) == 1


def test_structs_match_the_header():
    assert C.sizeof(binding._Heads) == 9 * 4 + 4 + 6 * 8
    assert C.sizeof(binding._Packed) == 5 * 4 + 4 + 4 * 8


def test_the_binding_refuses_tensors_off_the_gpu():
    x = torch.zeros(1, 1, 4, 128, dtype=torch.float16)
    with pytest.raises(ValueError, match="GPU"):
        dynakv_norm_rope(x, None, None, torch.zeros(1, 1, dtype=torch.int32), torch.zeros(4, 1, 1, 128, dtype=torch.float16), None, None)
    with pytest.raises(ValueError, match="GPU"):
        PackedCache.zeros(1, 4, "f16", 8, device="cpu")
    with pytest.raises(ValueError, match="8 or 4 bits"):
        PackedCache.zeros(1, 4, "f16", 16, device="cpu")


# --------------------------------------------------------------------------------------------------- norm + rotation
def _plain_rows(x, w, pos, freq, interleaved, eps):
    """x [B, T, heads, D] float64 -> (result, bound on its float32 arithmetic)."""
    if w is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    mag = x.abs()
    if freq is not None:
        h = freq.numel()
        ang = pos.double()[:, :, None, None] * freq.double()
        c, s = ang.cos(), ang.sin()
        y = x.clone()
        if interleaved:
            a, b = x[..., 0:2 * h:2], x[..., 1:2 * h:2]
            y[..., 0:2 * h:2], y[..., 1:2 * h:2] = a * c - b * s, b * c + a * s
            m = a.abs() + b.abs()
            mag[..., 0:2 * h:2], mag[..., 1:2 * h:2] = m, m
        else:
            a, b = x[..., :h], x[..., h:2 * h]
            y[..., :h], y[..., h:2 * h] = a * c - b * s, b * c + a * s
            m = a.abs() + b.abs()
            mag[..., :h], mag[..., h:2 * h] = m, m
        x = y
    # a float32 sum of 128 squares in 8 + 4 steps: 12 u, halved by the root; root, two products: 4 u; sine and cosine of an angle
    # rounded to float32 within half a turn (pi u) to 4 u, product and difference 2 u: 10 u + 6 u + slack of the library's root
    return x, 24 * U32 * mag


def _check_rows(got, want, bound, dt):
    got, lim = got.double(), bound + HALF[dt] * want.abs() + (2.0 ** -25 if dt == "f16" else 0.0)   # float16 below 2^-14: steps of 2^-24
    worst = ((got - want).abs() - lim).max().item()
    assert worst <= 0, worst


def _fused_rows(dt, B, T, H, G, gen):
    W = (H * G + 2 * H) * D
    fused = torch.randn(B, T, W, generator=gen, device=DEV).to(TORCH_DTYPES[dt])
    q, k, v = fused.split([H * G * D, H * D, H * D], dim=2)
    return q.unflatten(2, (H * G, D)), k.unflatten(2, (H, D)), v.unflatten(2, (H, D))


def _outputs(dt, B, T, H, G, fill=7.0):
    t = TORCH_DTYPES[dt]
    return [torch.full(s, fill, dtype=t, device=DEV) for s in ((B * H, T, G, D), (B * H, T, D), (B * H, T, D))]


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("B,T,H,G,rot,interleaved,norm", [
    (1, 1, 8, 4, 128, False, True), (3, 5, 2, 7, 128, True, True), (2, 33, 1, 1, 64, False, True), (5, 2, 3, 16, 96, True, False),
    (1, 129, 4, 3, 8, False, False), (2, 7, 5, 2, 0, False, True), (1, 3, 7, 6, 120, False, True), (300, 1, 2, 4, 128, False, True),
    (2, 700, 1, 5, 32, True, True), (3, 701, 1, 3, 128, False, True), (1, 2100, 1, 1, 32, False, True), (2, 1100, 2, 9, 64, False, True),
    (1, 1500, 4, 8, 128, False, True), (1, 401, 16, 8, 128, True, True), (1, 2, 16, 16, 96, False, True)])
def test_norm_rope(dt, B, T, H, G, rot, interleaved, norm):
    gen = torch.Generator(DEV).manual_seed(B * 1000 + T)
    q, k, v = _fused_rows(dt, B, T, H, G, gen)
    pos = torch.randint(0, 131072, (B, T), generator=gen, device=DEV, dtype=torch.int32)
    pos[0, 0] = 0
    pos[-1, -1] = 2 ** 31 - 1
    pad = torch.rand(B, T, generator=gen, device=DEV) < 0.2
    pad[0, 0] = False
    pos[pad] = -1 - pos[pad] % 5
    w = (1 + 0.3 * torch.randn(2, D, generator=gen, device=DEV)).to(TORCH_DTYPES[dt]) if norm else (None, None)
    freq = (10000.0 ** (-torch.arange(0, rot, 2, device=DEV).double() / max(rot, 1))).float() if rot else None
    Q, K, V = _outputs(dt, B, T, H, G)
    dynakv_norm_rope(q, k, v, pos, Q, K, V, w[0], w[1], freq, 1e-5, interleaved)
    keep = pos >= 0
    for x, y, ww in ((q, Q, w[0]), (k, K, w[1])):
        want, bound = _plain_rows(x.double(), None if ww is None else ww.double(), pos.clamp_min(0), freq, interleaved, 1e-5)
        got = y.reshape(B, H, T, -1, D).transpose(1, 2).reshape(B, T, -1, D)
        _check_rows(got[keep], want[keep], bound[keep], dt)
        assert (got[~keep] == 7.0).all()                       # padding is left as it was
    got = V.reshape(B, H, T, D).transpose(1, 2)
    assert torch.equal(got[keep], v[keep]) and (got[~keep] == 7.0).all()


@gpu
def test_norm_rope_alone_strided_and_of_extreme_rows():
    gen = torch.Generator(DEV).manual_seed(5)
    # keys alone, tokens in reverse memory order of a wider array, sequences overlapping in memory
    base = torch.randn(64, 5, D, generator=gen, device=DEV).half()
    k = base.as_strided((3, 4, 2, D), (5 * D, 2 * 5 * D, D, 1), D)
    pos = torch.arange(12, dtype=torch.int32, device=DEV).reshape(3, 4)
    K = torch.empty(6, 4, D, dtype=torch.float16, device=DEV)
    dynakv_norm_rope(None, k, None, pos, None, K, None)
    assert torch.equal(K, k.permute(0, 2, 1, 3).reshape(6, 4, D))          # no weight, no frequencies: a copy by unit
    # an all-zero row with eps, a row of the type's largest values, infinities and NaN stay in their rows
    for dt, big in (("f16", 60000.0), ("bf16", 1e18), ("f32", 1e18)):
        x = torch.randn(1, 6, 1, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt])
        x[0, 1] = 0
        x[0, 2] = big
        x[0, 3, 0, 17] = float("inf")
        x[0, 4, 0, 5] = float("nan")
        w = torch.ones(D, dtype=x.dtype, device=DEV)
        out = torch.zeros(1, 6, D, dtype=x.dtype, device=DEV)
        dynakv_norm_rope(None, x, None, torch.zeros(1, 6, dtype=torch.int32, device=DEV), None, out, None, None, w)
        assert (out[0, 1] == 0).all() and torch.allclose(out[0, 2].float(), torch.ones(D, device=DEV), atol=2 * HALF[dt])
        assert out[0, 4].isnan().all() and out[0, [0, 1, 2, 5]].isfinite().all()


@gpu
def test_norm_rope_refusals_of_the_binding():
    q, k, v = _fused_rows("f16", 2, 3, 2, 4, torch.Generator(DEV).manual_seed(1))
    pos = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    Q, K, V = _outputs("f16", 2, 3, 2, 4)
    freq = torch.ones(64, device=DEV)
    for args in ((q, k, v, pos.long(), Q, K, V), (q, k, v, pos, Q, K, None), (q.float(), k, v, pos, Q, K, V), (q, k, v, pos, Q[:, :2], K, V),
                 (q, k.transpose(1, 2), v, pos, Q, K, V), (q[:, :, :7], k, v, pos, Q, K, V), (q.double(), None, None, pos, Q.double(), None, None)):
        with pytest.raises(ValueError):
            dynakv_norm_rope(*args, inv_freq=freq)
    with pytest.raises(ValueError):
        dynakv_norm_rope(q, k, v, pos, Q, K, V, inv_freq=freq.double())
    with pytest.raises(RuntimeError):
        dynakv_norm_rope(q, k, v, pos, Q, K, V, inv_freq=freq[:3])          # six rotated elements
    assert (Q == 7.0).all() and (K == 7.0).all()


# ------------------------------------------------------------------------------------------------------ packed caches
def _plain_pack(x, dt, bits):
    """The values that a packed cache of type dt holds for x, float64, and the scale bytes."""
    qmax = 127 if bits == 8 else 7
    top = 16 if dt == "f16" else 128
    lo, hi = (-24 if dt == "f16" else -126), top - (bits - 1)
    b = x.double().cpu().numpy().reshape(*x.shape[:-1], 4, 32)
    amax = np.abs(b).max(-1)
    with np.errstate(invalid="ignore", over="ignore"):
        m, e = np.frexp(amax / qmax)                            # division of a value of the type by 127 or 7 hits a power of two only exactly
        e = np.where(m == 0.5, e - 1, e)
        e = np.clip(np.where(amax == 0, lo, e), lo, hi)
        step = np.ldexp(1.0, e)[..., None]
        y = np.clip(np.rint(b / step), -qmax, qmax) * step
    bad = ~np.isfinite(amax)
    y[bad] = np.nan
    s = np.where(bad, 255, e + 127)
    return torch.from_numpy(y.reshape(x.shape)), torch.from_numpy(s.astype(np.uint8))


def _rows(dt, U, n, gen):
    x = torch.randn(U, n, D, generator=gen, device=DEV) * torch.exp(2 * torch.randn(U, n, 1, generator=gen, device=DEV))
    x[..., 3] *= 30
    return x.to(TORCH_DTYPES[dt])


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("U,n,cap", [(1, 1, 1), (3, 5, 40), (128, 1, 9), (2, 777, 1000), (17, 33, 33)])
def test_packed_rows_are_the_nearest_of_their_scale(dt, bits, U, n, cap):
    gen = torch.Generator(DEV).manual_seed(n)
    K, V = _rows(dt, U, n, gen), _rows(dt, U, n, gen)
    c = PackedCache.zeros(U, cap, dt, bits, DEV)
    start = torch.randint(0, cap - n + 1, (U,), generator=gen, device=DEV, dtype=torch.int32)
    c.dynakv_packed_write(K, V, start)
    pos = start[:, None] + torch.arange(n, device=DEV, dtype=torch.int32)
    k, v = torch.empty_like(K), torch.empty_like(V)
    c.dynakv_packed_read(pos.contiguous(), k, v)
    for x, y, scales in ((K, k, c.tensors[1]), (V, v, c.tensors[3])):
        want, s = _plain_pack(x, dt, bits)
        assert torch.equal(y.double().cpu(), want)               # exactly: the type holds every code times its scale
        assert torch.equal(scales[torch.arange(U, device=DEV)[:, None], pos.long()].cpu(), s)
    # in another order, some twice, some outside
    order = torch.randint(-2, cap + 2, (U, 2 * n + 3), generator=gen, device=DEV, dtype=torch.int32)
    k2 = torch.full((U, 2 * n + 3, D), 5.0, dtype=K.dtype, device=DEV)
    v2 = k2.clone()
    c.dynakv_packed_read(order, k2, v2)
    full_k, full_v = (torch.empty(U, cap, D, dtype=K.dtype, device=DEV) for _ in range(2))
    c.dynakv_packed_read(None, full_k, full_v)
    out = (order < 0) | (order >= cap)
    at = order.clamp(0, cap - 1).long()[:, :, None].expand(-1, -1, D)
    for got, full in ((k2, full_k), (v2, full_v)):
        assert torch.equal(got, torch.where(out[:, :, None], torch.full_like(got, 5.0), torch.gather(full, 1, at)))


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bits", [8, 4])
def test_packed_edges_of_the_type(dt, bits):
    t = TORCH_DTYPES[dt]
    fi = torch.finfo(t)
    qmax = 127.0 if bits == 8 else 7.0
    rows = torch.zeros(1, 16, D, dtype=torch.float64)
    rows[0, 1] = fi.max
    rows[0, 2] = -fi.max
    rows[0, 3, 5] = fi.smallest_normal
    rows[0, 4, 5] = float(torch.tensor(fi.smallest_normal, dtype=torch.float64) * fi.eps)        # the smallest value there is
    rows[0, 5, :32] = torch.linspace(-qmax, qmax, 32, dtype=torch.float64)                        # the largest code exactly
    rows[0, 6, :32] = torch.linspace(-qmax - 1, qmax + 1, 32, dtype=torch.float64)                # one code too many: the next scale
    rows[0, 7] = torch.arange(D, dtype=torch.float64) - 63.5                                     # ties
    rows[0, 8, 40] = float("inf")
    rows[0, 9, 100] = float("nan")
    rows[0, 10, 0] = -float("inf")
    rows[0, 11] = fi.max / 2
    rows[0, 12] = fi.max * (1 - fi.eps)
    rows[0, 13, ::3] = 1.0
    rows[0, 14, :] = torch.tensor([1.5, -0.5, 0.25, 8.0]).double().repeat(32)
    x = rows.to(t).to(DEV)
    c = PackedCache.zeros(1, 16, dt, bits, DEV)
    c.dynakv_packed_write(x, -x)
    k, v = torch.empty_like(x), torch.empty_like(x)
    c.dynakv_packed_read(None, k, v)
    for src, got in ((x, k), (-x, v)):
        want, _ = _plain_pack(src, dt, bits)
        assert torch.equal(got.double().cpu().nan_to_num(nan=12345.0), want.nan_to_num(nan=12345.0))
        assert torch.equal(got.isnan().cpu(), want.isnan()) and not got.isinf().any()


@gpu
@pytest.mark.parametrize("bits", [8, 4])
def test_packed_writes_leave_the_rest_alone(bits):
    U, cap, n = 5, 20, 7
    gen = torch.Generator(DEV).manual_seed(2)
    K, V = _rows("f16", U, n, gen), _rows("f16", U, n, gen)
    c = PackedCache.zeros(U, cap, "f16", bits, DEV)
    for t in c.tensors:
        t.fill_(113)
    start = torch.tensor([0, -3, 16, 2 ** 31 - 3, 13], dtype=torch.int32, device=DEV)
    count = torch.tensor([3, 7, 100, 7, -1], dtype=torch.int32, device=DEV)
    c.dynakv_packed_write(K, V, start, count)
    ref = PackedCache.zeros(U, n, "f16", bits, DEV)
    ref.dynakv_packed_write(K, V)
    written = {(0, i): (0, i) for i in range(3)}
    written.update({(1, i - 3): (1, i) for i in range(3, 7)})
    written.update({(2, 16 + i): (2, i) for i in range(4)})
    for got, want in zip(c.tensors, ref.tensors):
        expect = torch.full_like(got, 113)
        for (u, p), (uu, i) in written.items():
            expect[u, p] = want[uu, i]
        assert torch.equal(got, expect)


@gpu
def test_packed_offsets_beyond_32_bits():
    cap = (1 << 25) + 77                                        # 4.3 GB of codes for the keys, as many for the values
    c = PackedCache.zeros(1, cap, "bf16", 8, DEV)
    gen = torch.Generator(DEV).manual_seed(3)
    K, V = torch.randn(1, 50, D, generator=gen, device=DEV).bfloat16(), torch.randn(1, 50, D, generator=gen, device=DEV).bfloat16()
    start = torch.tensor([cap - 50], dtype=torch.int32, device=DEV)
    c.dynakv_packed_write(K, V, start)
    k, v = torch.empty_like(K), torch.empty_like(V)
    c.dynakv_packed_read((start[:, None] + torch.arange(50, device=DEV, dtype=torch.int32)).contiguous(), k, v)
    assert torch.equal(k.double().cpu(), _plain_pack(K, "bf16", 8)[0]) and torch.equal(v.double().cpu(), _plain_pack(V, "bf16", 8)[0])
    # attention over all of it: cap - 50 entries with logit 0 and value 0, and those 50
    Q = (20 * k[:, :1, None, :].float()).bfloat16().expand(1, 1, 2, D).contiguous()
    out, lse = torch.empty_like(Q), torch.empty(1, 1, 2, device=DEV)
    c.dynakv_packed_attend(None, Q, None, None, None, out, lse, tree_scratch(1, 1, 2, DEV))
    logit = (Q[0, 0].double() @ k[0].double().T) / D ** 0.5
    den = logit.exp().sum(-1) + (cap - 50)
    want = (logit.exp() @ v[0].double()) / den[:, None]
    h = HALF["bf16"]
    delta = 132 * U32 * (Q[0, 0].double().abs() @ k[0].double().abs().T).max() / D ** 0.5
    bound = (logit.exp() @ v[0].double().abs()) / den[:, None] * (h + 2 * delta + 2e-5) + h * want.abs()
    # a weight under 2^-126 of the largest is below float32's normal range and may vanish: 50 of them, values under 8: 400 * 2^-126
    bound = bound + 1e-30
    assert bool(((out[0, 0].double() - want).abs() <= bound).all())
    assert bool(((lse[0, 0].double() - den.log()).abs() <= 1e-4).all())     # 3e7 terms of a float32 sum in 32-entry and wavefront parts


# ----------------------------------------------------------------------------------------------- calls beyond the caches
# More than 256 MiB: the kernels' accesses go past the caches there.  The rows are those of calls on parts of them, to the bit.
@gpu
@pytest.mark.parametrize("dt,T,H,G,rot,interleaved", [("bf16", 6601, 8, 8, 128, False), ("f16", 45003, 2, 4, 64, False), ("f32", 13305, 4, 3, 96, True)])
def test_norm_rope_of_more_than_the_caches_hold(dt, T, H, G, rot, interleaved):
    t = TORCH_DTYPES[dt]
    gen = torch.Generator(DEV).manual_seed(T)
    x = torch.randn(1, T, (G + 2) * H, D, generator=gen, device=DEV).to(t)
    assert 2 * x.numel() * x.element_size() > 256 << 20
    w = (1 + 0.1 * torch.randn(D, generator=gen, device=DEV)).to(t)
    freq = torch.rand(rot // 2, generator=gen, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)[None].contiguous()
    pos[0, T // 3] = -1

    def call(a, b):
        rows, n = x[:, a:b], b - a
        out = [torch.full(s, 3.0, dtype=t, device=DEV) for s in ((H, n, G, D), (H, n, D), (H, n, D))]
        dynakv_norm_rope(rows[:, :, :H * G], rows[:, :, H * G:H * G + H], rows[:, :, H * G + H:], pos[:, a:b].contiguous(), *out, w, w, freq,
                         interleaved=interleaved)
        return out
    whole, step = call(0, T), T // 3 + 1
    for a in range(0, T, step):
        for got, want in zip(whole, call(a, min(T, a + step))):
            assert torch.equal(got[:, a:a + step], want)


@gpu
@pytest.mark.parametrize("dt,bits,n", [("bf16", 8, 33001), ("f16", 4, 33001), ("f32", 8, 16501), ("f32", 4, 16501), ("bf16", 4, 33001), ("f16", 8, 33001)])
def test_packed_rows_of_more_than_the_caches_hold(dt, bits, n):
    U, step, gen = 16, n // 3 + 1, torch.Generator(DEV).manual_seed(n)
    K, V = (torch.randn(U, n, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    assert 2 * K.numel() * K.element_size() > 256 << 20
    whole, parts = PackedCache.zeros(U, n, dt, bits, DEV), PackedCache.zeros(U, n, dt, bits, DEV)
    whole.dynakv_packed_write(K, V)
    for a in range(0, n, step):
        parts.dynakv_packed_write(K[:, a:a + step].contiguous(), V[:, a:a + step].contiguous(), torch.full((U,), a, dtype=torch.int32, device=DEV))
    for x, y in zip(whole.tensors, parts.tensors):
        assert torch.equal(x, y)
    k, v = torch.empty_like(K), torch.empty_like(V)
    whole.dynakv_packed_read(None, k, v)
    for a in range(0, n, step):
        at = torch.arange(a, min(n, a + step), dtype=torch.int32, device=DEV).expand(U, -1).contiguous()
        k1, v1 = (torch.empty(U, at.shape[1], D, dtype=K.dtype, device=DEV) for _ in range(2))
        whole.dynakv_packed_read(at, k1, v1)
        assert torch.equal(k[:, a:a + step], k1) and torch.equal(v[:, a:a + step], v1)


# ------------------------------------------------------------------------------------------- attention of drafted tokens
def _plain_tree(Q, K, V, K1, V1, seen, scale):
    """One unit in float64: Q [T, G, D], K, V [L, D], K1, V1 [T, D], seen bool [T, T].  Returns out, lse and the quantities that
    bound the error: sum p|v|, sum |v|, largest |q||k| of a logit."""
    T = Q.shape[0]
    K, V = torch.cat((K, K1)), torch.cat((V, V1))
    ok = torch.cat((torch.ones(T, K.shape[0] - K1.shape[0], dtype=torch.bool, device=Q.device), seen), 1)[:, None, :].expand(-1, Q.shape[1], -1)
    logits = (Q @ K.T * scale).masked_fill(~ok, -float("inf"))
    reach = torch.cat(((Q.abs() @ K.abs().T * scale).masked_fill(~ok, 0.0), Q.new_zeros(*Q.shape[:2], 1)), -1).amax(-1)
    lse = torch.logsumexp(logits, -1)
    p = (logits - lse.masked_fill(lse == -float("inf"), 0.0)[..., None]).exp().masked_fill(~ok, 0.0)
    Vz = V
    out, spread = p @ Vz, p @ Vz.abs()
    return out, lse, spread, ok.double() @ Vz.abs(), reach


def _check_tree(got, got_lse, ref, dt, L):
    out, lse, spread, total, reach = ref
    h = HALF[dt]
    # a logit: 128 products summed in float32 and three roundings of its scaling: delta; a weight: twice that (its own and the
    # denominator's), the sums over L entries and the hardware's exponential 2^-22; the weight's rounding h (16-bit types), in float16 at
    # least 2^-25 of the largest weight; the output's rounding h
    delta = 132 * U32 * reach[..., None]
    rel = 2 * delta + (L / 4 + 64) * U32 + 2.0 ** -21
    bound = spread * (rel + (h if dt != "f32" else 0)) * 1.01 + h * out.abs()
    if dt == "f16":
        bound = bound + 2.0 ** -25 * (total + 1)
    # the output before its rounding is off by the first part: its rounding too
    err = (got.double() - out).abs()
    # (1e-30: weights under 2^-126 of the largest are below float32's normal range and may vanish)
    assert bool((err <= bound + 1e-30).all()), ((err - bound).max().item(), (err / (bound + 1e-30)).max().item())
    if got_lse is not None:
        gone = lse == -float("inf")
        assert torch.equal(got_lse == -float("inf"), gone)
        lim = delta[..., 0] + (L / 4 + 64) * U32 + 2.0 ** -21 + 4 * U32 * lse.abs()
        assert bool(((got_lse.double() - lse).abs()[~gone] <= lim[~gone]).all())


def _random_tree(U, T, gen):
    seen = torch.rand(U, T, T, generator=gen, device=DEV) < 0.4
    seen = torch.tril(seen) | torch.eye(T, dtype=torch.bool, device=DEV)
    seen[:, T // 2] = False                                      # a node that sees no drafted token
    return seen


def _bits(seen):
    U, T, _ = seen.shape
    word = torch.zeros(U, T, dtype=torch.int64, device=DEV)
    for j in range(T):
        word |= seen[:, :, j].long() * (-(1 << 63) if j == 63 else 1 << j)
    return word


def _drafts(dt, U, T, G, gen, scale=1.0):
    t = TORCH_DTYPES[dt]
    r = lambda *s: (scale * torch.randn(*s, generator=gen, device=DEV)).to(t)  # noqa: E731
    return r(U, T, G, D), r(U, T, D), r(U, T, D), torch.full((U, T, G, D), 3.0, dtype=t, device=DEV), torch.full((U, T, G), 3.0, device=DEV)


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 8), ("f16", 4), ("bf16", 8), ("bf16", 4), ("f32", 8), ("f32", 4)])
@pytest.mark.parametrize("U,T,G,cap", [(1, 1, 1, 1), (3, 1, 8, 700), (2, 5, 4, 95), (5, 33, 3, 300), (2, 64, 16, 1500), (1, 64, 1, 64),
                                       (40, 7, 7, 129), (2, 17, 2, 4096), (300, 2, 1, 40),
                                       (600, 1, 2, 90), (100, 4, 4, 2000), (9, 3, 16, 9000), (130, 9, 4, 700)])
def test_packed_attention(dt, bits, U, T, G, cap):
    gen = torch.Generator(DEV).manual_seed(U + T + cap)
    K, V = (torch.randn(U, cap, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    c = PackedCache.zeros(U, cap, dt, bits, DEV)
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)                              # what the cache holds
    lengths = torch.randint(0, cap + 1, (U,), generator=gen, device=DEV, dtype=torch.int32)
    lengths[0] = cap
    if U > 2:
        lengths[1], lengths[2] = 0, -5
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    seen = _random_tree(U, T, gen)
    # the rows behind a unit's length may hold anything
    for u in range(U):
        c.tensors[1][u, max(0, int(lengths[u])):] = 255
        c.tensors[3][u, max(0, int(lengths[u])):] = 255
    c.dynakv_packed_attend(lengths, Q, K1, V1, _bits(seen), out, lse, tree_scratch(U, T, G, DEV))
    for u in range(U):
        n = max(0, int(lengths[u]))
        ref = _plain_tree(Q[u].double(), K[u, :n].double(), V[u, :n].double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, n + T)


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 8), ("f16", 4), ("bf16", 8), ("bf16", 4), ("f32", 8), ("f32", 4)])
@pytest.mark.parametrize("T,G", [(1, 3), (20, 4)])
def test_packed_attention_over_blocks_that_are_nan(dt, bits, T, G):
    # a value that is not finite makes its block NaN: of a key for all who see it, of a value in the block's 32 columns alone
    U, cap = 3, 200
    gen = torch.Generator(DEV).manual_seed(31)
    K, V = (torch.randn(U, cap, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    K[0, 77, 5], V[1, 120, 40] = float("inf"), float("nan")
    c = PackedCache.zeros(U, cap, dt, bits, DEV)
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    assert K[0, 77, :32].isnan().all() and V[1, 120, 32:64].isnan().all() and K.isnan().sum() == 32 and V.isnan().sum() == 32
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    seen = _random_tree(U, T, gen)
    c.dynakv_packed_attend(None, Q, K1, V1, _bits(seen), out, lse, tree_scratch(U, T, G, DEV))
    assert out[0].isnan().all() and lse[0].isnan().all()
    assert out[1, ..., 32:64].isnan().all()
    out[1, ..., 32:64], V[1, :, 32:64], V1[1, :, 32:64] = 0, 0, 0
    for u in (1, 2):
        ref = _plain_tree(Q[u].double(), K[u].double(), V[u].double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, cap + T)


@gpu
def test_packed_attention_of_a_unit_beyond_32_bits():
    cap = (1 << 25) + 77                                        # the second unit's codes begin 4.3 GB into theirs
    c = PackedCache.zeros(2, cap, "f16", 8, DEV)
    gen = torch.Generator(DEV).manual_seed(4)
    K, V = (torch.randn(2, 300, D, generator=gen, device=DEV).half() for _ in range(2))
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    lengths = torch.tensor([20, 300], dtype=torch.int32, device=DEV)
    Q, K1, V1, out, lse = _drafts("f16", 2, 3, 4, gen)
    c.dynakv_packed_attend(lengths, Q, K1, V1, None, out, lse, tree_scratch(2, 3, 4, DEV))
    chain = torch.ones(3, 3, dtype=torch.bool, device=DEV).tril()
    for u, n in enumerate((20, 300)):
        ref = _plain_tree(Q[u].double(), K[u, :n].double(), V[u, :n].double(), K1[u].double(), V1[u].double(), chain, D ** -0.5)
        _check_tree(out[u], lse[u], ref, "f16", n + 3)


def _retrieved(dt, U, G, n, M, budget, seed, **more):
    """An index over random entries after a retrieval, and per unit the positions it gathered."""
    gen = torch.Generator(DEV).manual_seed(seed)
    t = TORCH_DTYPES[dt]
    centre = torch.randn(U, M, D, generator=gen, device=DEV)
    pick = torch.randint(0, M, (U, n), generator=gen, device=DEV)
    K = (torch.gather(centre, 1, pick[:, :, None].expand(-1, -1, D)) + 0.3 * torch.randn(U, n, D, generator=gen, device=DEV)).to(t)
    V = torch.randn(U, n, D, generator=gen, device=DEV).to(t)
    ix = binding.Index(binding.Config(U, G, dt, M, 4 * M, n + 64, 3, **more), DEV)
    init = torch.rand(U, n, generator=gen, device=DEV).topk(M, 1).indices.int().contiguous()
    ix.dynakv_build_index(K, V, init)
    Q0 = torch.randn(U, G, D, generator=gen, device=DEV).to(t)
    out = torch.empty(U, G, D, device=DEV)
    ix.dynakv_retrieve_attend(Q0, budget, out, None)
    s = ix.dynakv_export_state(["n_gathered", "gathered"])
    at = [s["gathered"][u, :int(s["n_gathered"][u])].long().to(DEV) for u in range(U)]
    return ix, K, V, at, gen, Q0, out


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("U,T,G,n,M,budget", [(1, 1, 1, 40, 4, 1), (1, 5, 4, 2048, 32, 256), (3, 64, 7, 1500, 50, 1000), (17, 8, 4, 600, 30, 333),
                                              (2, 33, 16, 900, 20, 900), (4, 3, 2, 300, 300, 40), (2, 9, 3, 500, 25, 0), (130, 4, 8, 256, 16, 200)])
def test_tree_attention_over_a_retrieval(dt, U, T, G, n, M, budget):
    ix, K, V, at, gen, Q0, flat = _retrieved(dt, U, G, n, M, budget, T)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    seen = _random_tree(U, T, gen)
    scratch = tree_scratch(U, T, G, DEV)
    ix.dynakv_attend_tree(Q, K1, V1, _bits(seen), out, lse, scratch)
    for u in range(U):
        ref = _plain_tree(Q[u].double(), K[u, at[u]].double(), V[u, at[u]].double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, len(at[u]) + T)
    # twice: the same bits
    again, lse2 = torch.empty_like(out), torch.empty_like(lse)
    ix.dynakv_attend_tree(Q, K1, V1, _bits(seen), again, lse2, scratch)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    # the root's queries without drafted tokens: the retrieval's own attention
    root = torch.empty(U, 1, G, D, dtype=Q.dtype, device=DEV)
    ix.dynakv_attend_tree(Q0[:, None].contiguous(), None, None, None, root, None, tree_scratch(U, 1, G, DEV))
    none = torch.zeros(1, 0, dtype=torch.bool, device=DEV)
    for u in range(U):
        empty = torch.zeros(0, D, dtype=torch.float64, device=DEV)
        ref = _plain_tree(Q0[u:u + 1].double(), K[u, at[u]].double(), V[u, at[u]].double(), empty, empty, none, D ** -0.5)
        _check_tree(root[u], None, ref, dt, len(at[u]))


# Rows beyond those of one wavefront, on so few and so many units that workgroups of two, four and eight wavefronts of rows, whole and shared units
# and several blocks of rows occur.
@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("U,T,G,n,M,budget", [(120, 59, 5, 500, 20, 393), (2, 64, 16, 1600, 50, 1500), (70, 33, 5, 1000, 30, 900), (30, 25, 4, 3300, 60, 3000),
                                              (27, 11, 5, 1500, 40, 1266), (110, 10, 5, 700, 20, 600)])
def test_tree_attention_of_many_rows(dt, U, T, G, n, M, budget):
    ix, K, V, at, gen, Q0, flat = _retrieved(dt, U, G, n, M, budget, T)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    seen = _random_tree(U, T, gen)
    ix.dynakv_attend_tree(Q, K1, V1, _bits(seen), out, lse, tree_scratch(U, T, G, DEV))
    for u in range(U):
        ref = _plain_tree(Q[u].double(), K[u, at[u]].double(), V[u, at[u]].double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, len(at[u]) + T)


@gpu
@pytest.mark.parametrize("dt,bits", [("f16", 8), ("f16", 4), ("bf16", 8), ("bf16", 4), ("f32", 8)])
@pytest.mark.parametrize("U,T,G,cap", [(120, 59, 5, 393), (130, 30, 3, 1500), (20, 60, 5, 6000), (28, 59, 5, 1214), (65, 20, 3, 3000)])
def test_packed_attention_of_many_rows(dt, bits, U, T, G, cap):
    gen = torch.Generator(DEV).manual_seed(U + T + cap)
    K, V = (torch.randn(U, cap, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    c = PackedCache.zeros(U, cap, dt, bits, DEV)
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    lengths = torch.randint(0, cap + 1, (U,), generator=gen, device=DEV, dtype=torch.int32)
    lengths[0], lengths[1] = cap, 0
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    seen = _random_tree(U, T, gen)
    c.dynakv_packed_attend(lengths, Q, K1, V1, _bits(seen), out, lse, tree_scratch(U, T, G, DEV))
    for u in range(U):
        n = int(lengths[u])
        ref = _plain_tree(Q[u].double(), K[u, :n].double(), V[u, :n].double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, n + T)


@gpu
@pytest.mark.parametrize("more", [dict(update_mode=binding.UPDATE_TOKENS), dict(launch=binding.launch_shape(3, 4, binding.LAUNCH_SEPARATE)),
                                  dict(search_copy=binding.SEARCH_MEAN), dict(softmax_scale=0.37)])
def test_tree_attention_after_every_kind_of_retrieval(more):
    U, T, G, n = 3, 6, 4, 256
    M = n if "update_mode" in more else 24
    ix, K, V, at, gen, Q0, _ = _retrieved("bf16", U, G, n, M, 100, 9, **more)
    for kind in ("plain", "static"):
        if kind == "static":
            assert ix.dynakv_retrieve_attend_static(Q0, 100, torch.empty(U, G, D, device=DEV), None) == binding.OK
        Q, K1, V1, out, lse = _drafts("bf16", U, T, G, gen)
        seen = _random_tree(U, T, gen)
        ix.dynakv_attend_tree(Q, K1, V1, _bits(seen), out, lse, tree_scratch(U, T, G, DEV))
        for u in range(U):
            ref = _plain_tree(Q[u].double(), K[u, at[u]].double(), V[u, at[u]].double(), K1[u].double(), V1[u].double(), seen[u],
                              more.get("softmax_scale", D ** -0.5))
            _check_tree(out[u], lse[u], ref, "bf16", len(at[u]) + T)


@gpu
def test_tree_attention_needs_the_retrieval_it_follows():
    ix, K, V, at, gen, Q0, flat = _retrieved("f16", 2, 4, 300, 20, 100, 4)
    Q, K1, V1, out, lse = _drafts("f16", 2, 3, 4, gen)
    scratch = tree_scratch(2, 3, 4, DEV)
    k1, v1 = K1[:, 0].contiguous(), V1[:, 0].contiguous()

    def attend():
        ix.dynakv_attend_tree(Q, K1, V1, None, out, lse, scratch)
    attend()
    snapshot = None
    for change in (lambda: ix.dynakv_append(k1, v1), lambda: ix.dynakv_split(), lambda: ix.dynakv_extend_index(K1, V1),
                   lambda: ix.dynakv_decode_step(Q0, 100, flat, None, k1, v1), lambda: ix.dynakv_import_state(snapshot),
                   lambda: ix.dynakv_build_index(K, V, torch.stack([torch.randperm(300)[:20] for _ in range(2)]).int().to(DEV))):
        ix.dynakv_retrieve_attend(Q0, 100, flat, None)
        attend()                                                 # right after a retrieval
        attend()                                                 # it changes nothing itself
        snapshot = ix.dynakv_export_state(binding.IMPORT_FIELDS, to_cpu=False)
        attend()                                                 # nor does a snapshot
        change()
        out.fill_(3.0)
        with pytest.raises(RuntimeError, match="out of order"):
            attend()
        assert (out == 3.0).all()


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,cap", [(1, 0), (40, 0), (40, 50), (64, 333)])
def test_what_a_node_does_not_see_has_no_part(dt, T, cap):
    U, G = 3, 5
    gen = torch.Generator(DEV).manual_seed(T + cap)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    c = PackedCache.zeros(U, max(cap, 1), dt, 8, DEV)
    K, V = (torch.randn(U, max(cap, 1), D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    lengths = torch.full((U,), cap, dtype=torch.int32, device=DEV)
    seen = _random_tree(U, T, gen)
    bad = [j for j in (0, T // 2, T - 1)]
    seen[1, :, bad] = False                                      # unit 1: nobody sees them; unit 2: only some do
    if T > 1:
        seen[2, :, bad[-1]] = False
        seen[2, T // 3, bad[-1]] = True
    K1[1, bad], V1[1, bad, ::7] = float("nan"), float("inf")
    V1[1, bad, 1] = float("nan")
    K1[1, bad[0]] = float("inf")
    V1[2, bad[-1], 4] = -float("inf")
    V1[2, bad[-1], 127] = float("nan")
    V1[2, bad[-1], 64] = float("inf")
    seen[0] = False                                              # unit 0: no node sees a drafted token
    words = _bits(seen)
    if T < 64:
        words |= 1 << T                                          # bits of tokens that are not there
        words |= -(1 << 63)
    c.dynakv_packed_attend(lengths, Q, K1, V1, words, out, lse, tree_scratch(U, T, G, DEV))
    for u in range(U):
        k1 = torch.where(seen[u].any(0)[:, None], K1[u], torch.zeros_like(K1[u])).double()
        v1 = torch.where(seen[u].any(0)[:, None], V1[u], torch.zeros_like(V1[u])).double()
        ref = list(_plain_tree(Q[u].double(), K[u, :cap].double(), V[u, :cap].double(), k1, v1.nan_to_num(0, 0, 0), seen[u], D ** -0.5))
        got = out[u].clone()
        if u == 2 and T > 1:
            # the rows that see the token have its infinities and NaN, the others are clean
            sees = seen[2, :, bad[-1]]
            assert (got[sees][..., 4] == -float("inf")).all() and (got[sees][..., 64] == float("inf")).all() and got[sees][..., 127].isnan().all()
            for col in (4, 64, 127):
                got[sees, :, col] = 0
                ref[0][sees, :, col] = 0
        _check_tree(got, lse[u], ref, dt, cap + T)
    if cap == 0:
        assert (out[0] == 0).all() and (lse[0] == -float("inf")).all()


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_attention_of_large_and_equal_logits(dt):
    # logits of 10^3 and more, all logits equal, one that dwarfs the others and comes last: the running maximum moves
    U, T, G, cap = 4, 3, 4, 500
    gen = torch.Generator(DEV).manual_seed(8)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    K, V = (torch.randn(U, cap, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    K[0] *= 40
    K[1] = 1.0
    K1[1] = 1.0
    K[2] = K[2] * torch.linspace(0, 6, cap, device=DEV)[:, None].to(K.dtype) + Q[2, 0, 0] * torch.linspace(0, 2, cap, device=DEV)[:, None].to(K.dtype)
    K[3], K1[3] = -K[2], Q[3, :, 0] * 8
    c = PackedCache.zeros(U, cap, dt, 8, DEV)
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    c.dynakv_packed_attend(None, Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV))
    chain = torch.ones(T, T, dtype=torch.bool, device=DEV).tril()
    for u in range(U):
        ref = _plain_tree(Q[u].double(), K[u].double(), V[u].double(), K1[u].double(), V1[u].double(), chain, D ** -0.5)
        _check_tree(out[u], lse[u], ref, dt, cap + T)


@gpu
@pytest.mark.parametrize("dt,tiny", [("f16", 2.0 ** -20), ("bf16", 2.0 ** -120), ("f32", 2.0 ** -120)])
def test_attention_keeps_small_values(dt, tiny):
    # float16 values below its normal range, and small ones of the others, as keys and values of entries and drafts
    U, T, G, cap = 2, 3, 4, 90
    gen = torch.Generator(DEV).manual_seed(14)
    Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
    K, V = (torch.randn(U, cap, D, generator=gen, device=DEV).to(TORCH_DTYPES[dt]) for _ in range(2))
    V, V1, K1 = (V.float() * tiny).to(V.dtype), (V1.float() * tiny).to(V.dtype), (K1.float() * tiny).to(V.dtype)
    c = PackedCache.zeros(U, cap, dt, 8, DEV)
    c.dynakv_packed_write(K, V)
    c.dynakv_packed_read(None, K, V)
    c.dynakv_packed_attend(None, Q, K1, V1, None, out, None, tree_scratch(U, T, G, DEV))
    chain = torch.ones(T, T, dtype=torch.bool, device=DEV).tril()
    for u in range(U):
        ref = _plain_tree(Q[u].double(), K[u].double(), V[u].double(), K1[u].double(), V1[u].double(), chain, D ** -0.5)
        # relative to the weighted sum of |v|: weights to 2 h (their rounding and that of products below the type's normal range), and half a
        # step of the smallest values there are for the output
        floor = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -149}[dt]
        err = (out[u].double() - ref[0]).abs()
        lim = ref[2] * (2 * HALF[dt] + 264 * U32 * ref[4][..., None] + 2.0 ** -20) + HALF[dt] * ref[0].abs() + floor
        assert bool((err <= lim).all()), (err - lim).max().item()
        assert out[u].any()


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_many_small_weights_beside_a_large_one(dt):
    # a sink whose weight is e^16 times that of each of 100 000 others: together they are worth a hundredth of it
    n, G = 100001, 2
    c = PackedCache.zeros(1, n, dt, 8, DEV)
    K, V = (torch.zeros(1, n, D, dtype=TORCH_DTYPES[dt], device=DEV) for _ in range(2))
    K[0, 777, 0] = 16.0
    V[0, :, 1] = 1.0
    V[0, 777, 1] = 0.0
    c.dynakv_packed_write(K, V)
    Q = torch.zeros(1, 1, G, D, dtype=K.dtype, device=DEV)
    Q[..., 0] = 1.0
    out, lse = torch.empty_like(Q), torch.empty(1, 1, G, device=DEV)
    c.dynakv_packed_attend(None, Q, None, None, None, out, lse, tree_scratch(1, 1, G, DEV), softmax_scale=1.0)
    small = (n - 1) * float(np.exp(-16.0))
    # each small weight, e^-16 = 0.97 * 2^-23 of the largest, is off by at most half a step: relative h, in float16, whose steps are 2^-31 of the
    # largest there, 2^-9; the output's rounding h
    off = {"f16": 2.0 ** -9 + 2.0 ** -11, "bf16": 2.0 ** -7, "f32": 2.0 ** -18}[dt]
    assert abs(out[0, 0, 0, 1].item() / (small / (1 + small)) - 1) <= off
    assert abs(lse[0, 0, 0].item() - (16 + np.log1p(small))) <= 1e-5


@gpu
def test_attention_refusals_of_the_binding():
    c = PackedCache.zeros(2, 64, "f16", 8, DEV)
    gen = torch.Generator(DEV).manual_seed(1)
    Q, K1, V1, out, lse = _drafts("f16", 2, 3, 4, gen)
    tree, scratch = torch.ones(2, 3, dtype=torch.int64, device=DEV), tree_scratch(2, 3, 4, DEV)
    bad = [(Q.float(), K1, V1, tree, out, lse, scratch), (Q, K1, None, tree, out, lse, scratch), (Q, K1[:, :2], V1, tree, out, lse, scratch),
           (Q, K1, V1, tree.int(), out, lse, scratch), (Q, K1, V1, tree[:1], out, lse, scratch), (Q, K1, V1, tree, out.float(), lse, scratch),
           (Q, K1, V1, tree, out, lse[:, :, :2], scratch), (Q, K1, V1, tree, out, lse, scratch.float()), (Q.transpose(1, 2), K1, V1, tree, out, lse, scratch),
           (Q[0], K1, V1, tree, out, lse, scratch)]
    for args in bad:
        with pytest.raises(ValueError):
            c.dynakv_packed_attend(None, *args)
    with pytest.raises(RuntimeError, match="scratch"):
        c.dynakv_packed_attend(None, Q, K1, V1, tree, out, lse, scratch[:16])
    with pytest.raises(ValueError):
        c.dynakv_packed_attend(torch.zeros(2, dtype=torch.int64, device=DEV), Q, K1, V1, tree, out, lse, scratch)
    with pytest.raises(ValueError):
        tree_scratch(1, 65, 1, DEV)
    with pytest.raises(ValueError):
        c.dynakv_packed_write(K1, V1.float())
    c.dynakv_packed_write(K1[:, :0], V1[:, :0])                              # nothing to do
    c.dynakv_packed_read(None, K1[:, :0], V1[:, :0])
    with pytest.raises(ValueError):
        c.dynakv_packed_read(torch.zeros(2, 2, dtype=torch.int32, device=DEV), K1, V1)
    assert (out == 3.0).all() and (lse == 3.0).all()


# ----------------------------------------------------------------------------------------------------- used together
def _layer(dt, B, H, G, prompt, T, M, seed):
    """One layer of B sequences: fused projections of a prompt and of T drafted tokens, what dynakv_norm_rope makes of them."""
    gen = torch.Generator(DEV).manual_seed(seed)
    freq = (500000.0 ** (-torch.arange(0, 128, 2, device=DEV).double() / 128)).float()
    w = (1 + 0.1 * torch.randn(2, D, generator=gen, device=DEV)).to(TORCH_DTYPES[dt])
    made = []
    for n, first in ((prompt, 0), (T, prompt)):
        q, k, v = _fused_rows(dt, B, n, H, G, gen)
        pos = (first + torch.arange(n, device=DEV, dtype=torch.int32)).expand(B, n).contiguous()
        rows = _outputs(dt, B, n, H, G)
        made.append((q, k, v, pos, rows))
    init = torch.rand(B * H, prompt, generator=gen, device=DEV).topk(M, 1).indices.int().contiguous()
    return gen, freq, w, made, init


@gpu
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_a_drafted_step_from_projections_to_attention(dt):
    # prompt and drafts -> norm + rotation -> index and packed cache -> retrieval at the root -> the tree over what it gathered and,
    # for a layer that is kept dense, over the packed cache; the accepted path goes into both; a session parked in the packed cache
    # comes back as an index
    B, H, G, n, T, M, budget = 2, 2, 4, 512, 7, 32, 200
    U = B * H
    gen, freq, w, made, init = _layer(dt, B, H, G, n, T, M, 11)
    for q, k, v, pos, rows in made:
        dynakv_norm_rope(q, k, v, pos, *rows, q_weight=w[0], k_weight=w[1], inv_freq=freq)
    (_, K, V), (Q, K1, V1) = made[0][4], made[1][4]
    ix = binding.Index(binding.Config(U, G, dt, M, 4 * M, n + 64, 3, var_alpha=1.5), DEV)
    ix.dynakv_build_index(K, V, init)
    cache = PackedCache.zeros(U, n + 64, dt, 8, DEV)
    cache.dynakv_packed_write(K, V)
    lengths = torch.full((U,), n, dtype=torch.int32, device=DEV)
    flat = torch.empty(U, G, D, device=DEV)
    ix.dynakv_retrieve_attend(Q[:, 0].contiguous(), budget, flat, None)
    s = ix.dynakv_export_state(["n_gathered", "gathered"])
    seen = _random_tree(U, T, gen)
    outs = [torch.empty_like(Q) for _ in range(2)]
    lses = [torch.empty(U, T, G, device=DEV) for _ in range(2)]
    scratch = tree_scratch(U, T, G, DEV)
    ix.dynakv_attend_tree(Q, K1, V1, _bits(seen), outs[0], lses[0], scratch)
    cache.dynakv_packed_attend(lengths, Q, K1, V1, _bits(seen), outs[1], lses[1], scratch)
    pk, pv = torch.empty_like(K), torch.empty_like(V)
    cache.dynakv_packed_read(None, pk, pv)
    for u in range(U):
        at = s["gathered"][u, :int(s["n_gathered"][u])].long().to(DEV)
        for o, l, k, v in ((outs[0], lses[0], K[u, at], V[u, at]), (outs[1], lses[1], pk[u], pv[u])):
            ref = _plain_tree(Q[u].double(), k.double(), v.double(), K1[u].double(), V1[u].double(), seen[u], D ** -0.5)
            _check_tree(o[u], l[u], ref, dt, k.shape[0] + T)
    # nodes 0..2 are accepted
    for j in range(3):
        ix.dynakv_append(K1[:, j].contiguous(), V1[:, j].contiguous())
        ix.dynakv_split()
    cache.dynakv_packed_write(K1, V1, lengths, torch.full_like(lengths, 3))
    lengths += 3
    st = ix.dynakv_export_state(binding.IMPORT_FIELDS, to_cpu=False)
    assert (st["n_tokens"] == n + 3).all()
    # parked: the snapshot's keys and values come from the packed cache
    pos = torch.arange(n + 64, device=DEV, dtype=torch.int32).expand(U, -1).clone()
    pos[:, n + 3:] = -1
    cache.dynakv_packed_read(pos, st["keys"], st["values"])
    back = binding.Index(ix.cfg, DEV)
    back.dynakv_import_state(st)
    back.dynakv_retrieve_attend(Q[:, 2].contiguous(), budget, flat, None)
    again = back.dynakv_export_state(["n_gathered", "gathered", "keys", "values"], to_cpu=False)
    back.dynakv_attend_tree(Q, None, None, None, outs[0], lses[0], scratch)
    empty, none = torch.zeros(0, D, dtype=torch.float64, device=DEV), torch.zeros(T, 0, dtype=torch.bool, device=DEV)
    for u in range(U):
        at = again["gathered"][u, :int(again["n_gathered"][u])].long()
        assert torch.equal(again["keys"][u, :n], pk[u])
        ref = _plain_tree(Q[u].double(), again["keys"][u, at].double(), again["values"][u, at].double(), empty, empty, none, D ** -0.5)
        _check_tree(outs[0][u], lses[0][u], ref, dt, len(at))


@gpu
def test_captured_and_replayed_on_a_stream_of_their_own():
    # one decode step of drafts in a graph: norm + rotation, packed write and read, retrieval, both attentions; replayed with new
    # inputs in the same tensors, with eager work between the replays, and compared with eager calls each time
    dt, B, H, G, n, T, M, budget = "bf16", 2, 3, 4, 700, 9, 40, 300
    U = B * H
    gen, freq, w, made, init = _layer(dt, B, H, G, n, T, M, 12)
    q, k, v, pos, rows = made[0]
    dynakv_norm_rope(q, k, v, pos, *rows, q_weight=w[0], k_weight=w[1], inv_freq=freq)
    _, K, V = rows
    ix = binding.Index(binding.Config(U, G, dt, M, 4 * M, n + 64, 3), DEV)
    ix.dynakv_build_index(K, V, init)
    cache = PackedCache.zeros(U, n + T, dt, 4, DEV)
    cache.dynakv_packed_write(K, V)
    start = torch.full((U,), n, dtype=torch.int32, device=DEV)
    where = (start[:, None] + torch.arange(T, device=DEV, dtype=torch.int32)).contiguous()
    q, k, v, pos, (Q, K1, V1) = made[1]
    tree, scratch = _bits(_random_tree(U, T, gen)), [tree_scratch(U, T, G, DEV) for _ in range(2)]
    flat = torch.empty(U, G, D, device=DEV)
    res = [torch.empty_like(Q), torch.empty(U, T, G, device=DEV), torch.empty_like(Q), torch.empty(U, T, G, device=DEV), torch.empty_like(K1),
           torch.empty_like(V1)]
    root = torch.empty(U, G, D, dtype=Q.dtype, device=DEV)

    def step():
        dynakv_norm_rope(q, k, v, pos, Q, K1, V1, q_weight=w[0], k_weight=w[1], inv_freq=freq)
        root.copy_(Q[:, 0])
        ix.dynakv_retrieve_attend(root, budget, flat, None)
        ix.dynakv_attend_tree(Q, K1, V1, tree, res[0], res[1], scratch[0])
        cache.dynakv_packed_write(K1, V1, start)
        cache.dynakv_packed_read(where, res[4], res[5])
        cache.dynakv_packed_attend(start, Q, K1, V1, tree, res[2], res[3], scratch[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(4):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        for r in res:
            r.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [r.clone() for r in res] + [Q.clone(), flat.clone()]
        for r in res:
            r.fill_(9.0)
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, res + [Q, flat]):
            assert torch.equal(a, b), i


@gpu
def test_two_streams_with_scratch_of_their_own():
    dt, U, T, G, cap = "f16", 2, 5, 4, 6000
    gen = torch.Generator(DEV).manual_seed(4)
    c = PackedCache.zeros(U, cap, dt, 8, DEV)
    K, V = (torch.randn(U, cap, D, generator=gen, device=DEV).half() for _ in range(2))
    c.dynakv_packed_write(K, V)
    jobs = []
    for i in range(2):
        Q, K1, V1, out, lse = _drafts(dt, U, T, G, gen)
        jobs.append((Q, K1, V1, None, out, lse, tree_scratch(U, T, G, DEV)))
    want = []
    for j in jobs:
        c.dynakv_packed_attend(None, *j)
        want.append((j[4].clone(), j[5].clone()))
        j[4].fill_(0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        for st, j in zip(streams, jobs):
            with torch.cuda.stream(st):
                c.dynakv_packed_attend(None, *j)
    torch.cuda.synchronize()
    for j, (o, l) in zip(jobs, want):
        assert torch.equal(j[4], o) and torch.equal(j[5], l)
