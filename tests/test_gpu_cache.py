"""s2o_decode, s2o_key_weights and s2o_evict on the GPU against their definitions in 64 bits (tests/cache_util.py).

Tolerances.  h: half a step of the element type (bf16 2^-8, f16 2^-11).  X: scale * max |q| max |k|, which bounds sum |q_d k_d| * scale.
A score made by the matrix instructions is off by at most 1e-6 X (the bound that the prefill's scores are held to), so a weight
exp(x - lse) by 2e-6 X of itself, and by 2e-6 more for the rounding of the exponent's argument and of exp2.
  lse      1e-6 X + 1e-6 (1 + |lse|): the scores, and two roundings of 2^-24 each in a sum, a logarithm and a product of it
  O        with A = sum_j p_j |v_j| / sum_j p_j: p rounded to the element type h A, the result h |O|, the weights 4e-6 X A,
           f16 numerators below 2^-14 2^-25 each of at most max |v|
  weights  (2e-6 X + 4e-6 + R 2^-25) w: R rows summed in fp32, a quarter of them a lane, each addition 2^-24 at most (R/4 + 4 of them)
Rows moved and indices are exact."""
import math

import numpy as np
import pytest
import torch

import cache_util as u
import paper_2602_22575_amd as s2o

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _needs(gpu):
    pass


def _i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda:0")


def _f(t):
    return None if t is None else u.f64(t)


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _x(scale, q, *keys):
    k = max([np.linalg.norm(x, axis=-1).max() for x in keys if x is not None and x.size], default=0.0)
    return scale * np.linalg.norm(q, axis=-1).max() * k


def check_decode(got, Q, K, V, own_K, own_V, lens, own_lens, dt, scale=None):
    O, lse = (_f(t) for t in got)
    D, h = Q.shape[-1], u.HALF_STEP[dt]
    scale = scale or 1 / math.sqrt(D)
    q, k, v, ok, ov = (_f(t) for t in (Q, K, V, own_K, own_V))
    ref, ref_lse, A = u.decode(q, k, v, ok, ov, lens, own_lens, scale)
    X = _x(scale, q, k, ok)
    n = (k.shape[2] if k is not None else 0) + (ok.shape[3] if ok is not None else 0)
    top = max(np.abs(t).max() for t in (v, ov) if t is not None)
    tol = h * (A + np.abs(ref)) + 4e-6 * X * A + (n * 2.0 ** -25 * top if dt == "f16" else 0.0)
    assert np.all(np.abs(O - ref) <= tol), np.max(np.abs(O - ref) / (tol + 1e-30))
    empty = np.isinf(ref_lse)
    assert np.array_equal(empty, np.isneginf(lse)) and np.all(O[empty] == 0)
    d = np.abs(np.where(empty, 0, lse) - np.where(empty, 0, ref_lse))
    assert np.all(d <= 1e-6 * X + 1e-6 * (1 + np.abs(np.where(empty, 0, ref_lse)))), d.max()


def make_decode(Z, B, H, Hkv, D, T, L, own, dt, token=False, seed=0, gain=2.0):
    g = _gen(seed)
    Q = u.randn(g, Z, B, H, T, D, dtype=dt, token=token, gain=gain)
    K, V = (u.randn(g, Z, Hkv, L, D, dtype=dt, token=token) if L else None for _ in range(2))
    oK, oV = (u.randn(g, Z, B, Hkv, own, D, dtype=dt, token=token) if own else None for _ in range(2))
    st = {}
    if token:
        st = {k + "_stride": u.strides(t) for k, t in (("q", Q), ("o", Q), ("k", K), ("v", V), ("own_k", oK), ("own_v", oV)) if t is not None}
    return (Q, K, V, oK, oV), s2o.make_decode_params(Z, B, H, Hkv, D, T, L, own, dtype=dt, **st)


def run_decode(t, p, lens=None, own_lens=None, **kw):
    Q, K, V, oK, oV = t
    got = s2o.s2o_decode(Q, K, V, p, own_K=oK, own_V=oV, lens=_i32(lens), own_lens=_i32(own_lens), **kw)
    torch.cuda.synchronize()
    return got


DECODE = [
    # Z B H Hkv D T L own dtype token lens own_lens
    (1, 1, 1, 1, 128, 1, 1, 0, "bf16", False, None, None),                    # one key
    (1, 2, 8, 2, 128, 1, 96, 24, "bf16", False, None, None),
    (1, 1, 4, 4, 64, 1, 0, 1, "f16", False, None, None),
    (2, 3, 6, 2, 64, 1, 33, 31, "f16", True, None, None),
    (1, 5, 7, 1, 128, 3, 500, 12, "bf16", False, None, [[12, 3, 2, 1, 0]]),   # T above the length
    (2, 3, 8, 2, 128, 3, 1500, 70, "bf16", True, [1500, 700], [[70, 2, 0], [5, 33, 1]]),
    (2, 2, 8, 1, 64, 5, 2000, 600, "f16", False, [0, 1999], [[0, 600], [3, 64]]),   # a sequence that sees nothing at all
    (1, 33, 8, 2, 128, 1, 1111, 40, "bf16", False, [1100], None),             # 132 rows on a KV head
    (1, 9, 16, 2, 64, 9, 3001, 0, "bf16", False, None, None),                 # 648
    (3, 1, 2, 2, 128, 1, 4097, 0, "f16", True, [4097, 1, 32], None),
    (1, 1, 4, 2, 128, 1, 0, 3333, "bf16", False, None, [[3300]]),
    (1, 4, 4, 2, 64, 40, 700, 900, "f16", False, None, [[900, 40, 39, 41]]),
    (1, 17, 40, 8, 128, 1, 600, 5, "f16", False, [0], None),
    (5, 7, 2, 1, 64, 2, 513, 3, "bf16", True, [513, 0, 1, 64, 65], None),
    (1, 64, 32, 8, 128, 1, 2500, 30, "bf16", False, None, None),
    (1, 5, 8, 2, 128, 1, 3000, 40, "bf16", False, None, None),                # 20 rows on a KV head
    (2, 2, 16, 4, 64, 3, 2000, 33, "f16", True, [2000, 31], [[33, 2], [0, 33]]),   # 24
    (1, 8, 4, 1, 64, 1, 1200, 0, "bf16", False, [1187], None),                # 32
    (1, 5, 8, 2, 128, 5, 700, 90, "bf16", False, None, [[90, 4, 5, 6, 0]]),   # 20 rows a sequence
    (2, 3, 10, 2, 64, 7, 900, 300, "f16", True, [900, 17], [[300, 7, 2], [31, 32, 33]]),   # 35
    (1, 4, 8, 2, 128, 12, 2000, 700, "bf16", False, None, [[700, 13, 64, 1]]),   # 48
    (1, 4, 5, 1, 128, 7, 0, 260, "bf16", False, None, [[260, 3, 0, 100]]),
    (1, 4, 8, 2, 64, 8, 40, 30, "f16", False, [39], [[30, 8, 1, 0]]),         # 32, nothing joined
    (2, 70, 8, 4, 64, 1, 90, 11, "bf16", False, [90, 33], [list(range(12)) * 5 + [11] * 10] * 2),   # few keys of many sequences
    (1, 140, 4, 4, 128, 2, 300, 0, "f16", True, [299], None),
]


@pytest.mark.parametrize("c", DECODE, ids=lambda c: "-".join(map(str, c[:9])))
def test_decode(c):
    Z, B, H, Hkv, D, T, L, own, dt, token, lens, own_lens = c
    t, p = make_decode(Z, B, H, Hkv, D, T, L, own, dt, token, seed=L + own)
    got = run_decode(t, p, lens, own_lens)
    check_decode(got, *t, lens or [L] * Z, own_lens or [[own] * B] * Z, dt)


def test_decode_scale_and_no_lse():
    t, p = make_decode(1, 2, 4, 2, 128, 1, 700, 20, "bf16")
    p.softmax_scale = 0.25
    O, lse = run_decode(t, p, want_lse=False)
    assert lse is None
    check_decode((O, run_decode(t, p)[1]), *t, [700], [[20, 20]], "bf16", scale=0.25)


def test_decode_large_logits():
    """Rows whose maximum lies far beyond the lazily moving reference, rising along the cache."""
    t, p = make_decode(1, 3, 8, 2, 128, 1, 4000, 50, "bf16", gain=1.0)
    K = t[1]
    K.mul_(torch.linspace(0.1, 6, 4000, device="cuda:0").view(1, 1, -1, 1))
    check_decode(run_decode(t, p), *t, [4000], [[50] * 3], "bf16")


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("L,own", [(300, 70), (1500, 700)])
def test_decode_bad_values_where_nobody_looks(dt, L, own):
    """NaN and infinities behind the lengths, and in own rows that only later query tokens see: those are as the formula says."""
    Z, B, H, Hkv, D, T = 2, 2, 4, 2, 64, 4
    t, p = make_decode(Z, B, H, Hkv, D, T, L, own, dt)
    lens, own_lens = [L - 37, 5], [[own - 1, 3], [own, 20]]
    clean = run_decode(t, p, lens, own_lens)
    Q, K, V, oK, oV = t
    for z in range(Z):
        for x, bad in ((K, math.nan), (V, math.inf)):
            x[z, :, lens[z]:] = bad
        for b in range(B):
            oK[z, b, :, own_lens[z][b]:] = math.inf
            oV[z, b, :, own_lens[z][b]:] = math.nan
    got = run_decode(t, p, lens, own_lens)
    for x, y in zip(clean, got):
        assert torch.equal(x, y)
    # the last token's own row: only the last query token may be touched by it
    oV[0, 0, 0, own_lens[0][0] - 1, 3] = math.inf
    O, lse = run_decode(t, p, lens, own_lens)
    h = H // Hkv
    assert torch.isposinf(O[0, 0, :h, T - 1, 3]).all() and torch.equal(lse, clean[1])
    O2 = O.clone()
    O2[0, 0, :h, T - 1] = clean[0][0, 0, :h, T - 1]
    scale = clean[0].float().abs().max().item()
    assert torch.isfinite(O2).all() and (O2.float() - clean[0].float()).abs().max().item() <= 4 * u.HALF_STEP[dt] * scale
    # a NaN key that the last token sees
    oK[1, 1, 1, own_lens[1][1] - 1, 0] = math.nan
    O, lse = run_decode(t, p, lens, own_lens)
    assert torch.isnan(O[1, 1, h:, T - 1]).all() and torch.isnan(lse[1, 1, h:, T - 1]).all()
    assert torch.isfinite(O[1, 1, h:, :T - 1]).all() and torch.equal(lse[1, 1, h:, :T - 1], clean[1][1, 1, h:, :T - 1])


# Scores are set by the first element of the keys, in steps of the exponent: with Q's first element 8 and a scale of 1/8 a key's score is
# its own first element.
def _scored(x, Z, B, H, Hkv, D, dt, seed, gain=0.0):
    """Q, K, V with scores x [L] (rounded to the type) and a little more (gain)."""
    g = _gen(seed)
    L = len(x)
    Q = u.randn(g, Z, B, H, 1, D, dtype=dt, gain=gain)
    K, V = u.randn(g, Z, Hkv, L, D, dtype=dt, gain=gain), u.randn(g, Z, Hkv, L, D, dtype=dt)
    Q[..., 0] = 8.0
    K[..., 0] = torch.as_tensor(x, device="cuda:0").to(u.DTYPES[dt])
    return Q, K, V


def _steps(kind, L):
    x = np.zeros(L)
    i = np.arange(L)
    if kind == "one far above":                  # in the middle of a tile of 64 keys, more than any numerator's room above the others
        x[L // 2 + 5] = 100.0
    elif kind == "rising":                       # references move in nearly every tile
        x = i * (90.0 / L)
    elif kind == "falling":
        x = -i * (90.0 / L)
    elif kind == "first unseen":                 # the first keys' scores are -infinity: no reference there
        x[:70] = -np.inf
    elif kind == "every other unseen":
        x[::2] = -np.inf
    elif kind == "few jumps":
        x[i % 97 == 50] = 14.0
        x[i % 389 == 100] = 30.0
    return x


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("D,B", [(64, 40), (128, 40), (128, 3)])                     # 160 rows on a KV head, and 12
@pytest.mark.parametrize("kind", ["one far above", "rising", "falling", "first unseen", "every other unseen", "few jumps"])
def test_decode_scores_far_apart(kind, D, B, dt):
    L = 1500
    Q, K, V = _scored(_steps(kind, L), 1, B, 8, 2, D, dt, seed=31, gain=0.25)
    p = s2o.make_decode_params(1, B, 8, 2, D, 1, L, dtype=dt, softmax_scale=0.125)
    Q = Q.abs()                                                                      # (no -1 * -inf)
    got = run_decode((Q, K, V, None, None), p)
    O, lse = (_f(t) for t in got)
    q, k, v = _f(Q), _f(K), _f(V)
    ref, ref_lse, A = u.decode(q, k, v, None, None, [L], None, 0.125)
    X = _x(0.125, q, np.where(np.isinf(k), 0, k))
    tol = u.HALF_STEP[dt] * (A + np.abs(ref)) + 4e-6 * X * A + (L * 2.0 ** -25 * np.abs(v).max() if dt == "f16" else 0.0)
    assert np.all(np.abs(O - ref) <= tol), np.max(np.abs(O - ref) / tol)
    assert np.all(np.abs(lse - ref_lse) <= 1e-6 * X + 1e-6 * (1 + np.abs(ref_lse)))


def test_decode_huge_values_under_far_apart_scores():
    """Values of 1e30 and a score 2^50 above the others in the middle: no accumulator overflows."""
    L = 1000
    x = np.zeros(L)
    x[333] = 35.0
    Q, K, V = _scored(x, 1, 40, 8, 2, 128, "bf16", seed=4)
    V.mul_(1e30)
    p = s2o.make_decode_params(1, 40, 8, 2, 128, 1, L, softmax_scale=0.125)
    check_decode(run_decode((Q, K, V, None, None), p), Q, K, V, None, None, [L], None, "bf16", scale=0.125)


@pytest.mark.parametrize("rows", [1, 12, 30, 70])                                    # 16, 32 and 64 rows a wavefront
@pytest.mark.parametrize("kind", ["one far above", "rising", "falling", "first unseen", "every other unseen"])
def test_weights_scores_far_apart(kind, rows):
    L = 3000
    Q, K, _ = _scored(_steps(kind, L) * (1.0 if kind != "rising" else 1.2), 1, rows, 8, 2, 128, "bf16", seed=6, gain=0.25)
    Q = Q.abs()
    p = s2o.make_weights_params(1, rows, 8, 2, 128, 1, L, softmax_scale=0.125)
    w = _f(s2o.s2o_key_weights(Q, K, p))
    with np.errstate(invalid="ignore"):
        ref = u.key_weights(_f(Q), _f(K), [L], 0, 0.125)
    k = _f(K)
    tol = (2e-6 * _x(0.125, _f(Q), np.where(np.isinf(k), 0, k)) + 4e-6 + rows * 4 * 2.0 ** -25) * np.abs(ref)
    tol += rows * 4 * 2.0 ** -126                          # exp2 gives 0 in place of a number below 2^-126: of each row's term at most that is lost
    assert np.all(np.abs(w - ref) <= tol), np.max(np.abs(w - ref) / tol)


def test_lengths_beyond_the_memory_are_clamped():
    t, p = make_decode(2, 2, 4, 2, 64, 1, 600, 40, "bf16")
    got = run_decode(t, p, [10 ** 9, -5], [[41, -1], [2 ** 31 - 1, 0]])
    check_decode(got, *t, [600, 0], [[40, 0], [40, 0]], "bf16")


def test_decode_strides_padded_and_broadcast():
    """Rows with padding between them, one query broadcast over the sequences, an own cache shared by two of them, O inside a larger buffer."""
    g = _gen(3)
    Q = u.randn(g, 1, 1, 4, 1, 128).expand(1, 3, 4, 1, 128)
    K, V = (torch.zeros(1, 2, 900, 136, dtype=torch.bfloat16, device="cuda:0")[..., :128] for _ in range(2))
    K.copy_(u.randn(g, 1, 2, 900, 128)), V.copy_(u.randn(g, 1, 2, 900, 128))
    oK, oV = (u.randn(g, 1, 1, 2, 60, 128).expand(1, 3, 2, 60, 128) for _ in range(2))
    buf = torch.full((1, 3, 4, 1, 200), 7.0, dtype=torch.bfloat16, device="cuda:0")
    O = buf[..., 40:168]
    p = s2o.make_decode_params(1, 3, 4, 2, 128, 1, 900, 60, q_stride=u.strides(Q), k_stride=u.strides(K), v_stride=u.strides(V),
                               own_k_stride=u.strides(oK), own_v_stride=u.strides(oV), o_stride=u.strides(O))
    t = (Q, K, V, oK, oV)
    check_decode(run_decode(t, p, O=O), *t, [900], [[60] * 3], "bf16")
    assert (buf[..., :40] == 7).all() and (buf[..., 168:] == 7).all()


def test_a_head_of_more_than_4_gib():
    """Row offsets beyond 32 bits: 70000 rows, 64 KiB apart."""
    g = _gen(5)
    L, st = 70000, 32768
    rows = u.randn(g, 1, 1, L, 64)
    base = torch.empty(((L - 1) * st + 64,), dtype=torch.bfloat16, device="cuda:0")
    K = base.as_strided((1, 1, L, 64), (0, 0, st, 1))
    K.copy_(rows)
    Q = u.randn(g, 1, 2, 2, 1, 64, gain=2.0)
    far = dict(k_stride=(8, 8, st))
    assert (L - 1) * st * 2 > 2 ** 32
    a = s2o.s2o_decode(Q, K, K, s2o.make_decode_params(1, 2, 2, 1, 64, 1, L, v_stride=(8, 8, st), **far))
    b = s2o.s2o_decode(Q, rows, rows, s2o.make_decode_params(1, 2, 2, 1, 64, 1, L))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    wa = s2o.s2o_key_weights(Q, K, s2o.make_weights_params(1, 2, 2, 1, 64, 1, L, **far), lse=a[1])
    wb = s2o.s2o_key_weights(Q, rows, s2o.make_weights_params(1, 2, 2, 1, 64, 1, L), lse=a[1])
    assert torch.equal(wa, wb) and abs(wa.sum().item() - 4) < 1e-4
    ea = s2o.s2o_evict(K, K, wa, s2o.make_evict_params(1, 1, 64, L, 1000, 4, 100, v_stride=(8, 8, st), **far))
    eb = s2o.s2o_evict(rows, rows, wb, s2o.make_evict_params(1, 1, 64, L, 1000, 4, 100))
    assert torch.equal(ea.kept, eb.kept) and torch.equal(ea.K, eb.K) and torch.equal(ea.V, eb.V) and int(ea.kept[0, 0, -1]) == L - 1


# ------------------------------------------------------------------------------------ accumulated weights
WEIGHTS = [
    # Z B H Hkv D T L dtype causal given token lens
    (1, 1, 1, 1, 128, 1, 1, "bf16", 1, 0, False, None),
    (1, 1, 8, 2, 128, 16, 300, "bf16", 1, 0, False, None),
    (2, 3, 4, 2, 64, 2, 777, "f16", 0, 1, True, [777, 500]),
    (1, 2, 8, 2, 128, 100, 1000, "bf16", 1, 0, True, [900]),
    (2, 1, 6, 2, 64, 700, 650, "f16", 1, 0, False, [650, 0]),                 # more queries than rows
    (1, 40, 8, 2, 128, 3, 520, "bf16", 0, 0, False, None),
    (3, 1, 4, 1, 64, 5, 70, "bf16", 1, 0, False, [70, 3, 64]),
    (1, 2, 4, 4, 128, 70, 300, "f16", 1, 1, False, [257]),
    (1, 1, 2, 1, 128, 1, 5000, "bf16", 0, 0, False, None),
    (1, 64, 8, 2, 64, 1, 2049, "f16", 0, 1, False, [2000]),
    (1, 1, 4, 2, 128, 1025, 1025, "bf16", 1, 0, False, None),                 # all queries of a prompt
]


@pytest.mark.parametrize("c", WEIGHTS, ids=lambda c: "-".join(map(str, c[:10])))
def test_weights(c):
    Z, B, H, Hkv, D, T, L, dt, causal, given, token, lens = c
    g = _gen(L + T)
    Q = u.randn(g, Z, B, H, T, D, dtype=dt, token=token, gain=2.0)
    K = u.randn(g, Z, Hkv, L, D, dtype=dt, token=token)
    lse = (math.log(L) + 2 * torch.rand(Z, B, H, T, generator=g)).cuda() if given else None
    prev = torch.rand(Z, Hkv, L, generator=g).cuda() if given else None
    st = dict(q_stride=u.strides(Q), k_stride=u.strides(K)) if token else {}
    p = s2o.make_weights_params(Z, B, H, Hkv, D, T, L, dtype=dt, causal=causal, **st)
    out = torch.full((Z, Hkv, L), 77.0, device="cuda:0")
    s2o.s2o_key_weights(Q, K, p, lse=lse, lens=_i32(lens), prev=prev, out=out)
    torch.cuda.synchronize()
    w, n = _f(out), lens or [L] * Z
    scale = 1 / math.sqrt(D)
    ref = u.key_weights(_f(Q), _f(K), n, causal, scale, _f(lse), _f(prev))
    tol = (2e-6 * _x(scale, _f(Q), _f(K)) + 4e-6 + B * T * (H // Hkv) * 2.0 ** -25) * np.abs(ref)
    for z in range(Z):
        assert np.all(np.abs(w - ref)[z, :, :n[z]] <= tol[z, :, :n[z]] + 1e-37), np.max(np.abs(w - ref)[z, :, :n[z]] / (tol[z, :, :n[z]] + 1e-37))
        assert np.all(w[z, :, n[z]:] == 77.0)                                 # behind the last row: as it was
    if not given and causal:
        # every query row hands out one unit of weight, where it sees anything
        rows = sum(B * (H // Hkv) * sum(v > 0 for v in u.visible(n[z], T, causal)) for z in range(Z))
        total = sum(w[z, 0, :n[z]].sum() for z in range(Z))
        assert abs(total - rows) <= 1e-4 * rows + 1e-6


def test_weights_in_place_and_fresh_output():
    g = _gen(9)
    Q, K = u.randn(g, 2, 3, 4, 1, 64), u.randn(g, 2, 2, 400, 64)
    p = s2o.make_weights_params(2, 3, 4, 2, 64, 1, 400)
    lens = _i32([400, 130])
    w1 = s2o.s2o_key_weights(Q, K, p, lens=lens)
    assert (w1[1, :, 130:] == 0).all()
    acc = torch.zeros_like(w1)
    for _ in range(2):
        assert s2o.s2o_key_weights(Q, K, p, lens=lens, prev=acc, out=acc) is acc
    assert torch.allclose(acc, 2 * w1, rtol=1e-6, atol=0)


def test_weights_of_rows_with_infinite_lse_and_bad_values_behind_the_end():
    g = _gen(11)
    Q, K = u.randn(g, 1, 2, 4, 3, 128), u.randn(g, 1, 2, 500, 128)
    lse = torch.full((1, 2, 4, 3), 6.0, device="cuda:0")
    p = s2o.make_weights_params(1, 2, 4, 2, 128, 3, 500, causal=1)
    lens = _i32([400])
    lse[0, 1] = -math.inf
    lse[0, 0, 0, 0] = math.inf
    w = s2o.s2o_key_weights(Q, K, p, lse=lse, lens=lens)
    ref = u.key_weights(_f(Q), _f(K), [400], 1, 1 / math.sqrt(128), _f(lse))
    assert np.allclose(_f(w), ref, rtol=1e-4, atol=0)
    K[:, :, 400:] = math.nan
    for l in (lse, None):
        K[:, :, 400:] = math.nan
        a = s2o.s2o_key_weights(Q, K, p, lse=l, lens=lens)
        K[:, :, 400:] = 0
        assert torch.equal(a, s2o.s2o_key_weights(Q, K, p, lse=l, lens=lens)) and torch.isfinite(a).all()
    # a key that only the last query token sees: the other rows' weights do not feel it
    K[0, 0, 399] = math.nan
    b = s2o.s2o_key_weights(Q, K, p, lse=lse, lens=lens)
    assert torch.equal(b[0, :, :399], w[0, :, :399]) and torch.isnan(b[0, 0, 399])


# ------------------------------------------------------------------------------------ eviction
def _weights(g, Z, Hkv, L, kind):
    w = torch.exp(2 * torch.randn(Z, Hkv, L, generator=g))
    if kind == "ties":
        w = torch.round(2 * w) / 2
    elif kind == "equal":
        w = torch.full_like(w, 0.25)
    elif kind == "signed":
        w = torch.randn(Z, Hkv, L, generator=g)
        w[..., ::7] = 0.0
        w[..., 3::7] = -0.0
    elif kind == "wild":
        w[..., ::5] = math.nan
        w[..., 1::5] = -math.inf
        w[..., 2::11] = math.inf
        w[..., 3::13] = 1e-42                                                 # below the normal numbers
    return w.cuda()


EVICT = [
    # Z Hkv D L keep sink recent dtype token lens kind
    (1, 1, 64, 1, 1, 0, 0, "bf16", False, None, "ties"),
    (1, 2, 128, 300, 100, 4, 16, "bf16", False, None, "plain"),
    (2, 2, 64, 5000, 777, 4, 100, "f16", True, [5000, 300], "ties"),
    (1, 1, 64, 100, 1, 0, 0, "bf16", False, None, "plain"),
    (1, 1, 64, 100, 1, 1, 0, "bf16", False, None, "plain"),
    (1, 1, 64, 100, 1, 0, 1, "bf16", False, None, "plain"),
    (1, 1, 64, 100, 100, 0, 0, "f16", False, None, "ties"),
    (4, 1, 64, 100, 50, 0, 50, "bf16", False, [0, 49, 50, 51], "plain"),
    (3, 3, 128, 1000, 500, 250, 250, "bf16", True, [1000, 499, 501], "ties"),
    (1, 2, 128, 20000, 3000, 0, 0, "bf16", False, None, "equal"),
    (2, 2, 64, 3000, 1234, 7, 9, "bf16", False, [3000, 2999], "signed"),
    (1, 3, 64, 4097, 2049, 1, 1, "f16", False, None, "wild"),
    (1, 2, 64, 4096, 3900, 1, 1, "f16", False, None, "wild"),
    (1, 1, 128, 70001, 20011, 4, 1000, "bf16", False, None, "ties"),
    (9, 5, 64, 513, 200, 4, 10, "bf16", False, [513, 0, 1, 4, 10, 14, 199, 200, 201], "ties"),
]


def check_evict(e, K, V, w, lens, keep, sink, recent, untouched):
    ref = u.evict(w.cpu().numpy(), lens, keep, sink, recent)
    for z, row in enumerate(ref):
        for g, at in enumerate(row):
            m = len(at)
            assert int(e.lens[z]) == m == min(lens[z], keep)
            assert np.array_equal(e.kept[z, g, :m].cpu().numpy(), at), (z, g)
            i = torch.from_numpy(at).cuda()
            for got, src in ((e.K, K), (e.V, V)):
                assert torch.equal(got[z, g, :m].view(torch.int16), src[z, g, i].view(torch.int16))
            assert torch.equal(e.weights[z, g, :m].view(torch.int32), w[z, g, i].view(torch.int32))
            if untouched:
                assert (e.K[z, g, m:] == 7).all() and (e.V[z, g, m:] == 7).all() and (e.weights[z, g, m:] == 7).all() and (e.kept[z, g, m:] == 7).all()


@pytest.mark.parametrize("c", EVICT, ids=lambda c: "-".join(map(str, c[:8])) + "-" + c[-1])
def test_evict(c):
    Z, Hkv, D, L, keep, sink, recent, dt, token, lens, kind = c
    g = _gen(L + keep)
    K, V = (u.randn(g, Z, Hkv, L, D, dtype=dt, token=token) for _ in range(2))
    w = _weights(g, Z, Hkv, L, kind)
    oK, oV = (torch.full((Z, keep, Hkv, D) if token else (Z, Hkv, keep, D), 7.0, dtype=u.DTYPES[dt], device="cuda:0") for _ in range(2))
    if token:
        oK, oV = oK.transpose(1, 2), oV.transpose(1, 2)
    st = dict(k_stride=u.strides(K), v_stride=u.strides(V), out_k_stride=u.strides(oK), out_v_stride=u.strides(oV)) if token else {}
    p = s2o.make_evict_params(Z, Hkv, D, L, keep, sink, recent, dtype=dt, **st)
    ow = torch.full((Z, Hkv, keep), 7.0, device="cuda:0")
    kept = torch.full((Z, Hkv, keep), 7, dtype=torch.int32, device="cuda:0")
    e = s2o.s2o_evict(K, V, w, p, lens=_i32(lens), out_K=oK, out_V=oV, out_weights=ow, kept=kept)
    torch.cuda.synchronize()
    check_evict(e, K, V, w, lens or [L] * Z, keep, sink, recent, True)


@pytest.mark.parametrize("L,keep,sink,recent,lens,kind", [
    (70001, 30011, 0, 0, [70001, 65536], "equal"),         # all rows share the last one's key: more than 16384 entries
    (70001, 40000, 4, 64, [70001, 39999], "signed"),
    (40000, 1, 0, 0, [40000, 1], "plain"),
    (40000, 100, 50, 50, [40000, 100], "plain"),           # nothing to choose
    (40000, 30000, 10, 20, [0, 29999], "plain"),           # all stay
    (40000, 30000, 10, 20, [3, 30001], "wild"),
    (32769, 16000, 4096, 4096, [32769, 32768], "ties"),
])
def test_evict_long(L, keep, sink, recent, lens, kind):
    g = _gen(L + keep)
    K, V = (u.randn(g, 2, 2, L, 64) for _ in range(2))
    w = _weights(g, 2, 2, L, kind)
    p = s2o.make_evict_params(2, 2, 64, L, keep, sink, recent)
    e = s2o.s2o_evict(K, V, w, p, lens=_i32(lens))
    torch.cuda.synchronize()
    check_evict(e, K, V, w, lens, keep, sink, recent, False)


def test_evict_selects_among_nine_million():
    """Stretches of more than one block of rows."""
    g = _gen(8)
    L, keep = 9_000_001, 5000
    w = torch.rand(1, 1, L, generator=g).cuda()
    w[0, 0, ::1000] = 2.0                                  # 9001 rows share the highest weight
    e = s2o.s2o_evict(None, None, w, s2o.make_evict_params(1, 1, 64, L, keep, 3, 5))
    at = np.concatenate([[0, 1, 2], np.arange(1, keep - 7) * 1000, np.arange(L - 5, L)])
    assert at.size == keep and int(e.lens[0]) == keep and np.array_equal(e.kept[0, 0].cpu().numpy(), at)
    assert torch.equal(e.weights[0, 0], w[0, 0, torch.from_numpy(at).cuda()])


def test_evict_moves_bits_and_allocates():
    """Rows are moved, not read as numbers: NaNs keep their payload.  Outputs that are not given are allocated."""
    g = _gen(2)
    bits = torch.randint(-2 ** 15, 2 ** 15, (1, 2, 600, 64), generator=g, dtype=torch.int16).cuda()
    K = bits.view(torch.bfloat16)
    w = _weights(g, 1, 2, 600, "plain")
    p = s2o.make_evict_params(1, 2, 64, 600, 100, 2, 2)
    e = s2o.s2o_evict(K, K, w, p)
    check_evict(e, K, K, w, [600], 100, 2, 2, False)
    only = s2o.s2o_evict(None, None, w, p)
    assert only.K is None and only.V is None and torch.equal(only.kept, e.kept) and torch.equal(only.weights, e.weights)


# ------------------------------------------------------------------------------------ streams, graphs, workspaces
def _three(seed=0):
    """One call of each operator on buffers that stay, as [(run, outputs)]."""
    g = _gen(seed)
    t, p = make_decode(2, 5, 8, 2, 128, 1, 3000, 40, "bf16", seed=seed)
    lens, own_lens = _i32([3000, 1700]), _i32([[40, 3, 0, 17, 33], [1, 2, 3, 4, 5]])
    O, lse = torch.zeros_like(t[0]), torch.zeros(2, 5, 8, 1, device="cuda:0")
    pw = s2o.make_weights_params(2, 5, 8, 2, 128, 1, 3000)
    pc = s2o.make_weights_params(2, 5, 8, 2, 128, 1, 3000, causal=1)
    pe = s2o.make_evict_params(2, 2, 128, 3000, 500, 4, 64)
    w, w2 = (torch.zeros(2, 2, 3000, device="cuda:0") for _ in range(2))
    e = [torch.zeros(2, 2, 500, 128, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)]
    ew, ek, el = torch.zeros(2, 2, 500, device="cuda:0"), torch.zeros(2, 2, 500, dtype=torch.int32, device="cuda:0"), torch.zeros(2, dtype=torch.int32, device="cuda:0")
    sizes = [s2o.s2o_decode_sizes(p)["scratch"], s2o.s2o_key_weights_sizes(pw, True)["scratch"], s2o.s2o_key_weights_sizes(pc)["scratch"],
             s2o.s2o_evict_sizes(pe)["scratch"]]
    scratch = torch.full((max(sizes) + 256,), 255, dtype=torch.uint8, device="cuda:0")      # NaN, wherever it is read as a number
    Q, K, V, oK, oV = t

    def run(stream=None):
        s2o.s2o_decode(Q, K, V, p, own_K=oK, own_V=oV, lens=lens, own_lens=own_lens, O=O, lse=lse, scratch=scratch, stream=stream)
        s2o.s2o_key_weights(Q, K, pw, lse=lse, lens=lens, out=w, scratch=scratch, stream=stream)
        s2o.s2o_key_weights(Q, K, pc, lens=lens, prev=w, out=w2, scratch=scratch, stream=stream)
        s2o.s2o_evict(K, V, w2, pe, lens=lens, out_K=e[0], out_V=e[1], out_weights=ew, kept=ek, out_lens=el, scratch=scratch, stream=stream)

    return run, [O, lse, w, w2, *e, ew, ek, el], (Q, K, V, lens, own_lens, scratch)


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_same_bits_every_time_whatever_the_scratch_holds():
    run, outs, (*_, scratch) = _three()
    run()
    torch.cuda.synchronize()
    first = [x.clone() for x in outs]
    for fill in (0, 255, 17):
        scratch.fill_(fill)
        run()
        torch.cuda.synchronize()
        assert _same(first, outs)


def test_another_stream():
    run, outs, _ = _three()
    run()
    torch.cuda.synchronize()
    first = [x.clone() for x in outs]
    for x in outs:
        x.zero_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    run(stream=s)
    s.synchronize()
    assert _same(first, outs)
    # outputs and scratch that the calls allocate, on that stream
    t, p = make_decode(1, 3, 4, 2, 64, 1, 2000, 9, "f16")
    a = run_decode(t, p)
    torch.cuda.synchronize()
    b = run_decode(t, p, stream=s)
    w = s2o.s2o_key_weights(t[0], t[1], s2o.make_weights_params(1, 3, 4, 2, 64, 1, 2000, dtype="f16"), lse=b[1], lens=_i32([1999]), stream=s)
    s.synchronize()
    assert _same(a, b) and (w[..., 1999:] == 0).all()


def test_outputs_for_another_stream_do_not_take_over_memory_that_is_in_use():
    """Memory that the current stream has freed, but not passed, is not what a call on another stream writes to."""
    t, p = make_decode(1, 64, 32, 8, 128, 1, 600, 0, "bf16")
    w = torch.rand(1, 8, 600, device="cuda:0")
    pw, pe = s2o.make_weights_params(1, 64, 32, 8, 128, 1, 600), s2o.make_evict_params(1, 8, 128, 600, 100, 2, 2)

    def calls(stream):
        O, lse = s2o.s2o_decode(t[0], t[1], t[2], p, stream=stream)
        e = s2o.s2o_evict(t[1], t[2], w, pe, stream=stream)
        return [O, lse, s2o.s2o_key_weights(t[0], t[1], pw, stream=stream), e.K, e.V, e.weights, e.kept, e.lens]

    want = calls(None)
    a = torch.zeros(4096, 4096, dtype=torch.bfloat16, device="cuda:0")
    late = [torch.empty_like(x) for x in want]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(200):
        torch.mm(a, a)                                     # tens of milliseconds, and behind them:
    for x in late:
        x.fill_(7)
    del late, x
    got = calls(s)
    torch.cuda.synchronize()
    assert _same(got, want)


def test_two_streams_at_once():
    """Calls with buffers and workspaces of their own, on two streams together."""
    sides = [_three(seed) for seed in (3, 4)]
    for run, _, _ in sides:
        run()
    torch.cuda.synchronize()
    first = [[x.clone() for x in outs] for _, outs, _ in sides]
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(5):
        for (run, _, _), s in zip(sides, streams):
            run(stream=s)
    torch.cuda.synchronize()
    for (_, outs, _), want in zip(sides, first):
        assert _same(outs, want)


def test_captured_and_replayed():
    """Two graphs on buffers and workspaces of their own, replayed in turn with changed inputs and lengths, eager work between."""
    sides = [_three(seed) for seed in (1, 2)]
    eager = [_three(seed) for seed in (1, 2)]
    graphs = []
    for run, outs, _ in sides:
        g = torch.cuda.CUDAGraph()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(g, stream=s):
            run(stream=torch.cuda.current_stream())
        graphs.append(g)
    for step in range(4):
        for (run, outs, ins), (erun, eouts, eins), g in zip(sides, eager, graphs):
            for x, y in zip(ins[:3], eins[:3]):
                x.copy_(torch.roll(x, 1 + step, dims=-2))
                y.copy_(x)
            for x, y in zip(ins[3:5], eins[3:5]):
                x.copy_(torch.clamp(x - 7 * step, min=0))
                y.copy_(x)
            erun()
            g.replay()
        torch.cuda.synchronize()
        for (_, outs, _), (_, eouts, _) in zip(sides, eager):
            assert _same(outs, eouts), step


# ------------------------------------------------------------------------------------ together
def test_prefill_weigh_evict_decode_weigh_evict():
    """A prompt through the prefill, its cache cut down by what its last queries looked at, sequences decoded on what is left, the cache cut
    again by what those looked at: every step against the definitions in 64 bits on the step's own inputs."""
    Z, H, Hkv, L, D, S, W, B, own = 1, 8, 2, 2048, 128, 256, 32, 6, 20
    g = _gen(21)
    Q, K, V = u.randn(g, Z, H, L, D, gain=2.0), u.randn(g, Z, Hkv, L, D), u.randn(g, Z, Hkv, L, D)
    pp = s2o.make_params(Z, H, Hkv, L, D, S)
    plan = s2o.s2o_plan(Q, K, pp)
    O, _, _ = s2o.s2o_attention(Q, K, V, pp, plan.q_perm, plan.kv_perm, 0.0)
    # the prefill without skipping and the cache's own attention agree on the prompt's last queries
    last = Q[:, None, :, L - W:]
    pd = s2o.make_decode_params(Z, 1, H, Hkv, D, W, 0, L, q_stride=u.strides(last))
    O2, lse = s2o.s2o_decode(last, None, None, pd, own_K=K[:, None], own_V=V[:, None])
    assert (O[:, :, L - W:].float() - O2[:, 0].float()).abs().max().item() <= 2e-2
    pw = s2o.make_weights_params(Z, 1, H, Hkv, D, W, L, causal=1, q_stride=u.strides(last))
    w = s2o.s2o_key_weights(last, K, pw)
    scale = 1 / math.sqrt(D)
    assert np.allclose(_f(w), u.key_weights(_f(last), _f(K), [L], 1, scale), rtol=1e-4, atol=1e-30)
    given = s2o.s2o_key_weights(last, K, pw, lse=lse)                          # the same from the attention's own normaliser
    assert torch.allclose(w, given, rtol=2e-5, atol=0)
    keep = 500
    e = s2o.s2o_evict(K, V, w, s2o.make_evict_params(Z, Hkv, D, L, keep, 4, W))
    check_evict(e, K, V, w, [L], keep, 4, W, False)
    # six sequences on what is left
    q, oK, oV = u.randn(g, Z, B, H, 1, D, gain=2.0), u.randn(g, Z, B, Hkv, own, D), u.randn(g, Z, B, Hkv, own, D)
    lens = [1, 5, 20, 0, 7, 19]
    pd = s2o.make_decode_params(Z, B, H, Hkv, D, 1, keep, own)
    got = s2o.s2o_decode(q, e.K, e.V, pd, own_K=oK, own_V=oV, lens=e.lens, own_lens=_i32([lens]))
    torch.cuda.synchronize()
    check_decode(got, q, e.K, e.V, oK, oV, [keep], [lens], "bf16")
    pw = s2o.make_weights_params(Z, B, H, Hkv, D, 1, keep)
    w2 = s2o.s2o_key_weights(q, e.K, pw, lse=got[1], lens=e.lens, prev=e.weights)
    ref = u.key_weights(_f(q), _f(e.K), [keep], 0, scale, _f(got[1]), _f(e.weights))
    assert np.allclose(_f(w2), ref, rtol=1e-4, atol=1e-30)
    e2 = s2o.s2o_evict(e.K, e.V, w2, s2o.make_evict_params(Z, Hkv, D, keep, 200, 4, 10), lens=e.lens)
    check_evict(e2, e.K, e.V, w2, [keep], 200, 4, 10, False)
