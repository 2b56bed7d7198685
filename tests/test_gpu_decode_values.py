"""Decode kernels on calls that the definitions allow and ordinary inputs do not make: infinities, ties under a threshold that no
weight reaches, rows that begin between 16 bytes, fp32 angles of far positions.

u = 2^-24 (fp32), half a step of bf16 relative to the value 2^-8; tolerances are derived beside their use."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import zo_decode as od
from paper_2605_28760_amd import binding as zb
from test_gpu_decode import DEV, HALF, TT, U, ZT, Setup, _check_draw, _i32, _np


def _exact(s, t, head, scale):
    """(output, sum of weights times |values|, largest scale * |q| |k|) of a row and head in 64 bits."""
    i, pos = od.row_places(s.cu, s.kv)[t]
    n = head // (s.H // s.g)
    at = [(od.page_of(s.table, s.P, s.n_pages, i, j), j % s.P) for j in range(pos + 1)]
    pg, sl = np.array([x for x in at if x[0] is not None]).T
    k, v, q = _np(s.K[pg, n, sl]), _np(s.V[pg, n, sl]), _np(s.q[t]).reshape(s.H, s.dh)[head]
    z = scale * (k @ q)
    p = np.exp(z - z.max())
    p /= p.sum()
    return p @ v, p @ np.abs(v), abs(scale) * (np.abs(k) @ np.abs(q)).max(), len(p)


@pytest.mark.parametrize("H,g,dh,kv", [(4, 1, 128, [2, 16, 33, 257, 700]), (20, 1, 64, [5, 300]), (3, 3, 256, [31, 600]), (8, 2, 128, [3000])])
def test_bf16_attention_rounds_its_output_only(H, g, dh, kv):
    """The weights keep 15 bits and more (2^-15 + 2^-20 of each): what is left is the fp32 arithmetic, scores (dh + 3) u of
    scale * sum |q_d k_d| (twice that in the quotient) and n + 16 roundings of the sums, and the output's own half step."""
    s = Setup(H + dh, "bf16", H, g, dh, 16, [1] * len(kv), kv)
    out, scale = _np(s.attend()), dh ** -0.5
    for t in range(s.T):
        for head in range(H):
            want, size, big, n = _exact(s, t, head, scale)
            tol = (2 * (dh + 3) * U * big + (n + 16) * U + 2.0 ** -15 + 2.0 ** -20) * size + 2.0 ** -8 * np.abs(want)
            err = np.abs(out[t, head * dh:(head + 1) * dh] - want)
            assert (err <= tol).all(), (t, head, float((err / tol).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 300, 3001, 9001])
def test_min_p_above_one_keeps_the_first_of_the_largest(dtype, V):
    """No weight reaches it: max(1, 0) tokens are kept, also where several share the maximum."""
    rng = np.random.default_rng(V)
    z = np.round(rng.normal(size=(8, V)))
    z[0] = 0.25
    z[1, V // 2:] = z[1].max() + 1
    z[2, [0, V - 1]] = np.inf
    z[3] = np.inf
    z[4, ::2] = -np.inf
    z[5] = -np.inf
    z[6, V // 3:] = np.nan
    zt = torch.from_numpy(z).to(DEV).to(TT[dtype])
    u = [0.9, 0.9, 0.9, 0.5, 0.9, 0.9, 0.9, 1.0]
    for m in (1.5, float(np.nextafter(np.float32(1), np.float32(2))), np.inf):
        for k, p in ((None, None), ([V - 1] * 8, None), (None, [0.999] * 8), ([200] * 8, [0.999] * 8)):
            _check_draw(zt, [0.7] * 8, k, p, [m] * 8, u)
    _check_draw(zt, [0.7] * 8, None, None, [1.0] * 8, u)        # (the weight at the maximum reaches 1)
    _check_draw(zt, [0.7] * 8, None, None, [1.5, 1.0] * 4, u)   # rows of both kinds


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 24)])
@pytest.mark.parametrize("width", [64, 200])
def test_a_query_whose_scores_are_all_minus_infinity(dtype, dh, width):
    """Its softmax has no value: NaN, in whichever way the ranges are joined.  A range of them beside a finite one has no weight;
    a row that sees no position stays zero."""
    kv = [1, 45, 300, 700, 900, 0, 900]
    s = Setup(31, dtype, 4, 2, dh, 16, [1] * len(kv), kv, width=width)
    s.q[:, 0::dh] = s.q[:, 0::dh].abs() + 0.1
    for i, n in enumerate((1, 45, 300, 700, 640, 0, 0)):
        for p in range(n):
            s.K[int(s.table[i, p // 16]), :, p % 16, 0] = float("-inf")
    s.table[6] = -1
    s.d_table.copy_(_i32(s.table))
    got = _np(s.attend())[:, :4 * dh]
    assert np.isnan(got[:4]).all()
    assert (got[5:] == 0).all()
    s.kv[0:4] = [0] * 4
    got[:4] = 0
    s.check_attend(torch.from_numpy(got))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("bf16", 256), ("f32", 64), ("f32", 128), ("f32", 24)])
def test_infinite_values_that_are_seen_stay_infinite(dtype, dh):
    """The last position's value is infinite and its key stands in for the slots behind it, which have no weight."""
    kv = [1, 2, 17, 33, 45, 260, 700]
    s = Setup(32, dtype, 4, 2, dh, 16, [1] * len(kv), kv)
    for i, n in enumerate(kv):
        s.V[int(s.table[i, (n - 1) // 16]), :, (n - 1) % 16, 1] = float("inf")
        s.V[int(s.table[i, (n - 1) // 16]), :, (n - 1) % 16, 2] = float("-inf")
    got = _np(s.attend())[:, :4 * dh].reshape(len(kv), 4, dh)
    assert (got[:, :, 1] == np.inf).all() and (got[:, :, 2] == -np.inf).all()
    assert np.isfinite(got[:, :, 3:]).all()


@pytest.mark.parametrize("dh", [64, 80, 128, 256, 7])
@pytest.mark.parametrize("offset,pad", [(1, 0), (2, 3), (3, 1), (0, 1)])
def test_fp32_attention_rows_that_begin_between_16_bytes(dh, offset, pad):
    kv = [1, 40, 300, 600]
    s = Setup(33, "f32", 4, 2, dh, 16, [1] * 4, kv)
    plain = s.attend().clone()[:, :4 * dh]
    ld = 4 * dh + pad
    q, o = (torch.full((4 * ld + 8,), 7.0, device=DEV)[offset:offset + 4 * ld].view(4, ld) for _ in range(2))
    q[:, :4 * dh] = s.q
    ws = s.workspace()
    zb.zo_attention_paged(s.batch, q, ld, 4, dh ** -0.5, s.cache, o, ld, ws[0], ws[1])
    assert torch.equal(o[:, :4 * dh], plain) and (o[:, 4 * dh:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [64, 128, 256, 8])
def test_append_without_rotation_takes_infinities_as_they_are(dtype, dh):
    """No rotation: an infinite value turns neither itself nor its partner into NaN."""
    s = Setup(dh, dtype, 4, 2, dh, 16, [1, 3], [20, 3])
    for col, x in ((0, np.inf), (dh // 2 + 1, -np.inf), (4 * dh + 2, np.inf), (5 * dh + dh // 2 + 3, -np.inf)):
        s.qkv[:, col] = x
    s.append(None, None, 0.0)
    assert torch.equal(s.out, s.q)
    for i, pos, t in ((0, 19, 0), (1, 0, 1), (1, 2, 3)):
        for pool, rows in ((s.K, s.k), (s.V, s.v)):
            assert torch.equal(pool[int(s.table[i, pos // 16]), :, pos % 16].reshape(-1), rows[t])
    gain = torch.ones(dh, device=DEV)
    s.append(gain, gain, 0.0)                                  # the norm: 1 / inf of the others, NaN of the infinite one alone
    got = _np(s.out)[:, :dh]
    assert np.isnan(got[:, 0]).all() and (got[:, 1:dh // 2 + 1] == 0).all()


@pytest.mark.parametrize("dh", [64, 128, 256])
def test_fp32_rotation_does_not_depend_on_the_path(dh):
    """Without a norm a rotated pair is two products of the row and the rounded sine and cosine: aligned rows, rows that begin
    between 16 bytes and the packed prompt's rotation give the same bits."""
    H, g, n, far = 4, 2, 300, 131072 - 40
    for past in (0, far):
        kv = [n + past]
        s = Setup(dh, "f32", H, g, dh, 1024, [n], kv)
        s.append(None, None, 1e4)
        a, ka = s.out.clone(), s.K.clone()
        odd = torch.empty(n, s.ld + 1, device=DEV)[:, 1:]
        odd.copy_(s.qkv)
        out = torch.empty(n, H * dh, device=DEV)
        ld = odd.stride(0)
        s.K.zero_()
        zb.zo_cache_append(s.batch, odd, ld, odd[:, H * dh:], ld, odd[:, (H + g) * dh:], ld, H, None, None, 0.0, 1e4, s.cache, out, H * dh)
        page = [int(s.table[0, p // 1024]) for p in range(past, past + n)]
        at = (torch.tensor(page, device=DEV), slice(None), torch.arange(past, past + n, device=DEV) % 1024)
        assert torch.equal(a[:, :H * dh], out) and torch.equal(ka[at], s.K[at])
        if past == 0:
            qkv = s.qkv.clone()
            zb.zo_qk_norm_rope(s.batch, qkv, s.ld, qkv[:, H * dh:], s.ld, H, g, dh, None, None, 0.0, 1e4, zb.ZO_F32)
            assert torch.equal(qkv[:, :H * dh], out)
        # a rounded sine and cosine (u of 1 each), two products and a sum: 3 u of the pair's length
        q, _, _ = od.cache_append(_np(s.q), _np(s.k), _np(s.v), s.cu, H, None, None, 0.0, 1e4, _np(s.K), _np(s.V), s.table, kv)
        w = q.reshape(n, H, 2, dh // 2)
        tol = 3.01 * U * np.hypot(w[:, :, 0], w[:, :, 1])[:, :, None]
        assert (np.abs(_np(out).reshape(w.shape) - w) <= tol).all()


@pytest.mark.parametrize("dh", [128, 8])
def test_append_in_place_without_norm_and_rotation_leaves_the_queries(dh):
    """Not even a signalling NaN is made quiet; keys and values go to their slots, the rest of the pools stays."""
    s = Setup(dh + 1, "bf16", 4, 2, dh, 16, [1, 0, 40], [20, 0, 40], extra_rows=1)
    s.qkv[:, :4 * dh] = torch.tensor([0x7F81], dtype=torch.int16, device=DEV).view(torch.bfloat16)
    bits, K0, V0 = s.qkv.view(torch.int16).clone(), _np(s.K), _np(s.V)
    s.append(None, None, 0.0, out=s.qkv)
    assert torch.equal(s.qkv.view(torch.int16), bits)
    _, K, V = od.cache_append(np.zeros((41, 4 * dh)), _np(s.k)[:41], _np(s.v)[:41], s.cu, 4, None, None, 0.0, 0.0, K0, V0, s.table, s.kv)
    assert (_np(s.K) == K).all() and (_np(s.V) == V).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 33, 1000])
def test_positions_alone_are_advanced(dtype, n):
    pos = _i32(np.arange(n) * 7 - 3)
    for alias in (False, True):
        start, nxt = pos.clone(), torch.zeros_like(pos)
        nxt = start if alias else nxt
        zb.zo_embed_rows(torch.zeros_like(pos), start, n, None, 0, 0, None, 0, 0, 0, ZT[dtype], None, 0, nxt)
        assert torch.equal(nxt, pos + 1)
