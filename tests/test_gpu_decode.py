"""GPU parity of the decode entry points (paged cache, attention over it, sampling, embedding rows) against the fp64
oracle, at the sizes and tables where they can go wrong.

Tolerances, element by element.  u = 2^-24 (fp32), h = half a step of the storage type relative to the value (bf16 2^-8, fp32 u).
  append     a pair's values pass a sum of squares (dh/64 + 8 additions, halved by the root), 4 products and one
             rotation of rounded factors: 24 u of the pair's length, and h of the value
  attention  a score's error is (dh + 3) u of scale * sum |q_d k_d|; twice that, and n + 16 roundings of the sums, and h for
             the weight where it is stored as bf16, of sum_j p_j |v_j|; h of the value
  sampling   tokens and counts are exact; probabilities are formed in 64 bits and rounded once
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import zo_decode as od
from paper_2605_28760_amd import binding as zb

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}
TT = {"bf16": torch.bfloat16, "f32": torch.float32}
ZT = {"bf16": zb.ZO_BF16, "f32": zb.ZO_F32}


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.is_floating_point() else t.detach().cpu().numpy()


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


class Setup:
    """Random pools, a table whose pages lie in any order, rows of `rows[i]` tokens of sequences of `kv[i]` positions."""

    def __init__(self, seed, dtype, H, g, dh, P, rows, kv, extra_rows=0, width=None, ld_pad=0):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.H, self.g, self.dh, self.P, self.rows, self.kv = dtype, H, g, dh, P, list(rows), list(kv)
        tt = TT[dtype]
        pages = [-(-n // P) for n in kv]
        self.n_pages = sum(pages) + 3
        self.width = width or max(max(pages), 1)
        perm = rng.permutation(self.n_pages)
        self.table = np.full((len(kv), self.width), -1, np.int32)
        at = 0
        for i, n in enumerate(pages):
            self.table[i, :n] = perm[at:at + n]
            at += n
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        normal = lambda *s: torch.randn(s, device=DEV, generator=gen).to(tt)
        self.K, self.V = normal(self.n_pages, g, P, dh), normal(self.n_pages, g, P, dh)
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.S, self.T = len(rows), int(self.cu[-1]) + extra_rows
        pad = 8 * ld_pad
        self.qkv = normal(self.T, (H + 2 * g) * dh + pad)
        self.ld = self.qkv.stride(0)
        self.q, self.k, self.v = (self.qkv[:, a * dh:b * dh] for a, b in ((0, H), (H, H + g), (H + g, H + 2 * g)))
        self.out = torch.full((self.T, H * dh + pad), 7.0, device=DEV, dtype=tt)
        self.d_cu, self.d_kv, self.d_table = _i32(self.cu), _i32(kv), _i32(self.table)
        self.none = _i32(np.full(max(self.S, 1), -1))
        self.batch = zb.make_batch(self.T, self.d_cu, self.none, None, None, None, n_seqs=self.S, n_cands=0, n_dirs=0)
        self.cache = zb.make_cache(self.K, self.V, ZT[dtype], self.d_table, self.d_kv)

    def append(self, gq=None, gk=None, theta=0.0, out=None, stream=None):
        out = self.out if out is None else out
        zb.zo_cache_append(self.batch, self.q, self.ld, self.k, self.ld, self.v, self.ld, self.H, gq, gk, 1e-6, theta, self.cache,
                           out, out.stride(0), stream)
        return out

    def workspace(self):
        n = zb.zo_attention_paged_workspace_bytes(self.T, self.H, self.dh, self.width * self.P, ZT[self.dtype])
        return torch.empty(max(n, 256), device=DEV, dtype=torch.uint8), n

    def attend(self, scale=None, out=None, stream=None, ws=None):
        out = self.out if out is None else out
        ws = ws or self.workspace()
        zb.zo_attention_paged(self.batch, self.q, self.ld, self.H, self.dh ** -0.5 if scale is None else scale, self.cache, out,
                              out.stride(0), ws[0], ws[1], stream)
        return out

    def check_attend(self, got, scale=None):
        scale = self.dh ** -0.5 if scale is None else scale
        H, g, dh, P = self.H, self.g, self.dh, self.P
        q, K, V = _np(self.q), _np(self.K), _np(self.V)
        got = _np(got)[:, :H * dh].reshape(self.T, H, dh)
        h = HALF[self.dtype]
        places = od.row_places(self.cu, self.kv)
        for t, (i, pos) in enumerate(places):
            at = [(od.page_of(self.table, P, self.n_pages, i, j), j % P) for j in range(pos + 1)]
            at = [(p, s) for p, s in at if p is not None]
            if not at:
                assert (got[t] == 0).all(), (t, i, pos)
                continue
            pg, sl = np.array(at).T
            for n in range(g):
                k, v = K[pg, n, sl], V[pg, n, sl]
                for head in range(n * (H // g), (n + 1) * (H // g)):
                    x = q[t].reshape(H, dh)[head]
                    s = scale * (k @ x)
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    want, size = p @ v, p @ np.abs(v)
                    ds = (dh + 3) * U * abs(scale) * (np.abs(k[s > -np.inf]) @ np.abs(x)).max()
                    tol = (2 * ds + (len(p) + 16) * U + (h if self.dtype == "bf16" else 0)) * size + h * np.abs(want)
                    err = np.abs(got[t, head] - want)
                    assert (err <= tol).all(), (t, i, pos, head, float((err / tol).max()))


# ------------------------------------------------------------------ append

APPEND = [("bf16", 32, 8, 128, 16, [1] * 5, [1, 16, 17, 400, 33]), ("bf16", 4, 2, 128, 64, [70, 0, 3, 1], [70, 5, 130, 64]),
          ("bf16", 5, 5, 64, 32, [1, 40], [9, 40]), ("bf16", 2, 1, 256, 16, [3], [70000]), ("bf16", 3, 3, 8, 16, [2, 2], [20, 2]),
          ("f32", 8, 4, 64, 16, [1, 7], [300, 7]), ("f32", 3, 1, 80, 128, [5], [5]), ("f32", 2, 2, 2, 16, [1], [40]),
          ("f32", 4, 4, 256, 1024, [2], [131072]), ("bf16", 40, 40, 128, 16, [1] * 3, [2, 2048, 700])]


@pytest.mark.parametrize("dtype,H,g,dh,P,rows,kv", APPEND)
@pytest.mark.parametrize("norm,theta", [(True, 1e6), (False, 1e4), (True, 0.0), (False, 0.0)])
def test_append(dtype, H, g, dh, P, rows, kv, norm, theta):
    s = Setup(dh + H, dtype, H, g, dh, P, rows, kv, extra_rows=2, ld_pad=1)
    gain = (lambda: torch.from_numpy((1 + 0.1 * s.rng.normal(size=dh)).astype(np.float32)).to(DEV)) if norm else (lambda: None)
    gq, gk = gain(), gain()
    K0, V0 = _np(s.K), _np(s.V)
    s.append(gq, gk, theta)
    n = s.T - 2
    args = [_np(x) if x is not None else None for x in (gq, gk)]
    q, K, V = od.cache_append(_np(s.q)[:n], _np(s.k)[:n], _np(s.v)[:n], s.cu, H, args[0], args[1], 1e-6, theta, K0, V0, s.table, s.kv)
    got = _np(s.out)
    assert (got[n:] == 7).all() and (got[:, H * dh:] == 7).all()          # rows behind the last sequence, columns behind the heads
    assert (_np(s.V) == V).all()
    plain = not norm and theta <= 0
    for have, want in ((got[:n, :H * dh].reshape(n, H, dh), q.reshape(n, H, dh)), (_np(s.K), K)):
        half = dh // 2
        pair = np.hypot(want[..., :half], want[..., half:])
        tol = 24 * U * np.concatenate([pair, pair], -1) + HALF[dtype] * np.abs(want)
        assert (have == want if plain else np.abs(have - want) <= tol).all()
    moved = (_np(s.K) != K0).any(axis=(1, 3))
    slots = {(od.page_of(s.table, P, s.n_pages, i, p), p % P) for i, p in od.row_places(s.cu, s.kv)}
    assert all((int(a), int(b)) in slots for a, b in np.argwhere(moved))


def test_append_in_place_and_bad_tables():
    s = Setup(3, "bf16", 4, 2, 128, 16, [1, 1, 1, 1, 2], [20, 5, 64, 33, 1])
    table = s.table.copy()
    table[0, 1], table[1, 0] = -1, s.n_pages          # the pages of rows 0 and 1
    s.d_table.copy_(_i32(table))
    s.d_kv.copy_(_i32([20, 5, 65, 33, 1]))            # row 2 lies behind its table, row 4 before its sequence's first position
    K0, V0 = _np(s.K), _np(s.V)
    q0 = _np(s.q)
    s.append(None, None, 1e4, out=s.qkv)
    q, K, V = od.cache_append(q0, _np(s.k), _np(s.v), s.cu, 4, None, None, 0.0, 1e4, K0, V0, table, [20, 5, 65, 33, 1])
    assert (_np(s.V) == V).all() and (np.abs(_np(s.K) - K) <= 2 ** -8 * np.abs(K) + 1e-5).all()
    assert (np.abs(_np(s.q) - q) <= 2 ** -8 * np.abs(q) + 1e-5).all()


# ------------------------------------------------------------------ attention

LENS = [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 1025]
ATTEND = [("bf16", 4, 1, 128, 16, LENS), ("bf16", 2, 2, 128, 64, LENS), ("bf16", 8, 1, 64, 32, LENS), ("bf16", 12, 1, 256, 16, LENS[::2]),
          ("bf16", 16, 1, 128, 16, LENS[::2]), ("bf16", 17, 1, 128, 16, LENS[::3]), ("bf16", 40, 1, 64, 256, LENS[::3]),
          ("bf16", 32, 8, 128, 1024, [1, 700, 1500]), ("bf16", 5, 5, 128, 16, [9000]), ("bf16", 4, 2, 128, 64, [17000]),
          ("f32", 4, 1, 128, 16, LENS), ("f32", 2, 2, 64, 64, LENS), ("f32", 6, 3, 80, 16, LENS[::2]), ("f32", 3, 1, 1, 16, LENS[::3]),
          ("f32", 20, 1, 256, 32, LENS[::3]), ("f32", 2, 1, 7, 16, [300]), ("f32", 4, 2, 128, 16, [9000]), ("f32", 2, 1, 64, 16, [17000]),
          ("f32", 9, 1, 32, 16, [1, 70, 600])]


@pytest.mark.parametrize("dtype,H,g,dh,P,kv", ATTEND)
def test_attention(dtype, H, g, dh, P, kv):
    s = Setup(H * 1000 + dh, dtype, H, g, dh, P, [1] * len(kv), kv, extra_rows=1, ld_pad=2)
    out = s.attend()
    s.check_attend(out)
    assert (_np(out)[s.T - 1:] == 7).all() and (_np(out)[:, H * dh:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_several_rows_of_a_sequence(dtype):
    s = Setup(11, dtype, 8, 2, 128, 16, [3, 0, 1, 5, 70], [3, 40, 1, 300, 333])
    s.check_attend(s.attend())


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 128), ("f32", 24)])
def test_stale_slots_bad_pages_and_empty_rows(dtype, dh):
    kv = [1, 20, 40, 100, 300, 0, 700, 520, 2000]
    s = Setup(12, dtype, 4, 2, dh, 16, [1] * len(kv), kv, width=140)
    used = np.zeros((s.n_pages, 16), bool)
    for i, n in enumerate(kv):
        for p in range(n):
            used[s.table[i, p // 16], p % 16] = True
    free = torch.from_numpy(~used).to(DEV)
    for X in (s.K, s.V):                              # whatever the pool holds where nothing was stored
        X.masked_fill_(free[:, None, :, None], float("nan"))
        X[0:1].masked_fill_(free[0:1, None, :, None], float("inf"))
    s.check_attend(s.attend())
    s.table[3, 2] = -1                                # a hole
    s.table[4, :] = s.n_pages + 5                     # no page at all
    s.table[6, 5:20] = -7                             # a hole over several tiles
    s.table[7, :16] = 1 << 30                         # the first 256 positions
    s.table[8, 100:] = -1                             # the last ones
    s.d_table.copy_(_i32(s.table))
    s.check_attend(s.attend())
    s.kv[0], s.kv[1], s.kv[8] = -5, 0, 140 * 16       # lengths that leave nothing, and a whole table
    s.d_kv.copy_(_i32(s.kv))
    s.check_attend(s.attend())
    s.d_kv[8] = 140 * 16 + 1000                       # beyond the table: what it names is seen
    out = _np(s.attend())[8]
    s.d_kv[8] = 140 * 16
    np.testing.assert_allclose(_np(s.attend())[8], out, rtol=2e-2, atol=2e-2)


@pytest.mark.parametrize("scale,shift", [(1.0, 0.0), (30.0, 0.0), (-0.2, 0.0), (0.0, 0.0), (0.088, 300.0)])
def test_attention_of_large_scores(scale, shift):
    s = Setup(13, "f32", 4, 2, 64, 16, [1] * 3, [50, 257, 600])
    s.K += shift
    s.check_attend(s.attend(scale), scale)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64)])
def test_keys_at_minus_infinity_have_no_weight(dtype, dh):
    """Whole steps, whole ranges and only some heads' scores at -infinity before the first finite one."""
    kv = [45, 300, 700, 1400]
    s = Setup(16, dtype, 4, 2, dh, 16, [1] * 4, kv)
    s.q[:, 0::dh] = s.q[:, 0::dh].abs() + 0.1           # every head's first value: positive ..
    for i, n in enumerate((40, 270, 150, 1390)):
        for p in range(n):
            s.K[int(s.table[i, p // 16]), (0 if i == 2 else slice(None)), p % 16, 0] = float("-inf")   # .. times -infinity
    got = _np(s.attend())
    assert np.isfinite(got[:, :4 * dh]).all()
    s.check_attend(s.out)


def test_thousands_of_sequences():
    """More sequences than one look at the bounds holds, empty ones among them."""
    rng = np.random.default_rng(17)
    rows = rng.integers(0, 2, 4500)
    kv = rows + rng.integers(0, 30, 4500)
    s = Setup(17, "f32", 1, 1, 64, 16, rows, kv, extra_rows=3)
    K0, V0 = _np(s.K), _np(s.V)
    s.append(None, None, 1e4, out=s.out)
    q, K, V = od.cache_append(_np(s.q)[:s.T - 3], _np(s.k), _np(s.v), s.cu, 1, None, None, 0.0, 1e4, K0, V0, s.table, s.kv)
    assert (_np(s.V) == V).all() and (np.abs(_np(s.K) - K) <= 1e-5).all() and (np.abs(_np(s.out)[:s.T - 3] - q) <= 1e-5).all()
    s.check_attend(s.attend())
    assert (_np(s.out)[s.T - 3:] == 7).all()


def test_rows_do_not_depend_on_the_batch_or_the_table():
    kv = [1, 70, 256, 257, 900, 3000, 20000]
    for dtype, H, g, dh in (("bf16", 8, 2, 128), ("f32", 4, 2, 64), ("f32", 3, 1, 24)):
        s = Setup(14, dtype, H, g, dh, 16, [1] * len(kv), kv)
        whole = _np(s.attend()).copy()
        for i in (0, 2, 4, 6):                        # alone, with a table of its own width, behind a wider one
            for width in (-(-kv[i] // 16), s.width + 500):
                table = np.full((1, width), -1, np.int32)
                n = min(width, s.width)
                table[0, :n] = s.table[i, :n]
                d_table, d_kv, d_cu = _i32(table), _i32([kv[i]]), _i32([0, 1])
                batch = zb.make_batch(1, d_cu, s.none, None, None, None, n_seqs=1, n_cands=0, n_dirs=0)
                cache = zb.make_cache(s.K, s.V, ZT[dtype], d_table, d_kv)
                out = torch.empty(1, H * dh, device=DEV, dtype=TT[dtype])
                need = zb.zo_attention_paged_workspace_bytes(1, H, dh, width * 16, ZT[dtype])
                ws = torch.full((max(need, 256),), 255, device=DEV, dtype=torch.uint8)
                q = s.q[i:i + 1]
                zb.zo_attention_paged(batch, q, s.ld, H, dh ** -0.5, cache, out, H * dh, ws, need)
                assert (_np(out)[0] == whole[i]).all(), (dtype, i, width)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 36)])
def test_every_form_of_a_call_gives_a_row_the_same_bits(dtype, dh):
    """One workgroup per row, ranges joined by a second launch with a workgroup or a wave per row and head."""
    cap = 1024 if dtype == "bf16" else 512
    kv = [1, 100, cap // 4, cap // 4 + 1, cap // 2 + 7, cap // 4 * 3, cap - 1, cap]
    s = Setup(15, dtype, 4, 2, dh, 16, [1] * 8, kv, width=cap // 16)
    first = _np(s.attend()).copy()
    s.check_attend(s.out)
    for copies, width in ((1, cap // 16 + 1), (1, 4 * cap // 16), (40, cap // 16), (40, 2 * cap // 16)):
        table = np.full((8 * copies, width), -1, np.int32)
        table[:, :cap // 16] = np.tile(s.table, (copies, 1))
        d_table, d_kv, d_cu = _i32(table), _i32(np.tile(kv, copies)), _i32(np.arange(8 * copies + 1))
        none = _i32(np.full(8 * copies, -1))
        q = s.q.repeat(copies, 1)
        batch = zb.make_batch(8 * copies, d_cu, none, None, None, None, n_seqs=8 * copies, n_cands=0, n_dirs=0)
        cache = zb.make_cache(s.K, s.V, ZT[dtype], d_table, d_kv)
        out = torch.empty(8 * copies, 4 * dh, device=DEV, dtype=TT[dtype])
        need = zb.zo_attention_paged_workspace_bytes(8 * copies, 4, dh, width * 16, ZT[dtype])
        ws = torch.full((max(need, 256),), 255, device=DEV, dtype=torch.uint8)
        zb.zo_attention_paged(batch, q, q.stride(0), 4, dh ** -0.5, cache, out, 4 * dh, ws, need)
        assert (_np(out).reshape(copies, 8, -1) == first[None, :, :4 * dh]).all(), (copies, width)


def test_far_offsets():
    """Pages beyond 2^31 elements and 2^32 bytes of a pool."""
    P, g, dh = 1024, 8, 128
    n_pages = (1 << 32) // (P * g * dh * 2) + 200     # 4.6 GB a pool
    K = torch.zeros(n_pages, g, P, dh, device=DEV, dtype=torch.bfloat16)
    V = torch.zeros_like(K)
    far = n_pages - 1
    table, kv, cu = _i32([[far]]), _i32([37]), _i32([0, 37])
    none = _i32([-1])
    cache = zb.make_cache(K, V, zb.ZO_BF16, table, kv)
    batch = zb.make_batch(37, cu, none, None, None, None, n_seqs=1, n_cands=0, n_dirs=0)
    qkv = torch.randn(37, 3 * g * dh, device=DEV).bfloat16()
    out = torch.empty(37, g * dh, device=DEV, dtype=torch.bfloat16)
    ld = qkv.stride(0)
    zb.zo_cache_append(batch, qkv, ld, qkv[:, g * dh:], ld, qkv[:, 2 * g * dh:], ld, g, None, None, 0.0, 0.0, cache, out, g * dh)
    assert torch.equal(V[far, :, :37].transpose(0, 1).reshape(37, -1), qkv[:, 2 * g * dh:])
    assert torch.equal(K[far, :, :37].transpose(0, 1).reshape(37, -1), qkv[:, g * dh:2 * g * dh])
    assert not K[:far].any() and not V[:far].any() and not K[far, :, 37:].any()
    need = zb.zo_attention_paged_workspace_bytes(37, g, dh, P, zb.ZO_BF16)
    ws = torch.empty(max(need, 256), device=DEV, dtype=torch.uint8)
    zb.zo_attention_paged(batch, qkv, ld, g, 0.1, cache, out, g * dh, ws, need)
    q, k, v = (qkv[:, i * g * dh:(i + 1) * g * dh].float().view(37, g, dh).transpose(0, 1).contiguous() for i in range(3))
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * 0.1
    s = s.masked_fill(torch.triu(torch.ones(37, 37, device=DEV, dtype=torch.bool), 1), float("-inf"))
    want = torch.matmul(torch.softmax(s, -1), v).transpose(0, 1).reshape(37, -1)
    assert (out.float() - want).abs().max() < 3e-2


# ------------------------------------------------------------------ sampling

def _draw(z, temp, k, p, m, u, ld=None):
    T, V = z.shape
    f32 = lambda a: None if a is None else torch.tensor(np.asarray(a, np.float32), device=DEV)
    tok, prob, kept = (torch.full((T,), 77, device=DEV, dtype=d) for d in (torch.int32, torch.float32, torch.int32))
    dt = zb.ZO_BF16 if z.dtype == torch.bfloat16 else zb.ZO_F32
    need = zb.zo_sample_workspace_bytes(T, V, dt)
    ws = torch.full((max(need, 256),), 255, device=DEV, dtype=torch.uint8)
    zb.zo_sample(z, ld or z.stride(0), T, V, dt, f32(temp), None if k is None else _i32(k), f32(p), f32(m), f32(u), tok, prob, kept, ws,
                 need)
    return _np(tok), _np(prob), _np(kept)


def _check_draw(z, temp, k, p, m, u):
    got = _draw(z, temp, k, p, m, u)
    as32 = lambda a: None if a is None else np.asarray(a, np.float32).astype(np.float64)
    want = od.sample(_np(z), as32(temp), k, as32(p), as32(m), as32(u))
    assert (got[2] == want[2]).all(), (got[2], want[2])
    assert (got[0] == want[0]).all(), (got[0], want[0])
    np.testing.assert_allclose(got[1], want[1], rtol=U + 1e-11, atol=1e-38)


SIZES = [(1, 1), (3, 2), (5, 17), (4, 255), (4, 256), (4, 257), (7, 1000), (2, 1023), (3, 5003), (2, 50272), (1, 151936)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", SIZES)
def test_sample_filters(dtype, T, V):
    rng = np.random.default_rng(V + T)
    rows = 8 * T if V < 20000 else 8                  # every combination of filters
    z = torch.from_numpy(rng.normal(size=(rows, V)) * 2.5).to(DEV).to(TT[dtype])
    temp, u = rng.uniform(0.3, 1.5, rows), rng.uniform(size=rows)
    k = np.where(np.arange(rows) & 1, rng.integers(1, V + 2, rows), 0)
    p = np.where(np.arange(rows) & 2, rng.uniform(0.1, 1.0, rows), 1.0)
    m = np.where(np.arange(rows) & 4, rng.uniform(0, 0.3, rows), 0.0)
    _check_draw(z, temp, k, p, m, u)
    _check_draw(z, temp, None, None, None, u)
    _check_draw(z, temp * 0, k, p, m, u)
    _check_draw(z, temp, None, p, None, u)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_ties_and_masks(dtype):
    rng = np.random.default_rng(9)
    V, T = 3001, 24
    z = np.round(rng.normal(size=(T, V)) * 2) / 2     # a dozen values
    z[1] = 0.25                                       # one value
    z[2] = -np.inf
    z[3, 5:] = -np.inf
    z[4] = np.finfo(np.float32).min                   # a mask of the type's lowest value over everything
    z[5, ::2] = np.finfo(np.float32).min
    z[6, 100:] = np.nan
    z[7] = np.nan
    z[8, 77] = np.inf
    z[9, [3, 2000]] = np.inf
    z[10, ::2] = 0.0
    z[10, 1::2] = -0.0
    z[11, 17] = 1e30
    z[12] = -1e30
    z[13] = np.linspace(-40, 40, V)
    z[14] = -np.linspace(0, 200, V)                   # weights down to nothing
    zt = torch.from_numpy(z).to(DEV).to(TT[dtype])
    u = rng.uniform(size=T)
    temp = rng.uniform(0.5, 1.5, T)
    for k, p, m in ((None, None, None), (rng.integers(1, 900, T), None, None), (None, rng.uniform(0.05, 0.999, T), None),
                    (None, None, rng.uniform(0, 1, T)), (rng.integers(1, 3100, T), rng.uniform(0.3, 1, T), rng.uniform(0, 0.1, T)),
                    (np.ones(T, int), np.zeros(T), np.ones(T)), (np.full(T, -3), np.full(T, np.nan), np.full(T, np.nan)),
                    (np.full(T, 5000), np.full(T, 2.0), np.full(T, -1.0)), (None, np.full(T, -1.0), np.full(T, 7.0))):
        _check_draw(zt, temp, k, p, m, u)


def test_sample_extreme_uniforms_and_temperatures():
    rng = np.random.default_rng(10)
    z = torch.from_numpy(rng.normal(size=(12, 700)) * 3).to(DEV).float()
    temp = [1, 1, 1, 1, 1, 1e-4, 1e-30, 1e4, 1e30, -1, np.nan, 0.5]
    u = [0, 1, 2, -1, np.nan, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 1 - 2 ** -24]
    _check_draw(z, temp, None, None, None, u)
    _check_draw(z, temp, [40] * 12, [0.9] * 12, [0.01] * 12, u)


@pytest.mark.parametrize("dtype,pad", [("bf16", 1), ("bf16", 3), ("f32", 1), ("f32", 4)])
def test_sample_rows_of_any_alignment(dtype, pad):
    rng = np.random.default_rng(pad)
    buf = torch.from_numpy(rng.normal(size=(5, 2047 + pad)) * 2).to(DEV).to(TT[dtype])
    z = buf[:, pad:]
    _check_draw(z, [1.0] * 5, [50] * 5, [0.9] * 5, None, rng.uniform(size=5))


@pytest.mark.parametrize("dtype,pad,V", [("bf16", 1, 9001), ("bf16", 2, 1023), ("f32", 3, 5121), ("f32", 2, 1022), ("f32", 1, 1 << 19),
                                         ("bf16", 3, 1 << 19)])
def test_sample_rows_that_begin_anywhere(dtype, pad, V):
    """Every row begins at another place of a 16-byte piece; what lies around a row must not be drawn."""
    rng = np.random.default_rng(V + pad)
    T = 4 if V > 10000 else 8
    buf = torch.full((T * (V + pad) + 8,), 1e9, device=DEV).to(TT[dtype])
    z = buf[pad:pad + T * (V + pad)].view(T, V + pad)[:, :V]
    z.copy_(torch.from_numpy(rng.normal(size=(T, V)) * 2))
    u = rng.uniform(size=T)
    u[0], u[-1] = 0.0, 1.0
    one = [1.0] * T
    _check_draw(z, one, None, None, None, u)
    _check_draw(z, one, [30] * T, None, None, u)
    _check_draw(z, one, None, [0.3] * T, None, u)
    _check_draw(z, one, None, [0.97] * T, None, u)
    _check_draw(z, one, None, None, [0.02] * T, u)
    _check_draw(z, [0.0] * T, None, None, None, u)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_results_do_not_depend_on_where_a_row_begins(dtype):
    """The same row at every place of a 16-byte piece, with a prefix that fits in LDS and one that does not: the same bits."""
    rng = np.random.default_rng(12)
    V, T = 30011, 8                                   # (an odd leading dimension: neighbouring rows begin at different places)
    row = rng.normal(size=V)
    z = torch.from_numpy(np.tile(row, (T, 1))).to(DEV).to(TT[dtype])
    assert z.stride(0) == V
    for u in rng.uniform(size=6):
        for k, p, m in ((None, None, None), (None, [0.9] * T, None), (None, [0.2] * T, None), ([6000] * T, [0.95] * T, None),
                        ([40] * T, [0.9] * T, None), (None, None, [0.01] * T)):
            tok, prob, kept = _draw(z, [0.9] * T, k, p, m, [u] * T)
            assert len(set(tok)) == len(set(prob)) == len(set(kept)) == 1


def test_sample_draws_every_kept_token_in_proportion():
    V, T = 300, 4096
    rng = np.random.default_rng(4)
    row = rng.normal(size=V) * 2
    z = torch.from_numpy(np.tile(row, (T, 1))).to(DEV).float()
    u = (np.arange(T) + 0.5) / T
    tok, prob, kept = _draw(z, [1.0] * T, [20] * T, None, None, u)
    idx, w = od.kept_tokens(_np(z[0]), 1.0, 20, 1.0, 0.0)
    freq = np.bincount(tok, minlength=V)
    assert set(np.nonzero(freq)[0]) <= set(idx)
    np.testing.assert_allclose(freq[idx] / T, w / w.sum(), atol=1.01 / T)       # a stratified sample is off by less than one


def test_sample_optional_outputs():
    z = torch.randn(3, 100, device=DEV)
    one = torch.ones(3, device=DEV)
    tok = torch.empty(3, device=DEV, dtype=torch.int32)
    need = zb.zo_sample_workspace_bytes(3, 100, zb.ZO_F32)
    ws = torch.empty(max(need, 256), device=DEV, dtype=torch.uint8)
    zb.zo_sample(z, 100, 3, 100, zb.ZO_F32, one, None, None, None, one * 0.3, tok, None, None, ws, need)
    assert (_np(tok) == od.sample(_np(z), [1.0] * 3, None, None, None, [np.float32(0.3)] * 3)[0]).all()


# ------------------------------------------------------------------ embedding rows

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,pad", [(1, 0), (7, 1), (64, 8), (1000, 0), (4096, 0), (5120, 8), (8200, 3)])
def test_embed_rows(dtype, d, pad):
    rng = np.random.default_rng(d)
    dev = lambda *s: torch.from_numpy(rng.normal(size=s)).to(DEV).to(TT[dtype])
    E, Ep = dev(50, d + pad), dev(20, d + 2 * pad)
    tok = np.array([0, 49, -1, 50, 7, 7, 1 << 30, -(1 << 31), 3], np.int32)
    pos = np.array([0, 19, 3, 20, -1, 5, 2 ** 31 - 1, 6, 19], np.int32)
    for table in (None, Ep):
        for alias in (False, True):
            d_tok, d_pos = _i32(tok), _i32(pos)
            nxt = d_pos if alias else torch.zeros_like(d_pos)
            X = torch.full((9, d + pad), 7.0, device=DEV, dtype=TT[dtype])
            zb.zo_embed_rows(d_tok, d_pos, 9, E, d + pad, 50, table, 0 if table is None else d + 2 * pad, 0 if table is None else 20, d,
                             ZT[dtype], X, d + pad, nxt)
            want = od.embed_rows(tok, pos, _np(E)[:, :d], None if table is None else _np(table)[:, :d], dtype)
            assert (_np(X)[:, :d] == want).all() and (_np(X)[:, d:] == 7).all()
            assert (_np(nxt) == (pos.astype(np.int64) + 1).astype(np.int32)).all()
    X = torch.empty(9, d, device=DEV, dtype=TT[dtype])
    zb.zo_embed_rows(_i32(tok), None, 9, E, d + pad, 50, None, 0, 0, d, ZT[dtype], X, d, None)
    assert (_np(X) == od.embed_rows(tok, pos, _np(E)[:, :d], None, dtype)).all()


# ------------------------------------------------------------------ streams and graphs

def test_captured_steps_replay_and_another_stream():
    """Append, attention and the draw of one step, captured once and replayed over tables and lengths that change in place,
    with eager work between; two graphs with workspaces of their own in turn."""
    H, g, dh, P = 8, 2, 128, 16
    s = Setup(21, "bf16", H, g, dh, P, [1] * 4, [5, 300, 700, 40], width=80)
    V = 5000
    z = torch.randn(4, V, device=DEV) * 2
    temp, u, k = torch.ones(4, device=DEV), torch.rand(4, device=DEV), _i32([0, 10, 0, 50])
    p = torch.tensor([1.0, 0.9, 0.8, 1.0], device=DEV)
    need = zb.zo_sample_workspace_bytes(4, V, zb.ZO_F32)
    side = torch.cuda.Stream(device=DEV)
    graphs = []
    for _ in range(2):
        q2, out = torch.empty(4, H * dh, device=DEV, dtype=torch.bfloat16), torch.empty(4, H * dh, device=DEV, dtype=torch.bfloat16)
        tok, prob = torch.empty(4, device=DEV, dtype=torch.int32), torch.empty(4, device=DEV)
        ws_a, ws_s = s.workspace(), torch.empty(max(need, 256), device=DEV, dtype=torch.uint8)

        def step(stream, q2=q2, out=out, tok=tok, prob=prob, ws_a=ws_a, ws_s=ws_s):
            s.append(None, None, 1e4, out=q2, stream=stream)
            zb.zo_attention_paged(s.batch, q2, H * dh, H, 0.09, s.cache, out, H * dh, ws_a[0], ws_a[1], stream)
            zb.zo_sample(z, V, 4, V, zb.ZO_F32, temp, k, p, None, u, tok, prob, None, ws_s, need, stream)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(torch.cuda.current_stream())
        graphs.append((graph, step, out, tok, prob))
    for n in range(6):
        kv = [5 + n, 256 * (n + 1) - n % 2, 700 + n, 16 * n + 1]
        s.d_kv.copy_(_i32(kv))
        s.table[:] = s.rng.permutation(s.n_pages)[np.arange(4 * 80).reshape(4, 80) % s.n_pages]
        s.d_table.copy_(_i32(s.table))
        z.normal_()
        u.uniform_()
        torch.cuda.synchronize()
        graph, step, out, tok, prob = graphs[n % 2]
        K0, V0 = s.K.clone(), s.V.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, tok, prob, s.K, s.V)]
        s.K.copy_(K0)
        s.V.copy_(V0)
        for x in (out, prob):
            x.fill_(3.0)
        tok.fill_(-5)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.synchronize()
        for a, b in zip(got, (out, tok, prob, s.K, s.V)):
            assert torch.equal(a, b), n
