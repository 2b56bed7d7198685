"""Host side of the decode entry points, without a GPU: refusals before any device work, workspace queries, and the
same code under AddressSanitizer and UndefinedBehaviorSanitizer with stub launchers."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2605_28760_amd import binding as zb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000   # a non-NULL, 4 KiB aligned "device pointer" that is never dereferenced


def _status(fn, *a, **k):
    with pytest.raises(zb.ZoError) as e:
        fn(*a, **k)
    return e.value.status


def _batch(lens=(1, 1), mirrors=True):
    cu = np.zeros(len(lens) + 1, np.int32)
    cu[1:] = np.cumsum(lens)
    return zb.make_batch(int(cu[-1]), FAKE, FAKE, None, None, None, cu if mirrors else None, n_seqs=len(lens), n_cands=0,
                         n_dirs=0)


def _cache(**k):
    c = zb.zo_cache()
    for f, v in dict(n_pages=8, page_size=16, n_kv_heads=2, head_dim=128, dtype=zb.ZO_BF16, max_pages=4, K=FAKE, V=FAKE,
                     page_table=FAKE, kv_len=FAKE, host_page_table=None, host_kv_len=None).items():
        setattr(c, f, k.get(f, v))
    return c


CACHE_REFUSALS = [(dict(dtype=5), zb.ZO_ERR_UNSUPPORTED), (dict(n_pages=0), zb.ZO_ERR_SHAPE), (dict(max_pages=0), zb.ZO_ERR_SHAPE),
                  (dict(n_kv_heads=0), zb.ZO_ERR_SHAPE), (dict(page_size=8), zb.ZO_ERR_UNSUPPORTED),
                  (dict(page_size=48), zb.ZO_ERR_UNSUPPORTED), (dict(page_size=2048), zb.ZO_ERR_UNSUPPORTED),
                  (dict(max_pages=1 << 27), zb.ZO_ERR_SHAPE), (dict(K=None), zb.ZO_ERR_NULL), (dict(V=FAKE + 8), zb.ZO_ERR_SHAPE),
                  (dict(page_table=None), zb.ZO_ERR_NULL), (dict(kv_len=None), zb.ZO_ERR_NULL)]


def _append(batch=None, cache=None, **k):
    zb.zo_cache_append(batch or _batch(), k.get("Q", FAKE), k.get("ldq", 1024), k.get("K", FAKE), k.get("ldk", 1024),
                       k.get("V", FAKE), k.get("ldv", 1024), k.get("H", 4), k.get("gq", FAKE), k.get("gk", FAKE),
                       k.get("eps", 1e-6), 1e6, cache or _cache(), k.get("Qout", FAKE + 4096), k.get("ldqo", 512))


def _attend(batch=None, cache=None, **k):
    zb.zo_attention_paged(batch or _batch(), k.get("Q", FAKE), k.get("ldq", 512), k.get("H", 4), 0.1, cache or _cache(),
                          k.get("O", FAKE), k.get("ldo", 512), k.get("ws", FAKE), k.get("wsb", 1 << 30))


@pytest.mark.parametrize("change,status", CACHE_REFUSALS)
@pytest.mark.parametrize("call", [_append, _attend])
def test_cache_refusals(call, change, status):
    assert _status(call, cache=_cache(**change)) == status


@pytest.mark.parametrize("call", [_append, _attend])
def test_host_copies_of_the_tables_are_checked(call):
    table = np.array([[0, 1, 2, 3], [4, 5, -1, -1]], np.int32)
    for kv, rows in (([0, 3], (1, 1)), ([5, 65], (1, 1)), ([5, -1], (1, 0))):
        kv = np.array(kv, np.int32)
        assert _status(call, _batch(rows), _cache(host_kv_len=kv.ctypes.data)) == zb.ZO_ERR_INDEX
    for kv, tb in (([64, 33], table), ([64, 32], np.where(table == 2, 8, table).astype(np.int32))):
        kv = np.array(kv, np.int32)
        assert _status(call, _batch(), _cache(host_kv_len=kv.ctypes.data, host_page_table=tb.ctypes.data)) == zb.ZO_ERR_INDEX
    assert "page_table" in zb.last_error()


def test_append_refusals():
    assert _status(_append, Q=None) == zb.ZO_ERR_NULL
    assert _status(_append, V=None) == zb.ZO_ERR_NULL
    assert _status(_append, Qout=None) == zb.ZO_ERR_NULL
    assert _status(_append, gk=None) == zb.ZO_ERR_NULL
    assert _status(_append, gq=FAKE + 2) == zb.ZO_ERR_SHAPE
    assert _status(_append, H=3) == zb.ZO_ERR_SHAPE
    assert _status(_append, H=0) == zb.ZO_ERR_SHAPE
    assert _status(_append, eps=-1.0) == zb.ZO_ERR_SHAPE
    assert _status(_append, ldq=256) == zb.ZO_ERR_SHAPE
    assert _status(_append, ldk=128) == zb.ZO_ERR_SHAPE
    assert _status(_append, ldqo=516) == zb.ZO_ERR_SHAPE
    assert _status(_append, Qout=FAKE, ldq=1024, ldqo=512) == zb.ZO_ERR_SHAPE        # in place, other rows
    assert _status(_append, cache=_cache(head_dim=127)) == zb.ZO_ERR_UNSUPPORTED
    assert _status(_append, cache=_cache(head_dim=258)) == zb.ZO_ERR_UNSUPPORTED
    _append(_batch(lens=(0, 0)), Q=None, K=None, V=None, Qout=None)                    # no rows: nothing is touched


def test_attention_paged_refusals():
    assert _status(_attend, Q=None) == zb.ZO_ERR_NULL
    assert _status(_attend, O=None) == zb.ZO_ERR_NULL
    assert _status(_attend, H=5) == zb.ZO_ERR_SHAPE
    assert _status(_attend, H=65536) == zb.ZO_ERR_SHAPE
    assert _status(_attend, ldo=516) == zb.ZO_ERR_SHAPE
    assert _status(_attend, Q=FAKE + 2) == zb.ZO_ERR_SHAPE
    assert _status(_attend, cache=_cache(head_dim=80)) == zb.ZO_ERR_UNSUPPORTED
    assert _status(_attend, cache=_cache(head_dim=264, dtype=zb.ZO_F32), ldq=2048, ldo=2048) == zb.ZO_ERR_UNSUPPORTED
    _attend(_batch(lens=(0, 0)), Q=None, O=None, ws=None, wsb=0)


def test_sample_refusals():
    def draw(**k):
        zb.zo_sample(k.get("z", FAKE), k.get("ld", 1000), k.get("T", 2), k.get("V", 1000), k.get("dt", zb.ZO_F32),
                     k.get("temp", FAKE), None, None, None, k.get("u", FAKE), k.get("tok", FAKE), None, None, k.get("ws", FAKE),
                     k.get("wsb", 1 << 30))
    assert _status(draw, z=None) == zb.ZO_ERR_NULL
    assert _status(draw, temp=None) == zb.ZO_ERR_NULL
    assert _status(draw, u=None) == zb.ZO_ERR_NULL
    assert _status(draw, tok=None) == zb.ZO_ERR_NULL
    assert _status(draw, T=-1) == zb.ZO_ERR_SHAPE
    assert _status(draw, V=0) == zb.ZO_ERR_SHAPE
    assert _status(draw, V=(1 << 19) + 1, ld=1 << 20) == zb.ZO_ERR_UNSUPPORTED
    assert _status(draw, ld=999) == zb.ZO_ERR_SHAPE
    assert _status(draw, z=FAKE + 2) == zb.ZO_ERR_SHAPE
    assert _status(draw, z=FAKE + 1, dt=zb.ZO_BF16) == zb.ZO_ERR_SHAPE
    assert _status(draw, dt=4) == zb.ZO_ERR_UNSUPPORTED
    draw(T=0, z=None)


def test_embed_rows_refusals():
    def emb(**k):
        zb.zo_embed_rows(k.get("tok", FAKE), k.get("pos", FAKE), k.get("T", 2), k.get("E", FAKE), k.get("lde", 64), 100,
                         k.get("Ep", FAKE), k.get("ldp", 64), 10, k.get("d", 64), k.get("dt", zb.ZO_BF16), k.get("X", FAKE),
                         k.get("ldx", 64), k.get("nxt", FAKE))
    assert _status(emb, tok=None) == zb.ZO_ERR_NULL
    assert _status(emb, pos=None) == zb.ZO_ERR_NULL
    assert _status(emb, pos=None, Ep=None) == zb.ZO_ERR_NULL
    assert _status(emb, E=None) == zb.ZO_ERR_NULL
    assert _status(emb, X=None) == zb.ZO_ERR_NULL
    assert _status(emb, T=-1) == zb.ZO_ERR_SHAPE
    assert _status(emb, lde=63) == zb.ZO_ERR_SHAPE
    assert _status(emb, ldp=63) == zb.ZO_ERR_SHAPE
    assert _status(emb, X=FAKE + 1) == zb.ZO_ERR_SHAPE
    assert _status(emb, dt=2) == zb.ZO_ERR_UNSUPPORTED
    emb(T=0, tok=None)


def test_calls_beyond_one_launch_are_refused():
    big = zb.make_batch((1 << 21) + 1, FAKE, FAKE, None, None, None, None, n_seqs=3, n_cands=0, n_dirs=0)
    assert _status(_append, big, _cache(n_kv_heads=8), H=8, ldq=4096, ldk=4096, ldv=4096, ldqo=4096) == zb.ZO_ERR_UNSUPPORTED
    assert _status(_attend, big) == zb.ZO_ERR_UNSUPPORTED
    assert _status(zb.zo_sample, FAKE, 10, (1 << 21) + 1, 10, zb.ZO_F32, FAKE, None, None, None, FAKE, FAKE, None, None, None, 0) == \
        zb.ZO_ERR_UNSUPPORTED
    assert _status(zb.zo_embed_rows, FAKE, None, (1 << 23) + 1, FAKE, 8, 10, None, 0, 0, 8, zb.ZO_F32, FAKE, 8, None) == zb.ZO_ERR_UNSUPPORTED


def test_make_cache_checks_its_tensors():
    torch = pytest.importorskip("torch")
    K = torch.zeros(4, 2, 16, 8)
    table, kv = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    c = zb.make_cache(K, K.clone(), zb.ZO_F32, table, kv)
    assert (c.n_pages, c.n_kv_heads, c.page_size, c.head_dim, c.max_pages) == (4, 2, 16, 8, 2)
    for bad in (dict(V=torch.zeros(4, 2, 16, 9)), dict(V=K.bfloat16()), dict(K=K.transpose(1, 2)), dict(table=table.long()),
                dict(kv=kv[:2]), dict(table=torch.zeros(2, 3, dtype=torch.int32).t())):
        with pytest.raises(ValueError):
            zb.make_cache(bad.get("K", K), bad.get("V", K), zb.ZO_F32, bad.get("table", table), bad.get("kv", kv))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_decode_host_code_under_sanitizers(tmp_path):
    san, csrc = os.path.join(ROOT, "tests", "abi_sanitize"), os.path.join(ROOT, "paper_2605_28760_amd", "csrc")
    exe = str(tmp_path / "decode_host_check")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-static-libasan", "-static-libubsan", "-D__HIP_PLATFORM_AMD__",
           "-I/opt/rocm/include", "-I" + csrc, os.path.join(csrc, "zo_abi.cpp"), os.path.join(csrc, "zo_decode_abi.cpp"),
           os.path.join(san, "launch_stubs.cpp"), os.path.join(san, "decode_stubs.cpp"),
           os.path.join(san, "decode_host_check.cpp"), "-o", exe]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert "0 failed" in run.stdout, run.stdout
