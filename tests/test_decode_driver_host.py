"""The decode driver's bookkeeping without a GPU: tensors on the host, and a library that notes the calls and does nothing."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2605_28760_amd import binding as zb
from paper_2605_28760_amd import workloads as wl
from paper_2605_28760_amd.runner import DecodeDriver, DeviceBatch, DeviceModel, DeviceWorkload


class Recorder:
    """Workspace queries are the library's own; every other call is noted and succeeds."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        fn = getattr(self.real, name)
        if name.endswith("_bytes"):
            return fn

        def call(*args):
            self.calls.append((name, args))
            return zb.ZO_OK
        return call


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder(zb.lib())
    monkeypatch.setattr(zb, "_lib", r)
    return r


def _workload(cfg=40, R_used=None):
    w = wl.decoder_model("dec-host", cfg, "bf16", 2, 256, 2, 1, 128, 384, 777, 1, False, 8, 1e-2, 32,
                         wl._pair_batch([33, 5, 64], [0, 1, 0], 2, [20, 1]), qwen=True)
    for l in w.layers:
        l.R_used = l.P.shape[1] if R_used is None else R_used
    return w


def test_prefill_leaves_everything_to_its_stream(recorder):
    """The lengths of the caches are set by a call on the stream that the appends run on, not by an operation of torch's."""
    dec = DecodeDriver(DeviceModel(DeviceWorkload(_workload(), "cpu")), 4, page_size=16)
    kv = dec.cache.kv_len
    kv.fill_(99)
    dec.prefill(0x1230)
    dec.step(0x1230)
    assert (kv == 99).all()
    assert all(args[-1] == 0x1230 for _, args in recorder.calls)
    names = [n for n, _ in recorder.calls]
    setting = [i for i, (n, args) in enumerate(recorder.calls) if n == "zo_embed_rows" and args[13] == kv.data_ptr()]
    assert len(setting) == 2 and setting[0] < names.index("zo_cache_append")
    pos = recorder.calls[setting[0]][1][1]
    at = (C.c_int32 * dec.S).from_address(pos)
    assert list(at) == [n - 1 for n in np.diff(dec.d.batch.host["cu"])]


@pytest.mark.parametrize("mirrors", [True, False])
def test_decode_rows_are_under_the_tensors_of_the_models_batch(recorder, mirrors):
    d = DeviceWorkload(_workload(), "cpu", host_mirrors=mirrors)
    d.batch.dir_seed_v = d.batch.dir_seed.clone()
    d.batch.struct.dir_seed_v = d.batch.dir_seed_v.data_ptr()
    dec = DecodeDriver(DeviceModel(d), 4, page_size=16)
    a, b = d.batch.struct, dec.rows.batch.struct
    for field in ("seq_cand", "cand_dir", "cand_sign", "dir_seed", "dir_seed_v", "n_seqs", "n_cands", "n_dirs", "host_seq_cand",
                  "host_cand_dir"):
        assert getattr(a, field) == getattr(b, field), field
    assert b.n_tokens == b.n_seqs == d.batch.S and list(dec.rows.batch.cu) == list(range(d.batch.S + 1))
    assert list((C.c_int32 * (d.batch.S + 1)).from_address(b.host_cu_seqlens)) == list(range(d.batch.S + 1))
    assert a.n_tokens == d.batch.T and d.batch.host["cu"][-1] == d.batch.T      # the model's batch is as it was


def test_workspaces_have_room_for_the_whole_banks(recorder):
    """A bank that is widened after the driver was built (up to its capacity) fits into what the driver passes."""
    d = DeviceWorkload(_workload(R_used=8), "cpu")
    dec = DecodeDriver(DeviceModel(d), 4, page_size=16)
    for l in d.layers:
        l.bank.R_used = l.bank.R_cap
    dec.prefill()
    dec.step()
    linears = [args for n, args in recorder.calls if n == "zo_probe_linear"]
    assert len(linears) == 2 * (len(d.layers) + 1)
    for args in linears:
        batch, bank = args[0]._obj, args[12]._obj if args[12] is not None else None
        need = zb.zo_probe_linear_workspace_bytes(batch.n_tokens, batch.n_seqs, batch.n_dirs, args[6], args[7], args[9],
                                                  bank.R_used if bank else 0, args[8])
        assert args[18] >= need, (batch.n_tokens, args[6], args[7], args[18], need)


def test_another_batch_has_the_models_sequences(recorder):
    w = _workload()
    model = DeviceModel(DeviceWorkload(w, "cpu"))
    b = model.d.batch
    make = lambda cu, seq_cand: DeviceBatch(cu, seq_cand, b.host["cand_dir"], w.cand_sign, w.dir_seed, "cpu")
    for cu, sc in ((b.host["cu"] + (np.arange(b.S + 1) == 1), b.host["seq_cand"]), (b.host["cu"][:-1], b.host["seq_cand"][:-1])):
        with pytest.raises(ValueError, match="sequences"):
            DecodeDriver(model, 4, page_size=16, batch=make(cu, sc))
    other = make(b.host["cu"], b.host["seq_cand"])
    dec = DecodeDriver(model, 4, page_size=16, batch=other)
    dec.prefill()
    dec.step()
    seeds = {args[0]._obj.dir_seed for n, args in recorder.calls if n == "zo_probe_linear" and args[0]._obj.n_dirs}
    assert seeds == {other.dir_seed.data_ptr()} and model.d.batch is b


def test_blocks_share_what_one_of_them_uses_at_a_time(recorder):
    """One buffer of queries and one attention workspace for all blocks' steps; prompts run in the model's activations."""
    model = DeviceModel(DeviceWorkload(_workload(), "cpu"))
    dec = DecodeDriver(model, 4000, page_size=16)
    dec.prefill()
    dec.step()
    attend = [args for n, args in recorder.calls if n == "zo_attention_paged"]
    assert len(attend) == 2 and len({(a[1], a[8]) for a in attend}) == 1
    for a in attend:
        need = zb.zo_attention_paged_workspace_bytes(dec.S, 2, 128, dec.cache.max_len, zb.ZO_BF16)
        assert need > 256 and a[9] >= need
    for own, prompt in zip(model.blocks, dec.prompt_blocks):
        assert all(getattr(own, n) is getattr(prompt, n) for n in ("a1", "h1", "a2", "h2", "att", "g1", "gq", "h0"))
        assert own.d is model.d and prompt.d is dec.prompts
    assert len({b.h1.data_ptr() for b in dec.blocks}) == 2 and dec.blocks[0].h1.shape[0] == dec.S


def test_make_cache_takes_pools_of_the_stated_type_alone():
    """A pool of two-byte values under a four-byte type would be read behind its end; lengths in floats are no lengths."""
    K, V = torch.zeros(4, 2, 16, 8), torch.zeros(4, 2, 16, 8)
    table, kv = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    assert zb.make_cache(K, V, zb.ZO_F32, table, kv).head_dim == 8
    assert zb.make_cache(K.bfloat16(), V.bfloat16(), zb.ZO_BF16, table, kv).head_dim == 8
    for k, v, dt, t, n in ((K.bfloat16(), V.bfloat16(), zb.ZO_F32, table, kv), (K, V, zb.ZO_BF16, table, kv),
                           (K.half(), V.half(), zb.ZO_BF16, table, kv), (K, V, zb.ZO_F32, table.float(), kv),
                           (K, V, zb.ZO_F32, table, kv.float()), (K[0], V[0], zb.ZO_F32, table, kv), (K, V, zb.ZO_F32, kv, kv)):
        with pytest.raises(ValueError):
            zb.make_cache(k, v, dt, t, n)
