"""The decode driver on streams given as arguments, under candidates that change after it was built, and with banks that grow."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2605_28760_amd import workloads as wl
from paper_2605_28760_amd.runner import DecodeDriver, DeviceBatch, DeviceModel, DeviceWorkload
from test_gpu_decode_loop import DEV, _model


def _answer(dec, steps=4, stream=None):
    """Logits and tokens of prompts and steps, and the caches, with fixed uniforms."""
    out = []
    for n in range(steps):
        torch.cuda.synchronize()
        dec.u.fill_(0.15 + 0.2 * n)
        torch.cuda.synchronize()
        dec.prefill(stream) if n == 0 else dec.step(stream)
        torch.cuda.synchronize()
        out += [dec.logits.clone(), dec.tokens.clone()]
    return out + [dec.cache.kv_len.clone()]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_prefill_on_a_stream_of_its_own():
    """Only the stream that is passed orders the call: work that is waiting on the current one does not come into it."""
    w = _model("bf16", True, 70)
    new = lambda: DecodeDriver(DeviceModel(DeviceWorkload(w, DEV)), 12, temperature=0.8, top_k=40, page_size=16)
    want = _answer(new())
    dec, side = new(), torch.cuda.Stream(device=DEV)
    x = torch.randn(8192, 8192, device=DEV)
    dec.u.fill_(0.15)
    torch.cuda.synchronize()
    for _ in range(8):
        y = x @ x                                # the current stream is busy for tens of milliseconds
    dec.prefill(side)
    got = []
    for n in range(4):
        if n:
            dec.step(side)
        side.synchronize()
        with torch.cuda.stream(side):
            got += [dec.logits.clone(), dec.tokens.clone()]
            dec.u.fill_(0.15 + 0.2 * (n + 1))
    side.synchronize()
    assert _same(got, want[:-1])
    with torch.cuda.stream(side):                # and a second answer after the first, inside the stream's context
        dec.u.fill_(0.15)
        dec.prefill(side)
        first = dec.logits.clone()
        dec.step(side)
        kv = dec.cache.kv_len.clone()
    side.synchronize()
    assert torch.equal(first, want[0]) and torch.equal(kv, want[-1] - 2)
    torch.cuda.synchronize()
    del y


def test_steps_follow_the_candidates_that_the_batch_holds():
    """Seeds and signs written to the model's batch after the driver was built reach prompts and steps alike."""
    w = _model("bf16", True, 71)
    d = DeviceWorkload(w, DEV)
    dec = DecodeDriver(DeviceModel(d), 6, temperature=0.0, page_size=16)
    before = _answer(dec)
    w2 = _model("bf16", True, 71)
    w2.dir_seed = w.dir_seed + np.uint64(1000)
    w2.cand_sign = -w.cand_sign
    d.batch.dir_seed.copy_(torch.from_numpy(w2.dir_seed.view(np.int64)))
    d.batch.cand_sign.copy_(torch.from_numpy(w2.cand_sign))
    got = _answer(dec)
    assert _same(got, _answer(DecodeDriver(DeviceModel(DeviceWorkload(w2, DEV)), 6, temperature=0.0, page_size=16)))
    assert not torch.equal(got[0], before[0]) and not torch.equal(got[2], before[2])


def test_a_bank_that_grows_after_the_driver_was_built():
    w = _model("bf16", True, 72)
    for l in w.layers:
        l.R_used = 16
    d = DeviceWorkload(w, DEV)
    dec = DecodeDriver(DeviceModel(d), 6, temperature=0.0, page_size=16)
    for l in d.layers:
        l.bank.R_used = l.bank.R_cap
    got = _answer(dec)
    w2 = _model("bf16", True, 72)
    for l in w2.layers:
        l.R_used = l.P.shape[1]
    assert _same(got, _answer(DecodeDriver(DeviceModel(DeviceWorkload(w2, DEV)), 6, temperature=0.0, page_size=16)))


def test_answers_under_another_batch_of_candidates():
    """A batch of the same sequences with candidates of its own (two seeds per direction): prompts and steps run under it."""
    w = _model("bf16", True, 73)
    d = DeviceWorkload(w, DEV)
    b = d.batch
    seeds = w.dir_seed + np.uint64(5)
    other = DeviceBatch(b.host["cu"], b.host["seq_cand"], b.host["cand_dir"], w.cand_sign, w.dir_seed, DEV, dir_seed_v=seeds)
    got = _answer(DecodeDriver(DeviceModel(d), 6, temperature=0.0, page_size=16, batch=other))
    d2 = DeviceWorkload(w, DEV)
    d2.batch = other
    want = _answer(DecodeDriver(DeviceModel(d2), 6, temperature=0.0, page_size=16))
    assert _same(got, want)
    own = _answer(DecodeDriver(DeviceModel(d), 6, temperature=0.0, page_size=16))
    assert not torch.equal(got[0], own[0]) and not torch.equal(got[2], own[2])
