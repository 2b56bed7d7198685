"""The decode loop of a whole model (prompts into the caches, then token by token, every sequence under its own candidate)
against the oracle, which runs the whole sequence from its first token at every step, and against itself.

Tolerances: hidden rows as in the whole-model scoring tests (fp32 1e-4 of max(|value|, rms) after two blocks, bf16 4e-2);
logits one product further (bf16 5e-2); tokens are exact for the device's own logits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from oracle import zo_block as ob
from oracle import zo_decode as od
from paper_2605_28760_amd import workloads as wl
from paper_2605_28760_amd.runner import DecodeDriver, DeviceModel, DeviceWorkload
from zo_testlib import assert_close, oracle_batch, to_np

DEV = "cuda:0"


def _model(dtype, qwen, cfg):
    batch = wl._pair_batch([33, 5, 64], [0, 1, 0], 2, [20, 1])
    if dtype == "f32":
        return wl.decoder_model("dec-f32", cfg, "f32", 2, 96, 4, 2, 24, 160, 211, 1 if qwen else 0, not qwen, 4, 1e-2, 8, batch, qwen=qwen)
    return wl.decoder_model("dec-bf16", cfg, "bf16", 2, 256, 2, 1, 128, 384, 777, 1 if qwen else 0, not qwen, 8, 1e-2, 32, batch, qwen=qwen)


def _oracle_last(w, rows_of):
    """Final rows of the last position of every sequence, the sequences run whole from their rows."""
    cu = np.concatenate([[0], np.cumsum([len(r) for r in rows_of])])
    batch = oracle_batch(w)
    batch.cu_seqlens = cu.astype(np.int32)
    h = np.concatenate(rows_of)
    for blk in w.meta["blocks"]:
        h = ob.block_forward(batch, h, blk, w.r, w.eps, w.dtype)["h2"]
    gf, bf = w.meta["final_norm"]
    last = w.meta["blocks"][-1]
    _, fin = ob.add_norm(h, None, gf, bf, last.norm_kind, last.norm_eps, w.dtype)
    return fin[cu[1:] - 1]


@pytest.mark.parametrize("dtype,qwen", [("f32", True), ("f32", False), ("bf16", True), ("bf16", False)])
def test_decode_matches_whole_sequences(dtype, qwen):
    w = _model(dtype, qwen, 90 + qwen)
    d = DeviceWorkload(w, DEV)
    rng = np.random.default_rng(7)
    hidden, vocab = w.X.shape[1], w.head.shape[0]
    draw = lambda *s: wl.as_bf16_values(rng.normal(size=s)) if dtype == "bf16" else rng.normal(size=s).astype(np.float32)
    E, Ep = draw(vocab, hidden), None if qwen else draw(100, hidden) * np.float32(0.25)
    up = lambda a: None if a is None else torch.from_numpy(a).to(DEV).to(d.head.dtype)
    S = d.batch.S
    k = rng.integers(0, 60, S)
    p = rng.uniform(0.5, 1.0, S).astype(np.float32)
    temp = np.where(np.arange(S) == 1, 0.0, rng.uniform(0.5, 1.2, S)).astype(np.float32)
    dec = DecodeDriver(DeviceModel(d), 12, up(E), up(Ep), temp, k, p, 0.01, page_size=16)
    rows = [w.X[a:b].astype(np.float64) for a, b in zip(w.cu_seqlens[:-1], w.cu_seqlens[1:])]
    rtol = 1e-4 if dtype == "f32" else 4e-2
    for n in range(5):
        u = rng.uniform(size=S).astype(np.float32)
        dec.u.copy_(torch.from_numpy(u))
        if n == 0:
            dec.prefill()
        else:
            tok = to_np(dec.tokens)
            new = od.embed_rows(tok, to_np(dec.cache.kv_len), E.astype(np.float64), None if Ep is None else Ep.astype(np.float64), dtype)
            rows = [np.concatenate([r, x[None]]) for r, x in zip(rows, new)]
            dec.step()
        torch.cuda.synchronize()
        assert (to_np(dec.cache.kv_len) == [len(r) for r in rows]).all()
        want = _oracle_last(w, rows)
        final = to_np(dec.prompt_last if n == 0 else dec.final)
        assert_close(final, want, rtol, "final rows of step %d" % n)
        assert_close(to_np(dec.logits), final.astype(np.float64) @ w.head.astype(np.float64).T, 1e-4 if dtype == "f32" else 5e-2, "logits")
        f64 = lambda a: a.astype(np.float64)
        tok, prob, kept = od.sample(to_np(dec.logits).astype(np.float64), f64(temp), k, f64(p), np.full(S, np.float32(0.01), np.float64), f64(u))
        assert (to_np(dec.tokens) == tok).all() and (to_np(dec.n_kept) == kept).all()
        np.testing.assert_allclose(to_np(dec.prob), prob, rtol=1e-6)


def test_candidates_answer_under_their_own_weights_and_foreground_rows_under_the_base():
    w = _model("bf16", True, 93)
    runs = []
    for work in (w, wl.foreground_only(w)):
        dec = DecodeDriver(DeviceModel(DeviceWorkload(work, DEV)), 4, temperature=0.0, page_size=32)
        dec.prefill()
        first = dec.logits.clone()
        dec.tokens.copy_(torch.arange(dec.S, dtype=torch.int32))     # (the same tokens on both sides)
        dec.step()
        torch.cuda.synchronize()
        runs.append((first, dec.logits.clone()))
    fg = torch.from_numpy(w.seq_cand < 0).to(DEV)
    for a, b in zip(*runs):
        assert torch.equal(a[fg], b[fg])                             # bit for bit
        assert not torch.equal(a[~fg], b[~fg])
    a = runs[0][1]
    assert not torch.equal(a[0], a[1])                               # + and - of one example


def test_captured_steps_equal_eager_steps():
    def run(graph):
        w = _model("bf16", True, 94)
        dec = DecodeDriver(DeviceModel(DeviceWorkload(w, DEV)), 12, temperature=0.8, top_k=40, top_p=0.9, page_size=16)
        if graph:
            dec.prefill()
            dec.capture()
        gen = torch.Generator(device=DEV)
        gen.manual_seed(3)
        out = []
        dec.u.uniform_(generator=gen)
        dec.prefill()
        for n in range(6):
            out.append((dec.tokens.clone(), dec.prob.clone(), dec.logits.clone()))
            dec.u.uniform_(generator=gen)
            if graph:
                dec.replay()
                torch.randn(1 << 16, device=DEV).sum()               # unrelated eager work between replays
            else:
                dec.step()
            torch.cuda.synchronize()
        return out + [(dec.tokens, dec.prob, dec.logits, dec.cache.kv_len, *dec.cache.K)]
    for n, (a, b) in enumerate(zip(run(False), run(True))):
        for x, y in zip(a[:4], b[:4]):
            assert torch.equal(x, y), n


def test_driver_refusals():
    batch = wl._pair_batch([3], [0])
    w = wl.decoder_model("dec-empty", 95, "f32", 1, 32, 2, 1, 16, 32, 50, 1, False, 4, 1e-3, 8, batch)
    w.cu_seqlens = np.array([0, 0, 6], np.int32)
    with pytest.raises(ValueError, match="prompt"):
        DecodeDriver(DeviceModel(DeviceWorkload(w, DEV)), 2)
    w.cu_seqlens = np.array([0, 3, 6], np.int32)
    model = DeviceModel(DeviceWorkload(w, DEV))
    for bad in (torch.zeros(50, 32, device=DEV).bfloat16(), torch.zeros(50, 31, device=DEV), torch.zeros(32, 50, device=DEV).t()):
        with pytest.raises(ValueError, match="embed"):
            DecodeDriver(model, 2, bad)
        with pytest.raises(ValueError, match="positions"):
            DecodeDriver(model, 2, None, bad)
