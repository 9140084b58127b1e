"""A step loop that answers with the operators of a caller's own: the decoder's logits (mode 2), the 8-bit generator on the
attentional vectors, and rules on the logits."""

import numpy as np
import pytest
import torch

import workloads as W
from paper_1805_11462_amd import _lib, ops
from tests._gpu import translator_for
from tests.test_gpu_f8 import round8

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)


@pytest.mark.parametrize("wdtype,K", [("fp32", 3), ("bf16", 1)])
def test_logits_of_a_step(wdtype, K):
    w = W.Workload(**{**W.get("tiny").as_dict(), "wdtype": wdtype, "tgt_vocab": 1003})
    tr = translator_for(w, W.make_weights(w, peaked=True))
    src, lens = W.make_batch(w)
    B, S = src.shape
    ws = tr.encode(torch.from_numpy(src).cuda(), torch.from_numpy(lens).cuda())
    st = tr.decode_init(ws, B, S, K)
    tok = torch.full((B * K,), W.BOS_ID, dtype=torch.int32, device="cuda")
    full = tr.decode_step(ws, B, S, K, st, tok, mode=0)
    top = tr.decode_step(ws, B, S, K, st, tok, mode=1)
    raw = tr.decode_step(ws, B, S, K, st, tok, mode=2)
    assert raw[2] is None and raw[3] is None
    for a, b in zip(tr.state_views(full[0], B * K), tr.state_views(raw[0], B * K)):
        assert torch.equal(a, b)
    # the same logits less their logsumexp: both lse are sums of V terms in fp32, off by less than 2^-18
    assert (raw[1] - full[3][:, None] - full[1]).abs().max() <= 2.0 ** -18 * (1 + full[1].abs().max())
    out, _, lse = ops.constrain(raw[1], mode=0)
    assert (lse - full[3]).abs().max() <= 2.0 ** -18 * (1 + lse.abs().max())
    assert (out - full[1]).abs().max() <= 2.0 ** -18 * (1 + full[1].abs().max())
    out, ids, lse = ops.constrain(raw[1], mode=1, K=K)
    assert torch.equal(ids, top[2])
    assert (out - top[1]).abs().max() <= 2.0 ** -18 * (1 + out.abs().max())
    tr.close()


def test_a_greedy_loop_with_rules():
    """Greedy decoding without repeated bigrams and under a mask, with the 8-bit product on the attentional vectors; every
    step checked against a plain implementation on the step's own vectors."""
    w = W.Workload(**{**W.get("tiny").as_dict(), "hidden": 132, "emb": 36, "tgt_vocab": 1200})
    weights = W.make_weights(w, peaked=True)
    tr = translator_for(w, weights)
    src, lens = W.make_batch(w)
    B, S = src.shape
    V, T = w.tgt_vocab, 8
    w8 = ops.F8Weights(torch.from_numpy(weights["W_s"]).cuda())
    b_s = torch.from_numpy(weights["b_s"]).cuda()
    history = torch.zeros(B, T, dtype=torch.int32, device="cuda")
    n = torch.zeros(B, dtype=torch.int32, device="cuda")
    bits = np.random.default_rng(2).integers(0, 1 << 32, (2, (V + 31) // 32), dtype=np.uint64).astype(np.uint32)
    mask = torch.from_numpy(bits.view(np.int32)).cuda()
    row = torch.tensor([0, 1, -1, 0], dtype=torch.int32, device="cuda")
    rules = ops.LogitRules(history=history, history_len=n, no_repeat_ngram=1, mask=mask, mask_row=row,
                           repetition=torch.full((B,), 1.5, device="cuda", dtype=torch.float32))
    ws = tr.encode(torch.from_numpy(src).cuda(), torch.from_numpy(lens).cuda())
    st = tr.decode_init(ws, B, S, 1)
    tok = torch.full((B,), W.BOS_ID, dtype=torch.int32, device="cuda")
    said = [[] for _ in range(B)]
    for t in range(T):
        st, model_logits, _, _, _ = tr.decode_step(ws, B, S, 1, st, tok, mode=2)
        feed = tr.state_views(st, B)[2]
        logits = w8.linear(feed, b_s)
        # the 8-bit product stands near the model's own generator: an e4m3 rounding of either side is off by 2^-4 at most
        size = feed.abs() @ torch.from_numpy(weights["W_s"]).cuda().abs().t()
        assert ((logits - model_logits).abs() <= 0.13 * size + 1e-4).all()
        logp, ids, lse = ops.constrain(logits, rules, mode=1, K=1)
        x = logits.double().cpu().numpy()
        for b in range(B):
            z = x[b].copy()
            z[said[b]] = -np.inf
            if int(row[b]) >= 0:
                v = np.arange(V)
                z[((bits[int(row[b])][v >> 5] >> (v & 31).astype(np.uint32)) & 1) == 0] = -np.inf
            want = int(np.argmax(z))
            assert int(ids[b, 0]) == want
            ref = z[want] - (z.max() + np.log(np.exp(z - z.max()).sum()))
            assert abs(float(logp[b, 0]) - ref) <= 2.0 ** -18 * (1 + abs(ref) + abs(z[want]))
            said[b].append(want)
        tok = ids[:, 0].contiguous()
        history[:, t] = tok
        n += 1
    assert all(len(set(s)) == T for s in said)
    tr.close()


def _log_softmax(y):
    top = y.max(axis=1, keepdims=True)
    return y - (top + np.log(np.exp(y - top).sum(axis=1, keepdims=True)))


def _model(wdtype="fp32", **kw):
    w = W.Workload(**{**W.get("tiny").as_dict(), "hidden": 136, "emb": 40, "tgt_vocab": 1500, "wdtype": wdtype, **kw})
    weights = W.make_weights(w, peaked=True)
    tr = translator_for(w, weights)
    return w, weights, tr, ops.F8Weights(torch.from_numpy(weights["W_s"]).cuda())


@pytest.mark.parametrize("wdtype,K,B", [("fp32", 3, 4), ("bf16", 1, 4), ("fp32", 5, 40)])
def test_steps_with_an_8_bit_generator(wdtype, K, B):
    """Every mode of a step against the definition in 64 bits on the step's own attentional vectors. Tolerance: sums of 136 exact
    products in fp32 (137 x 2^-24 of the products' sizes), then the softmax's 2^-18."""
    w, weights, tr, w8 = _model(wdtype, batch=B)
    src, lens = W.make_batch(w)
    S, N = src.shape[1], B * K
    ws = tr.encode(torch.from_numpy(src).cuda(), torch.from_numpy(lens).cuda())
    st = tr.decode_init(ws, B, S, K)
    tok = torch.full((N,), W.BOS_ID, dtype=torch.int32, device="cuda")
    own = tr.decode_step(ws, B, S, K, st, tok, mode=0)
    tr.set_generator(w8)
    full, top, raw = (tr.decode_step(ws, B, S, K, st, tok, mode=m) for m in (0, 1, 2))
    for other in (full, top, raw):
        for a, b in zip(tr.state_views(own[0], N), tr.state_views(other[0], N)):
            assert torch.equal(a, b)
    feed = round8(tr.state_views(raw[0], N)[2].cpu().numpy())
    wq = round8(weights["W_s"])
    y = feed @ wq.T + weights["b_s"].astype(np.float64)
    tol = (w.hidden + 1) * 2.0 ** -24 * (np.abs(feed) @ np.abs(wq).T) + 2.0 ** -24 * np.abs(y)
    assert (np.abs(raw[1].double().cpu().numpy() - y) <= tol).all()
    ref = _log_softmax(y)
    assert (np.abs(full[1].double().cpu().numpy() - ref) <= 2 * tol.max(axis=1, keepdims=True) + 2.0 ** -18 * (1 + np.abs(ref))).all()
    order = torch.sort(raw[1], dim=1, descending=True, stable=True)
    assert torch.equal(top[2], order.indices[:, :K].to(torch.int32))
    assert (top[1] - full[1].gather(1, order.indices[:, :K])).abs().max() <= 2.0 ** -18 * (1 + full[1].abs().max())
    tr.set_generator(None)
    again = tr.decode_step(ws, B, S, K, st, tok, mode=0)
    assert torch.equal(again[1], own[1])
    tr.close()


@pytest.mark.parametrize("beam,banned", [(1, ()), (4, ()), (3, (5, 17, 200))])
def test_searches_with_an_8_bit_generator(beam, banned):
    """A search is the external loop over steps: the same sums of log-probabilities, the same choices."""
    w, weights, tr, w8 = _model()
    tr.set_generator(w8)
    src, lens = W.make_batch(w)
    src_d, lens_d = torch.from_numpy(src).cuda(), torch.from_numpy(lens).cuda()
    B, S = src.shape
    T = 6
    buf = tr.search_buffers(B, S, beam, T, trace=True, banned=banned)
    tr.beam_search(src_d, lens_d, buf)
    slot, tok, cand = (buf[f"trace_{k}"].cpu().numpy() for k in ("slot", "tok", "cand"))
    steps = buf["trace_steps"].cpu().numpy()
    ws = tr.encode(src_d, lens_d)
    st = tr.decode_init(ws, B, S, beam)
    score = np.full((B, beam), -np.inf)
    score[:, 0] = 0.0
    prev = np.full((B, beam), W.BOS_ID)
    parent = None
    live = np.ones(B, bool)
    for t in range(T):
        st, logp, _, _, _ = tr.decode_step(ws, B, S, beam, st, torch.from_numpy(prev.reshape(-1).astype(np.int32)).cuda(), parent,
                                           mode=0)
        lp = logp.double().cpu().numpy().reshape(B, beam, -1)
        lp[:, :, list(banned)] = -np.inf
        both = score[:, :, None] + lp
        nparent = np.tile(np.arange(beam), (B, 1))
        for b in range(B):
            live[b] &= t < steps[b]
            if not live[b]:
                continue
            flat = np.argsort(-both[b].reshape(-1), kind="stable")[:beam]
            # the step's own fp32 log-probabilities: both sides add the same numbers but for the softmax's last bits
            assert np.allclose(cand[t, b], both[b].reshape(-1)[flat], rtol=0, atol=2.0 ** -17 * (t + 1) * 20)
            assert (tok[t, b] == flat % w.tgt_vocab).all() and (slot[t, b] == flat // w.tgt_vocab).all()
            n = 0
            score[b] = -np.inf
            for k in range(beam):
                if tok[t, b, k] == W.EOS_ID or t == T - 1:
                    continue
                score[b, n], prev[b, n], nparent[b, n] = cand[t, b, k], tok[t, b, k], slot[t, b, k]
                n += 1
        parent = torch.from_numpy((np.arange(B)[:, None] * beam + nparent).reshape(-1).astype(np.int32)).cuda()
    assert not set(banned) & set(tok[tok >= 0].tolist())
    tr.close()


def test_calls_without_an_8_bit_form():
    w, weights, tr, w8 = _model()
    with pytest.raises(ValueError):
        tr.set_generator(ops.F8Weights(torch.zeros(8, 136, device="cuda", dtype=torch.float32)))
    src, lens = W.make_batch(w)
    src_d, lens_d = torch.from_numpy(src).cuda(), torch.from_numpy(lens).cuda()
    B, S = src.shape
    buf = tr.search_buffers(B, S, 1, 4)
    sbuf = tr.score_buffers(B, S, 3)
    tr.set_generator(w8)
    with pytest.raises(_lib.OnmtError) as e:                   # allocated before: too small now
        tr.beam_search(src_d, lens_d, buf)
    assert e.value.code == _lib.ONMT_ESIZE
    tgt = torch.full((B, 3), 7, dtype=torch.int32, device="cuda")
    with pytest.raises(_lib.OnmtError) as e:
        tr.score(src_d, lens_d, tgt, torch.full((B,), 3, dtype=torch.int32, device="cuda"), sbuf)
    assert e.value.code == _lib.ONMT_EUNSUPPORTED
    tr.set_generator(None)
    tr.beam_search(src_d, lens_d, buf)
    tr.close()


def test_a_captured_step_with_an_8_bit_generator():
    w, weights, tr, w8 = _model(batch=6)
    tr.set_generator(w8)
    tr.lib.onmt_set_validation(tr.handle, 1)
    src, lens = W.make_batch(w)
    B, S = src.shape
    ws = tr.encode(torch.from_numpy(src).cuda(), torch.from_numpy(lens).cuda())
    st = tr.decode_init(ws, B, S, 2)
    tok = torch.full((2 * B,), W.BOS_ID, dtype=torch.int32, device="cuda")
    tr.decode_step(ws, B, S, 2, st, tok, mode=1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = tr.decode_step(ws, B, S, 2, st, tok, mode=1)
    for seed in range(4):
        tok.copy_(torch.randint(4, w.tgt_vocab, (2 * B,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32))
        graph.replay()
        want = tr.decode_step(ws, B, S, 2, st, tok, mode=1)
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
        torch.cuda.synchronize()
    tr.close()
