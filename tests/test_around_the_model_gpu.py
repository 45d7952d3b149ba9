"""The calls around a model as they are used together, without a read-back between them: documents -> ids (tt_encode_batch) -> blocks and
slots (tt_blocks_extend) -> a model that reads its cache through them -> scores of the same ids and their gradient; a conversation whose
append replaces the end of its tokens."""
import numpy as np
import pytest

import workloads as wl
from gpu_util import cpu_vocab, gpu_vocab, to_dev
from test_blocks import Pool
from test_logprobs import check_grad, check_scores

pytestmark = pytest.mark.gpu
BLOCK, WIDTH = 16, 120


def _documents(lengths, seed):
    docs = [wl.generate(wl.KIND_MIX_UNI, seed + i, n) if n else np.zeros(0, np.uint8) for i, n in enumerate(lengths)]
    return docs, np.r_[0, np.cumsum([d.size for d in docs])].astype(np.int64)


def test_batch_to_scores_and_gradient():
    import torch
    import paper_2607_29678_b200 as tt
    cfg = wl.CONFIGS["C1"]
    v, cv = gpu_vocab("C1"), cpu_vocab("C1")
    docs, doc_off = _documents([700, 0, 1, 350, 2_000, 33], 11)
    text = np.concatenate(docs)
    n_docs, vocab, dim = len(docs), 256 + cfg.n_merges, 32
    want = [cv.encode(d, cfg.pattern_id)[0] if d.size else np.zeros(0, np.int32) for d in docs]
    total = sum(w.size for w in want)
    cap = total + 40                                                       # room behind the last token, as a server's buffers have
    bufs = v.alloc(text.size, max_docs=n_docs)
    d_text, d_off = to_dev(text), torch.from_numpy(doc_off).cuda()
    state, maps = tt.alloc_blocks(n_docs, WIDTH, 500, cap)
    scores = tt.alloc_logprobs(cap, 4)
    gen = torch.Generator(device="cuda").manual_seed(4)
    emb, head = torch.randn((vocab, dim), generator=gen, device="cuda"), torch.randn((dim, vocab), generator=gen, device="cuda") * 0.4
    cache = torch.zeros((500 * BLOCK + 1, dim), device="cuda")              # its last row takes what has no slot
    grad_lp = torch.full((cap,), -1.0 / total, device="cuda")

    # nothing below waits for the device
    v.encode_batch(d_text, d_off, bufs)
    tt.blocks_extend(bufs["ids_off"], state, BLOCK, maps)
    ids = bufs["ids"][:cap].clamp(0, vocab - 1)
    rows = emb[ids.long()]
    slots = maps["slots"]
    cache.index_copy_(0, torch.where(slots >= 0, slots, 500 * BLOCK), rows)
    logits = (rows @ head).to(torch.bfloat16)
    tt.logprobs(logits, ids, scores, ids_off=bufs["ids_off"])
    grad = torch.full_like(logits, 3.0)
    tt.logprobs_grad(logits, ids, scores, grad_lp, grad, ids_off=bufs["ids_off"])
    torch.cuda.synchronize()

    assert int(bufs["status"]) == int(maps["status"]) == int(scores["status"]) == 0
    off = bufs["ids_off"].cpu().numpy()
    assert np.array_equal(off, np.r_[0, np.cumsum([w.size for w in want])]) and np.array_equal(bufs["ids"][:total].cpu().numpy(), np.concatenate(want))
    table = state["block_table"].cpu().numpy()
    for r, w in enumerate(want):                                           # the cache, read the way attention reads it
        place = np.arange(w.size)
        at = table[r, place // BLOCK].astype(np.int64) * BLOCK + place % BLOCK
        if w.size:
            assert np.array_equal(cache[torch.from_numpy(at).cuda()].cpu().numpy(), emb[torch.from_numpy(w).long().cuda()].cpu().numpy())
    before = {k: np.zeros_like(t.cpu().numpy()) for k, t in scores.items()}
    check_scores(logits, ids, scores, ids_off=bufs["ids_off"], untouched=before)
    check_grad(logits, ids, scores, grad_lp, None, grad, ids_off=bufs["ids_off"], untouched=np.full(tuple(grad.shape), 3.0))
    # the offsets that go with the scores in an answer: those of the longest document alone
    r = int(np.argmax([w.size for w in want]))
    ids_r = torch.from_numpy(want[r]).cuda()
    count = torch.tensor([want[r].size], dtype=torch.int64, device="cuda")
    b_off, c_off = (torch.empty(want[r].size + 1, dtype=torch.int32, device="cuda") for _ in range(2))
    v.spans(ids_r, count, docs[r].size, b_off, c_off, bufs["status"])
    torch.cuda.synchronize()
    assert int(bufs["status"]) == 0 and int(b_off[-1]) == docs[r].size


def test_conversation_keeps_what_an_append_kept():
    """An append replaces the last tokens of a session: the blocks behind the kept ones go back, the new tokens get slots."""
    import torch
    import paper_2607_29678_b200 as tt
    session = tt.Session(gpu_vocab("C1"), 60_000)
    state, maps = tt.alloc_blocks(1, 2_000, 1_500, 20_000)
    pool = Pool(state["block_table"].cpu().numpy(), np.zeros(1, np.int64), state["free_blocks"].cpu().numpy(), 1_500, BLOCK)
    old_ids, old_off = np.zeros(0, np.int32), np.zeros(1, np.int32)
    for turn in range(6):
        session.append(wl.generate(wl.KIND_MIX_UNI, 50 + turn, 900 + 211 * turn))
        ids, off, _ = session.records()
        ids, off = ids.cpu().numpy(), off.cpu().numpy()
        n = min(ids.size, old_ids.size)
        differ = np.flatnonzero((ids[:n] != old_ids[:n]) | (off[:n] != old_off[:n]))
        keep = int(differ[0]) if differ.size else n
        tt.blocks_release(torch.tensor([keep], dtype=torch.int32, device="cuda"), state, BLOCK, maps)
        tt.blocks_extend(torch.tensor([0, ids.size - keep], dtype=torch.int64, device="cuda"), state, BLOCK, maps)
        torch.cuda.synchronize()
        assert int(maps["status"]) == 0
        pool.release(np.array([keep]))
        slots, pos, _ = pool.extend([0, ids.size - keep])
        assert np.array_equal(maps["slots"].cpu().numpy()[:slots.size], slots) and np.array_equal(maps["positions"].cpu().numpy()[:pos.size], pos)
        assert int(state["seq_len"]) == ids.size and int(state["n_free"]) == pool.n_free
        blocks = -(-ids.size // BLOCK)
        assert np.array_equal(state["block_table"].cpu().numpy()[0, :blocks], pool.table[0, :blocks]) and len(set(pool.table[0, :blocks])) == blocks
        old_ids, old_off = ids, off


def test_a_smaller_batch_in_the_buffers_of_a_larger_one():
    """ids_off has room for more documents than the batch has: its end is the earlier batch's, and may ascend."""
    import torch
    import paper_2607_29678_b200 as tt
    cfg = wl.CONFIGS["C1"]
    v, cv = gpu_vocab("C1"), cpu_vocab("C1")
    docs, doc_off = _documents([300, 200, 150, 700, 90, 260], 31)
    bufs = v.alloc(int(doc_off[-1]), max_docs=len(docs))
    v.encode_batch(to_dev(np.concatenate(docs)), torch.from_numpy(doc_off).cuda(), bufs)
    torch.cuda.synchronize()
    cap = int(bufs["ids_off"][-1])
    few, few_off = _documents([120, 60], 71)
    v.encode_batch(to_dev(np.concatenate(few)), torch.from_numpy(few_off).cuda(), bufs)
    torch.cuda.synchronize()
    off = bufs["ids_off"].cpu().numpy()
    want = [cv.encode(d, cfg.pattern_id)[0] for d in few]
    assert np.array_equal(off[:3], np.r_[0, np.cumsum([w.size for w in want])]) and (np.diff(off) >= 0).all() and off[-1] == cap > off[2]
    n_vocab = 256 + cfg.n_merges
    ids = bufs["ids"][:cap].clamp(0, n_vocab - 1)
    logits = torch.randn((cap, n_vocab), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.bfloat16)
    scores = tt.alloc_logprobs(cap, 2)
    before = {k: np.zeros_like(t.cpu().numpy()) for k, t in scores.items()}
    tt.logprobs(logits, ids, scores, ids_off=bufs["ids_off"], n_docs=2)
    g, grad = torch.randn(cap, device="cuda"), torch.full_like(logits, 3.0)
    tt.logprobs_grad(logits, ids, scores, g, grad, ids_off=bufs["ids_off"], n_docs=2)
    torch.cuda.synchronize()
    assert int(scores["status"]) == 0
    check_scores(logits, ids, scores, ids_off=bufs["ids_off"][:3], untouched=before)
    check_grad(logits, ids, scores, g, None, grad, ids_off=bufs["ids_off"][:3], untouched=np.full(tuple(grad.shape), 3.0))
    tt.logprobs(logits, ids, scores, ids_off=bufs["ids_off"], n_docs=0)
    torch.cuda.synchronize()
    assert int(scores["status"]) == 0
    for off_, n in ((bufs["ids_off"], 7), (bufs["ids_off"], -1), (None, 0)):
        with pytest.raises(ValueError):
            tt.logprobs(logits, ids, scores, ids_off=off_, n_docs=n)
        with pytest.raises(ValueError):
            tt.logprobs_grad(logits, ids, scores, g, grad, ids_off=off_, n_docs=n)
