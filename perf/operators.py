"""The operators around the model that the token ids go to and come from, and the sizes they are used at.

``op`` names the operator; each works on device data as ``Vocab.encode_batch`` leaves it (packed ids, ``ids_off``) without a read-back:

  extend    ``blocks_extend``: new tokens of every request -> blocks from the free list, block table, slot and position of every token
  release   ``blocks_release``: tokens that a request keeps -> blocks that go back to the free list
  logprobs  ``logprobs``: logits and ids -> log probability, entropy, rank of the id, top alternatives
  grad      ``logprobs_grad``: gradients of those log probabilities and entropies -> gradient of the logits

Vocabularies are 256 byte tokens plus the merges of the stored tables (4,352 / 32,256 / 100,256 / 200,000), and odd sizes beside them
(a vocabulary with an added token).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
VOCABS = (4_352, 32_256, 100_256, 200_000)
MOST_LOGITS = 4_096 * 200_000
MOST_TOKENS = 20_000_000


def listed():
    return [
        # One step of one conversation: the sampled token with the five alternatives that an API answer shows.
        {"name": "logprobs 1 row", "op": "logprobs", "rows": 1, "vocab": 100_256, "type": "bf16", "top": 5, "docs": 0, "mask": "none", "scale": 1.0},
        # A decode step of a server, with twenty alternatives, at a temperature.
        {"name": "logprobs 64 rows top 20", "op": "logprobs", "rows": 64, "vocab": 200_000, "type": "bf16", "top": 20, "docs": 0, "mask": "none", "scale": 1.25},
        # Constrained decoding: a grammar leaves few entries of each row; one added token makes the row length odd.
        {"name": "logprobs 300 rows masked", "op": "logprobs", "rows": 300, "vocab": 32_257, "type": "fp16", "top": 3, "docs": 0, "mask": "inf", "scale": 1.0},
        # Logits that were left in 32 bits, scored over short packed documents.
        {"name": "logprobs 1000 fp32", "op": "logprobs", "rows": 1_000, "vocab": 100_256, "type": "fp32", "top": 1, "docs": 37, "mask": "none", "scale": 1.0},
        # Scoring packed documents: the training and evaluation pass, the largest one.
        {"name": "logprobs 4096 documents", "op": "logprobs", "rows": 4_096, "vocab": 200_000, "type": "bf16", "top": 0, "docs": 11, "mask": "none", "scale": 1.0},
        # The gradient of a few positions in 32 bits.
        {"name": "grad 7 rows fp32", "op": "grad", "rows": 7, "vocab": 4_352, "type": "fp32", "docs": 0, "entropy": True, "mask": "none", "scale": 1.0},
        # Policy gradients with an entropy term over sampled tokens, entries masked by the type's lowest value, an odd row length.
        {"name": "grad 1000 rows entropy", "op": "grad", "rows": 1_000, "vocab": 32_257, "type": "fp16", "docs": 0, "entropy": True, "mask": "low", "scale": 0.7},
        # Next-token training over packed documents.
        {"name": "grad 4096 documents", "op": "grad", "rows": 4_096, "vocab": 200_000, "type": "bf16", "docs": 11, "entropy": False, "mask": "none", "scale": 1.0},
        # A decode step: one more token for each of 256 conversations.
        {"name": "extend 256 decode", "op": "extend", "requests": 256, "tokens": 1, "cached": 4_000, "block": 16, "even": True},
        # Ingestion of the 256 long requests of the batch benchmark: some 23 million tokens.
        {"name": "extend 256 long", "op": "extend", "requests": 256, "tokens": 90_000, "cached": 0, "block": 64, "even": False},
        # A thousand conversations, each with a new message of its own length.
        {"name": "release 1000 messages", "op": "release", "requests": 1_000, "tokens": 230, "cached": 900, "block": 16, "even": False},
        # The long requests end: all their blocks go back.
        {"name": "release 256 long", "op": "release", "requests": 256, "tokens": 90_000, "cached": 0, "block": 16, "even": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("logprobs", "logprobs", "grad", "extend", "release"))
    if op in ("logprobs", "grad"):
        c = {"op": op, "vocab": rng.choice(VOCABS) + rng.choice((0, 1, 5)) if rng.random() < 0.6 else _log_uniform(rng, 500, 200_000), "type": rng.choice(tuple(TYPES))}
        c["rows"] = _log_uniform(rng, 1, min(4_096, MOST_LOGITS // c["vocab"] // (2 if c["type"] == "fp32" else 1)))
        c["docs"] = rng.randint(1, max(1, c["rows"] // 8)) if c["rows"] > 8 and rng.random() < 0.5 else 0
        c["mask"] = rng.choice(("none", "none", "inf", "low"))
        c["scale"] = rng.choice((1.0, 1.0, 0.7, 1.25))
        if op == "logprobs":
            c["top"] = rng.choice((0, 1, 5, 20, 32))
        else:
            c["entropy"] = rng.random() < 0.5
        return c
    c = {"op": op, "requests": _log_uniform(rng, 1, 2_000), "block": rng.choice((16, 16, 32, 64, 48)), "even": rng.random() < 0.3}
    c["tokens"] = _log_uniform(rng, 1, min(90_000, MOST_TOKENS // c["requests"]))
    c["cached"] = rng.choice((0, _log_uniform(rng, 1, 20_000)))
    return c


def _lengths(case):
    """New tokens of every request: all alike, or lognormal around the median; the same lengths for every seed."""
    n, mid = case["requests"], case["tokens"]
    if case["even"]:
        return np.full(n, mid, dtype=np.int64)
    x = mid * np.exp(0.6 * np.random.default_rng(n * 1_000_003 + mid).standard_normal(n)) * 0.85
    return np.maximum(0, np.minimum(x, 8.6 * mid)).astype(np.int64)


def _cached(case):
    n = case["requests"]
    return np.random.default_rng(7 * n + case["cached"]).integers(0, 2 * case["cached"] + 1, n) if case["cached"] else np.zeros(n, dtype=np.int64)


def _document_offsets(case):
    """Documents of random lengths that leave the last rows of the buffer to none."""
    rows, docs = case["rows"], case["docs"]
    used = rows - rows // 50
    cuts = np.sort(np.random.default_rng(rows + docs).integers(0, used + 1, docs - 1))
    return np.concatenate([[0], cuts, [used]]).astype(np.int64)


def _prepare_blocks(case, seed):
    rng = np.random.default_rng(seed)
    n, block = case["requests"], case["block"]
    new, old = rng.permutation(_lengths(case)), rng.permutation(_cached(case))
    have, want = -(-old // block), -(-(old + new) // block)
    n_blocks = int((have + -(-new // block)).sum()) + 100                  # the same for every seed, whichever lengths meet
    width = int(have.max() + (-(-new // block)).max()) + 1
    ids = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((n, width), -1, dtype=np.int32)
    filled = have if case["op"] == "extend" else want
    inside = np.arange(width)[None, :] < filled[:, None]
    used = int(filled.sum())
    table[inside] = ids[:used]
    free = np.full(n_blocks, -1, dtype=np.int32)
    free[: n_blocks - used] = ids[used:]
    s = {"op": case["op"], "block": block,
         "state": {"block_table": torch.from_numpy(table).cuda(), "free_blocks": torch.from_numpy(free).cuda(),
                   "n_free": torch.tensor([n_blocks - used], dtype=torch.int64, device="cuda")}}
    out = {"seq_len": torch.zeros(n, dtype=torch.int32, device="cuda"), "n_free": torch.zeros(1, dtype=torch.int64, device="cuda"),
           "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "workspace": torch.empty(24 * n + 4_096, dtype=torch.uint8, device="cuda")}
    if case["op"] == "extend":
        off = np.concatenate([[0], np.cumsum(new)])
        total = int(off[-1])
        s["new_off"] = torch.from_numpy(off).cuda()
        s["state"]["seq_len"] = torch.from_numpy(old.astype(np.int32)).cuda()
        out["slots"] = torch.full((max(total, 1),), -1, dtype=torch.int64, device="cuda")
        out["positions"] = torch.full((max(total, 1),), -1, dtype=torch.int32, device="cuda")
        out["requests"] = torch.full((max(total, 1),), -1, dtype=torch.int32, device="cuda")
    else:
        s["state"]["seq_len"] = torch.from_numpy((old + new).astype(np.int32)).cuda()
        s["keep"] = torch.from_numpy(old.astype(np.int32)).cuda()
    s["out"] = out
    return s


def prepare(case, seed):
    op = case["op"]
    if op in ("extend", "release"):
        return _prepare_blocks(case, seed)
    rows, vocab, kind = case["rows"], case["vocab"], TYPES[case["type"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    # a model's logits: most entries spread around a low level, some rows sure of one entry
    logits = torch.empty((rows, vocab), dtype=kind, device="cuda").normal_(-1.0, 2.2, generator=g)
    ids = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    sure = torch.rand(rows, generator=g, device="cuda")
    shift = 1 if case["docs"] else 0
    at = torch.arange(rows - shift, device="cuda")
    logits[at, ids[shift:]] += (14.0 * sure[: rows - shift]).to(kind)
    if case["mask"] != "none":
        gone = torch.rand((rows, vocab), generator=g, device="cuda") < sure[:, None]
        gone[at, ids[shift:]] = False
        gone[:, 0] = False                                                 # the end of the text is always allowed
        logits.masked_fill_(gone, -math.inf if case["mask"] == "inf" else torch.finfo(kind).min)
        del gone
    s = {"op": op, "logits": logits, "ids": ids.to(torch.int32), "ids_off": None, "scale": case["scale"]}
    if case["docs"]:
        s["ids_off"] = torch.from_numpy(_document_offsets(case)).cuda()
    else:
        s["ids"][5::11] = -1                                               # positions that nothing is asked of
    floats = lambda *shape: torch.zeros(shape, dtype=torch.float32, device="cuda")  # noqa: E731
    s["out"] = {"logprob": floats(rows), "lse": floats(rows), "entropy": floats(rows), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if op == "logprobs":
        s["top"] = case["top"]
        s["out"]["rank"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        if case["top"]:
            s["out"]["top_ids"] = torch.zeros((rows, case["top"]), dtype=torch.int32, device="cuda")
            s["out"]["top_logprobs"] = floats(rows, case["top"])
        return s
    s["grad_logprob"] = torch.randn(rows, generator=g, device="cuda")
    s["grad_entropy"] = torch.randn(rows, generator=g, device="cuda") * 0.1 if case["entropy"] else None
    s["grad"] = torch.zeros_like(logits)
    for lo in range(0, rows, 256):                                         # what the forward pass left, from its definition in 64 bits
        x = logits[lo:lo + 256].double() * case["scale"]
        lse = torch.logsumexp(x, 1)
        p = torch.exp(x - lse[:, None])
        s["out"]["lse"][lo:lo + 256] = lse.float()
        s["out"]["entropy"][lo:lo + 256] = (lse - torch.where(p > 0, p * x, 0.0).sum(1)).float()
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------


def _targets(s):
    """(id that each row is asked for, whether it is asked for one, whether the row is in use)."""
    ids = s["ids"].long()
    rows = ids.numel()
    row = torch.arange(rows, device=ids.device)
    off = s["ids_off"]
    if off is None:
        return ids.clamp(min=0), ids >= 0, torch.ones_like(ids, dtype=torch.bool)
    end = off[torch.searchsorted(off, row, right=True).clamp(max=off.numel() - 1)]
    nxt = torch.cat([ids[1:], ids[:1]])
    return nxt, row + 1 < end, row < off[-1]


def _plain_logprobs(s):
    x, scale, out = s["logits"].float(), s["scale"], s["out"]
    rows, vocab = x.shape
    target, asked, used = _targets(s)
    top = x.amax(1, keepdim=True)
    d = (x - top) * scale
    e = torch.exp(d)
    total = e.sum(1)
    lse = top[:, 0] * scale + torch.log(total)
    entropy = torch.log(total) - torch.where(e > 0, e * d, 0.0).sum(1) / total
    logprob = d.gather(1, target[:, None])[:, 0] - torch.log(total)
    at = x.gather(1, target[:, None])
    col = torch.arange(vocab, device=x.device)
    rank = 1 + (x > at).sum(1) + ((x == at) & (col < target[:, None])).sum(1)
    keep = lambda new, old: torch.where(used, new, old)  # noqa: E731
    got = {"logprob": keep(torch.where(asked, logprob, 0.0), out["logprob"]), "lse": keep(lse, out["lse"]), "entropy": keep(entropy, out["entropy"]),
           "rank": keep(torch.where(asked, rank, 0).int(), out["rank"]), "status": torch.zeros_like(out["status"])}
    if s["top"]:
        bits = (x + 0.0).view(torch.int32).long()                          # in the order of the values; equal values by their place
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * 2**32 + (vocab - 1 - col)
        best = vocab - 1 - (key.topk(s["top"], dim=1).values & 0xFFFFFFFF)
        got["top_ids"] = torch.where(used[:, None], best.int(), out["top_ids"])
        got["top_logprobs"] = torch.where(used[:, None], d.gather(1, best) - torch.log(total)[:, None], out["top_logprobs"])
    return got


def _plain_grad(s):
    x, scale, out = s["logits"].float(), s["scale"], s["out"]
    target, asked, used = _targets(s)
    logp = x * scale - out["lse"][:, None]
    p = torch.exp(logp)
    g = torch.where(asked, s["grad_logprob"], 0.0)[:, None]
    dx = -g * p
    dx.scatter_add_(1, target[:, None], g)
    if s["grad_entropy"] is not None:
        dx -= s["grad_entropy"][:, None] * torch.where(p > 0, p * (logp + out["entropy"][:, None]), 0.0)
    dx = (dx * scale).to(s["grad"].dtype)
    return {"grad": torch.where(used[:, None], dx, s["grad"]), "status": torch.zeros_like(out["status"])}


def _plain_extend(s):
    off, state, out, block = s["new_off"], s["state"], s["out"], s["block"]
    table, free, n_free = state["block_table"], state["free_blocks"], state["n_free"]
    old, new = state["seq_len"].long(), off[1:] - off[:-1]
    have = (old + block - 1) // block
    need = (old + new + block - 1) // block - have
    before = torch.cumsum(need, 0) - need
    col = torch.arange(table.shape[1], device=table.device)
    k = col - have[:, None]
    taken = free[(n_free - 1 - before[:, None] - k).clamp(0, free.numel() - 1)]
    table = torch.where((k >= 0) & (k < need[:, None]), taken, table)
    token = torch.arange(out["slots"].numel(), device=table.device)
    r = torch.searchsorted(off, token, right=True) - 1
    used = token < off[-1]
    r = r.clamp(max=old.numel() - 1)
    position = old[r] + token - off[r]
    slot = table[r, (position // block).clamp(max=table.shape[1] - 1)].long() * block + position % block
    state["block_table"].copy_(table)
    return {"slots": torch.where(used, slot, out["slots"]), "positions": torch.where(used, position.int(), out["positions"]), "requests": torch.where(used, r.int(), out["requests"]),
            "block_table": state["block_table"], "seq_len": (old + new).int(), "n_free": n_free - need.sum(), "status": torch.zeros_like(out["status"])}


def _plain_release(s):
    keep, state, block = s["keep"].long(), s["state"], s["block"]
    table, free, n_free = state["block_table"], state["free_blocks"], state["n_free"]
    have, left = (state["seq_len"].long() + block - 1) // block, (keep + block - 1) // block
    drop = have - left
    before = torch.cumsum(drop, 0) - drop
    total = drop.sum()
    q = torch.arange(free.numel(), device=free.device) - n_free               # place among the blocks that come back
    q = total - 1 - q
    r = torch.searchsorted(before + drop, q, right=True).clamp(max=keep.numel() - 1)
    back = table[r, (left[r] + q - before[r]).clamp(0, table.shape[1] - 1)]
    free.copy_(torch.where((q >= 0) & (q < total), back, free))
    return {"free_blocks": free, "seq_len": s["keep"], "n_free": n_free + total, "status": torch.zeros_like(s["out"]["status"])}


PLAIN = {"logprobs": _plain_logprobs, "grad": _plain_grad, "extend": _plain_extend, "release": _plain_release}


def run(state):
    op = state["op"]
    if not own:
        return PLAIN[op](state)
    import paper_2607_29678_b200 as tt
    out = state["out"]
    if op == "logprobs":
        tt.logprobs(state["logits"], state["ids"], out, ids_off=state["ids_off"], scale=state["scale"])
        return out
    if op == "grad":
        tt.logprobs_grad(state["logits"], state["ids"], out, state["grad_logprob"], state["grad"], ids_off=state["ids_off"],
                         grad_entropy=state["grad_entropy"], scale=state["scale"])
        return {"grad": state["grad"], "status": out["status"]}
    if op == "extend":
        tt.blocks_extend(state["new_off"], state["state"], state["block"], out)
        return {"slots": out["slots"], "positions": out["positions"], "requests": out["requests"], "block_table": state["state"]["block_table"],
                "seq_len": out["seq_len"], "n_free": out["n_free"], "status": out["status"]}
    tt.blocks_release(state["keep"], state["state"], state["block"], out)
    return {"free_blocks": state["state"]["free_blocks"], "seq_len": out["seq_len"], "n_free": out["n_free"], "status": out["status"]}


def work(case):
    """Logits once in (and their gradient once out); ids, lengths and blocks once in, tables and maps once out."""
    if case["op"] in ("logprobs", "grad"):
        rows, vocab, size = case["rows"], case["vocab"], TYPES[case["type"]].itemsize
        rows = int(_document_offsets(case)[-1]) if case["docs"] else rows
        if case["op"] == "grad":
            return {"bytes": rows * (2 * vocab * size + 16 + 8 * case["entropy"]), "flops": rows * vocab * (5 + 3 * case["entropy"])}
        return {"bytes": rows * (vocab * size + 20 + 8 * case["top"]), "flops": rows * vocab * 7}
    n, new, old, block = case["requests"], _lengths(case), _cached(case), case["block"]
    old = np.sort(old)
    blocks = int(new.sum()) / block                                           # which lengths meet is the seed's
    if case["op"] == "extend":
        return {"bytes": 16 * n + 8 * blocks + 16 * int(new.sum()), "flops": 0}
    return {"bytes": 12 * n + 8 * blocks, "flops": 0}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------


def exact(case, seed):
    """Row by row blocks in double precision, from softmax probabilities; whole numbers are left to the comparison of both forms."""
    if case["op"] not in ("logprobs", "grad"):
        return None
    s = prepare(case, seed)
    rows, scale, out = case["rows"], case["scale"], s["out"]
    want = s["ids"].cpu().numpy().astype(np.int64)
    used = rows
    if case["docs"]:
        off = _document_offsets(case)
        used = int(off[-1])
        want = np.concatenate([want[1:], [-1]])
        want[off[1:][off[1:] > 0] - 1] = -1                                   # the last token of a document predicts nothing
    want = torch.from_numpy(want).cuda()
    if case["op"] == "logprobs":
        got = {"logprob": out["logprob"].double(), "lse": out["lse"].double(), "entropy": out["entropy"].double(), "rank": None, "status": None}
        if case["top"]:
            got.update(top_ids=None, top_logprobs=out["top_logprobs"].double())
    else:
        got = {"grad": s["grad"].double(), "status": None}
    for lo in range(0, used, 64):
        hi = min(used, lo + 64)
        z = s["logits"][lo:hi].double() * scale
        lse = z.logsumexp(1, keepdim=True)
        logp = z - lse
        p = logp.exp()
        plogp = torch.where(p == 0, 0.0, p * logp)
        t = want[lo:hi, None]
        has = t >= 0
        if case["op"] == "logprobs":
            got["lse"][lo:hi] = lse[:, 0]
            got["entropy"][lo:hi] = -plogp.sum(1)
            got["logprob"][lo:hi] = torch.where(has, logp.gather(1, t.clamp(min=0)), 0.0)[:, 0]
            if case["top"]:
                got["top_logprobs"][lo:hi] = logp.topk(case["top"], dim=1).values
            continue
        one = torch.zeros_like(p).scatter_(1, t.clamp(min=0), has.double())
        dx = s["grad_logprob"][lo:hi, None].double() * (one - p * has)
        if case["entropy"]:
            dx -= s["grad_entropy"][lo:hi, None].double() * (plogp - p * plogp.sum(1, keepdim=True))
        got["grad"][lo:hi] = scale * dx
    return got
