"""Generation for many texts at once over a paged key/value cache that forgets what little was attended to, and the sampled choice of
the next token, as cases that can be timed and compared.

A case names one of four ways into the library and its sizes; `listed` holds the ones that stand for ordinary use from the smallest
call to the largest, `draw` any other of the same ranges.

  step    tl_k_paged_append and tl_k_attention_paged as one decoding step of one layer makes them: a token of each sequence into its
          pages, its attention over them, and with "weights" the attention that every token got added to what it got before
  prompt  tl_k_paged_append and tl_k_attention_weights: a prompt's keys and values into pages, the attention that its tokens got
  evict   tl_k_paged_evict: each head keeps its most recent tokens and those that got most attention, in the first slots
  sample  tl_k_sample: temperature, top-k, top-p, min-p, and a token drawn by a given number

The cache: bf16 keys and values, [pages, heads, tokens of a page, d_head].  Slot j of sequence s lies on page table[s, j / page] at
j % page.  A head's slots are its own: after an eviction different heads hold different tokens in the same slot, and `positions` says
which.  What a token got of attention is the sum of its softmax weights over the queries and the query heads of its key head.

The choice: a token's weight is exp((x - largest) / temperature) in whole units of 2^-40, so that sums of weights are exact in any order.
"""
import math

import numpy as np
import torch

own = False

ONE = 2 ** 40             # the weight of the largest logit


def listed():
    return [
        # one text over a short window of a small decoder: latency
        {"name": "step_200", "kind": "step", "seqs": 1, "keys": 200, "heads": 4, "kv_heads": 4, "d_head": 64, "page": 16, "weights": False},
        # one text over the window that the 7B shape decodes from, the attention its tokens get kept for an eviction
        {"name": "step_3800", "kind": "step", "seqs": 1, "keys": 3800, "heads": 32, "kv_heads": 32, "d_head": 128, "page": 64, "weights": True},
        # one text of great length, four query heads to a key head: bytes
        {"name": "step_131072", "kind": "step", "seqs": 1, "keys": 131072, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 128, "weights": False},
        # a batch of texts of different lengths
        {"name": "step_64x4096", "kind": "step", "seqs": 64, "keys": 4096, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 64, "weights": False},
        # the same on small pages, five query heads to a key head, kept for an eviction
        {"name": "step_33x2000", "kind": "step", "seqs": 33, "keys": 2000, "heads": 40, "kv_heads": 8, "d_head": 128, "page": 16, "weights": True},
        # a short prompt of odd length
        {"name": "prompt_777", "kind": "prompt", "tokens": 777, "heads": 4, "kv_heads": 4, "d_head": 64, "page": 16},
        # a window and a chunk of the 7B shape
        {"name": "prompt_2048", "kind": "prompt", "tokens": 2048, "heads": 32, "kv_heads": 32, "d_head": 128, "page": 64},
        # a long prompt: arithmetic
        {"name": "prompt_8192", "kind": "prompt", "tokens": 8192, "heads": 32, "kv_heads": 8, "d_head": 128, "page": 128},
        # a batch that is cut back by a page, as decoding goes on
        {"name": "evict_64x2112", "kind": "evict", "seqs": 64, "keys": 2112, "budget": 2048, "recent": 256, "kv_heads": 8, "d_head": 128, "page": 64},
        # a long prompt cut down to a window
        {"name": "evict_32768", "kind": "evict", "seqs": 1, "keys": 32768, "budget": 4096, "recent": 1024, "kv_heads": 32, "d_head": 128, "page": 64},
        # the choice of a decoding step of one text
        {"name": "sample_1", "kind": "sample", "rows": 1, "vocab": 32000, "settings": 0},
        # of a large batch with settings of each row's own and a large vocabulary
        {"name": "sample_512", "kind": "sample", "rows": 512, "vocab": 128000, "settings": -1},
    ]


HEADS = ((4, 4), (8, 2), (16, 16), (12, 4), (32, 32), (32, 8), (40, 8), (24, 1))
# temperature, top-k, top-p, min-p
SETTINGS = ((0.8, 50, 0.95, 0.02), (1.0, 0, 0.9, 0.0), (0.7, 0, 1.0, 0.05), (1.3, 400, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0))


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("step", "step", "step", "prompt", "evict", "sample", "sample"))
    heads, kv_heads = rng.choice(HEADS)
    d_head, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128))
    if kind == "step":
        seqs = rng.choice((1, 1, _log(rng, 2, 64)))
        keys = _log(rng, 1, min(65536, 250000 * 4 // (seqs * kv_heads)))
        return {"kind": kind, "seqs": seqs, "keys": keys, "heads": heads, "kv_heads": kv_heads, "d_head": d_head, "page": page,
                "weights": rng.choice((False, True))}
    if kind == "prompt":
        return {"kind": kind, "tokens": _log(rng, 1, 6000), "heads": heads, "kv_heads": kv_heads, "d_head": d_head, "page": page}
    if kind == "evict":
        seqs = rng.choice((1, 1, _log(rng, 2, 64)))
        keys = _log(rng, 2, min(32768, 1000000 // (seqs * kv_heads)))
        budget = max(1, int(keys * rng.choice((rng.uniform(0.05, 0.5), rng.uniform(0.5, 1.0)))))
        return {"kind": kind, "seqs": seqs, "keys": keys, "budget": budget, "recent": int(budget * rng.uniform(0.0, 0.5)), "kv_heads": kv_heads,
                "d_head": d_head, "page": page}
    vocab = _log(rng, 700, 130000)
    return {"kind": kind, "rows": rng.choice((1, 1, _log(rng, 2, 256))), "vocab": vocab, "settings": rng.randint(-1, len(SETTINGS) - 1)}


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """how many tokens each sequence holds: the first as many as the case says, the others spread from a quarter of that upwards"""
    n, keys = case["seqs"], case["keys"]
    return [keys] + [max(1, int(keys * (0.25 + 0.75 * (0.6180339887 * i % 1)))) for i in range(1, n)]


def _normal_keys(gen, *shape):
    """bf16 keys: normal draws, a few columns larger, as trained decoders have them"""
    k = torch.randn(*shape, generator=gen, device="cuda").bfloat16()
    k[..., :: 16] *= 4
    return k


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").bfloat16()


def _pages(gen, lengths, case):
    """pages in a scattered order, a few of them nobody's; the table's entries behind a sequence's last page are -1"""
    page, h, d = case["page"], case["kv_heads"], case["d_head"]
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").int()
    table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return {"k": _normal_keys(gen, n_pages, h, page, d), "v": _normal(gen, n_pages, h, page, d), "table": table}


def _got(gen, *shape):
    """what tokens got of attention so far: most very little, some a lot"""
    return torch.exp(2.5 * torch.randn(*shape, generator=gen, device="cuda") - 3)


def _lse(q, k, heads, kv_heads):
    """fp32 [heads, T]: the log of the sum of exp over each row's scores, as a prompt's attention hands it over"""
    T, d = q.shape[0], q.shape[1] // heads
    out = torch.empty(heads, T, device="cuda")
    later = torch.ones(T, T, dtype=torch.bool, device="cuda").triu_(1)
    for j in range(heads):
        x = q[:, j * d:(j + 1) * d].float() @ k[:, j // (heads // kv_heads) * d:][:, :d].float().T.contiguous() / math.sqrt(d)
        out[j] = torch.logsumexp(x.masked_fill_(later, -math.inf), dim=1)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "step":
        lengths = _lengths(case)
        n, h, d = case["seqs"], case["kv_heads"], case["d_head"]
        s["cache"] = _pages(gen, lengths, case)
        s["after"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["before"] = s["after"] - 1
        s["q"], s["k"], s["v"] = _normal(gen, n, case["heads"] * d), _normal_keys(gen, n, h * d), _normal(gen, n, h * d)
        s["o"] = torch.empty_like(s["q"])
        if case["weights"]:
            width = max(lengths)
            s["weights"] = _got(gen, n, h, width)
            s["weights_out"] = torch.zeros_like(s["weights"])
            s["positions"] = torch.arange(width, dtype=torch.int32, device="cuda").expand(n, h, width).contiguous()
            s["pos"] = s["before"] + 1000
        s["workspace"] = torch.empty(n * case["heads"] * (case["keys"] + 16384), device="cuda")
    elif kind == "prompt":
        T, h, d = case["tokens"], case["kv_heads"], case["d_head"]
        s["cache"] = _pages(gen, [T], {**case, "seqs": 1})
        s["before"] = torch.zeros(1, dtype=torch.int32, device="cuda")
        s["first_row"] = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        s["pos"] = torch.arange(T, dtype=torch.int32, device="cuda")
        s["q"], s["k"], s["v"] = _normal(gen, T, case["heads"] * d), _normal_keys(gen, T, h * d), _normal(gen, T, h * d)
        s["lse"] = _lse(s["q"], s["k"], case["heads"], h)
        s["weights"] = torch.zeros(1, h, T, device="cuda")
        s["positions"] = torch.zeros(1, h, T, dtype=torch.int32, device="cuda")
    elif kind == "evict":
        lengths = _lengths(case)
        n, h, width = case["seqs"], case["kv_heads"], max(lengths)
        s["cache"] = _pages(gen, lengths, case)
        s["before"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["after"] = torch.empty_like(s["before"])
        s["weights"] = _got(gen, n, h, width)
        # the slots of the budget hold tokens of an earlier eviction in any order, those behind them what came since
        head = min(case["budget"], width)
        early = torch.rand(n, h, head, generator=gen, device="cuda").argsort(dim=2)
        late = torch.arange(head, width, device="cuda").expand(n, h, width - head)
        s["positions"] = torch.cat([early, late], dim=2).int().contiguous()
        s["weights_out"], s["positions_out"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["positions"])
        s["workspace"] = torch.empty(n * h * (2 * case["budget"] + 1), device="cuda")
    else:
        R, V = case["rows"], case["vocab"]
        # frequencies of tokens fall with their rank by a power, as in text, steeply where the model is sure
        power = 1 + torch.rand(R, 1, generator=gen, device="cuda")
        s["logits"] = 0.5 * torch.randn(R, V, generator=gen, device="cuda") - power * torch.log(1 + V * torch.rand(R, V, generator=gen, device="cuda")) + 10
        s["logits"][1::3] = s["logits"][1::3].masked_fill(torch.rand(V, generator=gen, device="cuda") < 0.75, -math.inf)     # a mask went over these
        which = [case["settings"] if case["settings"] >= 0 else r % len(SETTINGS) for r in range(R)]
        s["params"] = torch.tensor([SETTINGS[w] for w in which], device="cuda")
        s["u"] = torch.rand(R, generator=gen, device="cuda")
        s["choice"], s["kept"] = (torch.empty(R, dtype=torch.int32, device="cuda") for _ in range(2))
        s["prob"] = torch.empty(R, device="cuda")
        s["workspace"] = torch.empty(1 << 20, device="cuda")
    return s


# ---------------------------------------------------------------- the framework's calls
def _run_own(s):
    from paper_2401_11504_amd import api
    case, kind = s["case"], s["case"]["kind"]
    if "cache" in s:
        c = s["cache"]
        if "handle" not in c:      # a program makes it once, with the cache's memory
            c["handle"] = api.Paged(c["k"], c["v"], c["table"])
        cache = c["handle"]
    if kind == "step":
        more = {"weights": s["weights"], "positions": s["positions"], "pos": s["pos"]} if case["weights"] else {}
        api.tl_k_paged_append(cache, s["before"], s["k"], s["v"], **more)
        more = {"weights_in": s["weights"], "weights_out": s["weights_out"]} if case["weights"] else {}
        api.tl_k_attention_paged(cache, s["after"], s["q"], s["o"], case["heads"], max_len=case["keys"], workspace=s["workspace"], **more)
        return _of_step(s)
    if kind == "prompt":
        api.tl_k_paged_append(cache, s["before"], s["k"], s["v"], first_row=s["first_row"], weights=s["weights"], positions=s["positions"], pos=s["pos"])
        api.tl_k_attention_weights(s["q"], s["k"], case["heads"], case["kv_heads"], s["lse"], None, s["weights"][0])
        return {"k": c["k"], "v": c["v"], "weights": s["weights"], "positions": s["positions"]}
    if kind == "evict":
        api.tl_k_paged_evict(cache, s["before"], case["budget"], case["recent"], s["weights"], s["positions"], s["weights_out"], s["positions_out"],
                             s["after"], s["workspace"])
        return {"k": c["k"], "v": c["v"], "weights": s["weights_out"], "positions": s["positions_out"], "lengths": s["after"]}
    api.tl_k_sample(s["logits"], s["params"], s["u"], s["choice"], s["kept"], s["prob"], s["workspace"])
    return {"choice": s["choice"], "kept": s["kept"], "prob": s["prob"]}


def _of_step(s):
    out = {"o": s["o"], "k": s["cache"]["k"], "v": s["cache"]["v"]}
    if s["case"]["weights"]:
        out.update(weights=s["weights_out"], positions=s["positions"])
    return out


# ---------------------------------------------------------------- the plain form
def _put_plain(c, seq, slot, k, v):
    """rows of k and v into slot[i] of sequence seq[i]"""
    h, page, d = c["k"].shape[1:]
    at = c["table"][seq, slot // page].long()
    c["k"][at, :, slot % page] = k.view(-1, h, d)
    c["v"][at, :, slot % page] = v.view(-1, h, d)


def _rows_plain(pool, table, width):
    """fp32 [sequences, heads, width, d] of what lies in the sequences' slots; places without a page hold anything"""
    x = pool[table.long().clamp(min=0)]                     # [sequences, pages, heads, page, d]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :width].float().contiguous()


def _step_plain(s):
    c, case = s["cache"], s["case"]
    n, h, d, G, width = case["seqs"], case["kv_heads"], case["d_head"], case["heads"] // case["kv_heads"], case["keys"]
    seq = torch.arange(n, device="cuda")
    slot = s["before"].long()
    _put_plain(c, seq, slot, s["k"], s["v"])
    k, v = _rows_plain(c["k"], c["table"], width), _rows_plain(c["v"], c["table"], width)
    q = s["q"].float().view(n, h, G, d)
    x = torch.matmul(k, q.transpose(2, 3).contiguous()).transpose(2, 3).contiguous() / math.sqrt(d)      # [n, h, G, width]
    there = torch.arange(width, device="cuda") < s["after"].view(n, 1, 1, 1)
    x = x.masked_fill(~there, -math.inf)
    x = torch.exp(x - x.amax(dim=-1, keepdim=True))
    x = x / x.sum(dim=-1, keepdim=True)
    s["o"].copy_(torch.matmul(x, v).reshape(n, h * G * d).bfloat16())
    if case["weights"]:
        s["weights"][seq, :, slot] = 0.0
        s["positions"][seq, :, slot] = s["pos"][:, None].expand(n, h)
        s["weights_out"].copy_(torch.where(there[:, :, 0], s["weights"] + x.sum(dim=2), s["weights_out"]))
    return _of_step(s)


def _prompt_plain(s):
    c, case = s["cache"], s["case"]
    T, h, d, G = case["tokens"], case["kv_heads"], case["d_head"], case["heads"] // case["kv_heads"]
    slot = torch.arange(T, device="cuda")
    _put_plain(c, torch.zeros_like(slot), slot, s["k"], s["v"])
    s["positions"].copy_(s["pos"].expand(1, h, T))
    q = s["q"].float().view(T, h, G, d).permute(1, 2, 0, 3).reshape(h, G * T, d)
    k = s["k"].float().view(T, h, d).permute(1, 2, 0).contiguous()
    x = torch.bmm(q, k).view(h, G, T, T)
    x.div_(math.sqrt(d)).sub_(s["lse"].view(h, G, T, 1)).exp_()
    x.masked_fill_(slot > slot[:, None], 0.0)
    s["weights"].copy_(x.sum(dim=(1, 2))[None])
    return {"k": c["k"], "v": c["v"], "weights": s["weights"], "positions": s["positions"]}


def _evict_plain(s):
    c, case = s["cache"], s["case"]
    n, h, B = case["seqs"], case["kv_heads"], case["budget"]
    w, p = s["weights"], s["positions"].long()
    width, page = w.shape[2], c["k"].shape[2]
    slot = torch.arange(width, device="cuda")
    length = s["before"].long()
    there = (slot < length[:, None, None]).expand(n, h, width)
    newest = p.masked_fill(~there, -1).amax(dim=2, keepdim=True)
    key = torch.where(p > newest - case["recent"], math.inf, w).masked_fill(~there, -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True).indices
    keep = torch.zeros(n, h, width, dtype=torch.bool, device="cuda").scatter_(2, order[:, :, :B], True) & there
    hole, mover = there & ~keep & (slot < B), keep & (slot >= B)
    # the i-th hole receives the i-th of the kept slots behind the budget; there are as many of the ones as of the others
    count = mover.sum(dim=2, keepdim=True)
    most = max(0, min(B, width - B))
    i, j = (torch.arange(m, device="cuda").view(shape) for m, shape in ((n, (n, 1, 1)), (h, (1, h, 1))))
    which = torch.arange(most, device="cuda").expand(n, h, most)
    which = torch.where(which < count, which, 0)            # places without a pair copy the first one once more, or slot 0 to itself
    dst, src = (torch.zeros(n, h, width + 1, dtype=torch.long, device="cuda")
                .scatter_(2, torch.where(x, torch.cumsum(x, 2) - 1, width), slot.expand(n, h, width)).gather(2, which) * (count > 0)
                for x in (hole, mover))
    a, b = c["table"][i, dst // page].long(), c["table"][i, src // page].long()
    for x in (c["k"], c["v"]):
        x[a, j, dst % page] = x[b, j, src % page]
    first = there & (slot < B)
    for out, x in ((s["weights_out"], w), (s["positions_out"], s["positions"])):
        out.copy_(torch.where(first, x.scatter(2, dst, x.gather(2, src)), out))
    s["after"].copy_(length.clamp(max=B))
    return {"k": c["k"], "v": c["v"], "weights": s["weights_out"], "positions": s["positions_out"], "lengths": s["after"]}


def _sample_plain(s):
    x, V = s["logits"], s["logits"].shape[1]
    T, K, p, least = (c[:, None] for c in s["params"].double().unbind(1))
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(dim=1, keepdim=True)
    index = torch.arange(V, device=x.device)
    w = torch.round(torch.exp((x.double() - top.double()) * (1.0 / T)) * ONE)
    w = torch.where(x == top, float(ONE), torch.where(x == -math.inf, 0.0, w))
    first = torch.where(x == top, index, V).amin(dim=1, keepdim=True)
    w = torch.where(T > 0, w, torch.where(index == first, float(ONE), 0.0)).long()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    keep = (index < torch.where(K > 0, K, V)) & (ws > 0)
    ws = torch.where(keep, ws, 0)
    before = torch.cumsum(ws, 1) - ws
    limit = torch.ceil(p * ws.sum(dim=1, keepdim=True).double()).long()
    keep &= (p >= 1) | (before < limit) | (index == 0)
    keep &= ws >= torch.ceil(least * ONE).long()
    w = torch.where(torch.zeros_like(keep).scatter_(1, order, keep), w, 0)
    total = w.sum(dim=1, keepdim=True)
    at = torch.floor(s["u"].double()[:, None] * total.double()).long()
    at = torch.minimum(at, total - 1)
    choice = (torch.cumsum(w, 1) <= at).sum(dim=1)
    prob = w.gather(1, choice[:, None]).double() / total.double()
    return {"choice": choice.int(), "kept": keep.sum(dim=1).int(), "prob": prob[:, 0].float()}


def run(state):
    if own:
        return _run_own(state)
    return {"step": _step_plain, "prompt": _prompt_plain, "evict": _evict_plain, "sample": _sample_plain}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind == "step":
        n, h, d, H, keys = case["seqs"], case["kv_heads"], case["d_head"], case["heads"], sum(_lengths(case))
        # pages and queries read, outputs and the new rows (from where they come, to their pages) written; what tokens got, in and out
        return {"bytes": 4.0 * keys * h * d + n * (4.0 * H * d + 4.0 * h * d) + (8.0 * keys * h if case["weights"] else 0.0), "flops": 4.0 * keys * H * d}
    if kind == "prompt":
        T, h, d, H = case["tokens"], case["kv_heads"], case["d_head"], case["heads"]
        return {"bytes": 8.0 * T * h * d + 2.0 * T * H * d + 4.0 * T * H + 8.0 * T * h, "flops": 1.0 * T * (T + 1) * H * d}
    if kind == "evict":
        total = 0.0
        for n in _lengths(case):
            B, r = case["budget"], min(case["recent"], n)
            moved = 0.0
            if n > B:      # the recent tokens behind the budget, and their share of the others that stay
                late = min(r, n - B)
                moved = late + (B - r) * (n - B - late) / max(1, n - r)
            total += case["kv_heads"] * (8.0 * n + 8.0 * min(n, B) + moved * 8.0 * case["d_head"])
        return {"bytes": total, "flops": 0.0}
    return {"bytes": 4.0 * case["rows"] * case["vocab"], "flops": 8.0 * case["rows"] * case["vocab"]}


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(s)
    c = s["cache"]
    h, page, d = c["k"].shape[1:]
    table = c["table"].cpu().numpy()
    if kind == "step":
        H = case["heads"]
        o = torch.empty(case["seqs"], H, d, dtype=torch.float64, device="cuda")
        for i, n in enumerate(_lengths(case)):
            at, off = int(table[i, (n - 1) // page]), (n - 1) % page
            c["k"][at, :, off], c["v"][at, :, off] = s["k"][i].view(h, d), s["v"][i].view(h, d)
            ids = torch.from_numpy(table[i, :-(-n // page)].astype(np.int64)).cuda()
            for j in range(h):
                k, v = (c[x][ids, j].reshape(-1, d)[:n].double() for x in "kv")
                q = s["q"][i].double().view(h, H // h, d)[j]
                x = (k @ q.T) * d ** -0.5
                x = torch.exp(x - torch.logsumexp(x, dim=0))
                o[i, j * (H // h):(j + 1) * (H // h)] = x.T @ v
                if case["weights"]:
                    s["weights"][i, j, n - 1], s["positions"][i, j, n - 1] = 0.0, s["pos"][i]
                    s["weights_out"] = s["weights_out"].double()
                    s["weights_out"][i, j, :n] = s["weights"][i, j, :n].double() + x.sum(dim=1)
        out = {"o": o.view(case["seqs"], H * d), "k": c["k"].double(), "v": c["v"].double()}
        if case["weights"]:
            out.update(weights=s["weights_out"], positions=None)
        return out
    if kind == "prompt":
        T, H = case["tokens"], case["heads"]
        got = torch.zeros(1, h, T, dtype=torch.float64, device="cuda")
        for j in range(H):
            q, k = s["q"].view(T, H, d)[:, j].double(), s["k"].view(T, h, d)[:, j // (H // h)].double()
            for a in range(0, T, 2048):
                x = torch.exp((q[a:a + 2048] @ k.T) * d ** -0.5 - s["lse"][j, a:a + 2048, None].double())
                got[0, j // (H // h)] += x.tril(a).sum(dim=0)
        for t in range(-(-T // page)):
            m = min(page, T - t * page)
            for x in "kv":
                c[x][int(table[0, t]), :, :m] = s[x][t * page:t * page + m].view(m, h, d).transpose(0, 1)
        return {"k": c["k"].double(), "v": c["v"].double(), "weights": got, "positions": None}
    w, p = s["weights"].cpu().numpy(), s["positions"].cpu().numpy()
    w_out = np.zeros(w.shape)
    B = case["budget"]
    for i, n in enumerate(_lengths(case)):
        for j in range(h):
            first = (p[i, j, :n] <= p[i, j, :n].max() - case["recent"]).astype(np.int64)      # recent ones before others
            kept = np.lexsort((np.arange(n), -w[i, j, :n].astype(np.float64), first))[:B]
            src = np.sort(kept[kept >= B])
            dst = np.setdiff1d(np.arange(min(B, n)), kept)[:len(src)]
            w_out[i, j, :min(B, n)] = w[i, j, :min(B, n)]
            w_out[i, j, dst] = w[i, j, src]
            a, b = (torch.from_numpy(table[i, y // page].astype(np.int64)).cuda() for y in (dst, src))
            fr, to = torch.from_numpy(src % page).cuda(), torch.from_numpy(dst % page).cuda()
            for x in "kv":
                c[x][a, j, to] = c[x][b, j, fr]
    return {"k": c["k"].double(), "v": c["v"].double(), "weights": torch.from_numpy(w_out), "positions": None, "lengths": None}


def _exact_sample(s):
    logits, settings, u = s["logits"].double().cpu().numpy(), s["params"].cpu().numpy(), s["u"].cpu().numpy()
    prob = np.zeros(len(u))
    for r, x in enumerate(logits):
        T, K, p, least = (float(y) for y in settings[r])
        ranked = np.argsort(-x, kind="stable")
        if T <= 0:
            prob[r] = 1.0
            continue
        w = np.rint(np.exp((x[ranked] - x[ranked[0]]) / T) * ONE).astype(np.int64)
        n = int(K) if 0 < K < len(x) else len(x)
        if p < 1:
            total = int(w[:n].sum())
            n = min(n, max(1, int(np.searchsorted(np.cumsum(w), math.ceil(p * total))) + 1))
        n = min(n, int((w >= max(1, math.ceil(least * ONE))).sum()))
        of = np.sort(ranked[:n])
        w = np.rint(np.exp((x[of] - x[ranked[0]]) / T) * ONE).astype(np.int64)
        total = int(w.sum())
        at = min(total - 1, math.floor(float(u[r]) * float(total)))
        prob[r] = w[int(np.searchsorted(np.cumsum(w), at, side="right"))] / total
    return {"choice": None, "kept": None, "prob": torch.from_numpy(prob)}
