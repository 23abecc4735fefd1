"""Generation over a key/value cache held in 8 bits and the choice of the next token, as cases that can be timed and compared.

A case names one of five ways into the library and its sizes; `listed` holds the ones that stand for ordinary use from the
smallest call to the largest, `draw` any other of the same ranges.

  append  tl_k_cache8_append: keys and values of new tokens go into the cache, in pieces as the text arrives; what it holds
          of them is handed back as values (tl_k_cache8_read)
  attend  tl_k_attention_cache8: rows of queries, the last tokens of the text, over everything cached (one row: decoding)
  step    tl_k_cache8_append and tl_k_attention_cache8 as one decoding step of one layer makes them
  counts  tl_k_token_counts: how often each token of the vocabulary is in each row's history
  choose  tl_k_choose: penalties for the tokens counted, a bias, a mask of the allowed tokens, and the greedy choice

The cache: blocks of 64 tokens.  A complete block holds, for each head, codes in [-127, 127] and one scale for the keys and
one for the values, scale = max(largest magnitude, 2^-100) / 127 in fp32, code = value / scale rounded to the nearest, ties to
even.  The tokens of the last block, until it is complete, stay bf16 (the tail).  Keys lie as [block, head, D / 64, 64 tokens,
64 columns], values as [block, head, D columns, 64 tokens]; the tail's likewise, without the first axis.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 64
LEAST = 2.0 ** -100      # magnitudes below this one count as it


def listed():
    return [
        # a chunk's keys and values behind a window, one layer of the 7B shape (32 heads of 128); the text arrives in ragged
        # pieces, so that blocks are completed out of the tail
        {"name": "append_3x333", "kind": "append", "start": 1024, "new": 999, "piece": 333, "kv_heads": 32, "d_head": 128},
        # a long text at once: bytes
        {"name": "append_32768", "kind": "append", "start": 0, "new": 32768, "piece": 32768, "kv_heads": 32, "d_head": 128},
        # one token over a short window of a small decoder: latency
        {"name": "decode_200", "kind": "attend", "keys": 200, "rows": 1, "heads": 4, "kv_heads": 4, "d_head": 64},
        # one token over the window that the 7B shape decodes from, the tail half full
        {"name": "decode_3800", "kind": "attend", "keys": 3800, "rows": 1, "heads": 32, "kv_heads": 32, "d_head": 128},
        # one token over a long text, four query heads to a key head: bytes
        {"name": "decode_131072", "kind": "attend", "keys": 131072, "rows": 1, "heads": 32, "kv_heads": 8, "d_head": 128},
        # a draft of a few tokens verified at once
        {"name": "rows5_2500", "kind": "attend", "keys": 2500, "rows": 5, "heads": 32, "kv_heads": 32, "d_head": 128},
        # a chunk read behind a long context: arithmetic
        {"name": "rows2048_8192", "kind": "attend", "keys": 8192, "rows": 2048, "heads": 32, "kv_heads": 32, "d_head": 128},
        # one layer's part of a decoding step: the token's key and value into the tail, attention over what is there
        {"name": "step_1500", "kind": "step", "keys": 1500, "heads": 32, "kv_heads": 32, "d_head": 128},
        # the history of one text counted before its first step; a batch of ragged histories
        {"name": "counts_4096", "kind": "counts", "rows": 1, "tokens": 4096, "vocab": 32000},
        {"name": "counts_batch", "kind": "counts", "rows": 128, "tokens": 2000, "vocab": 50001},
        # the choice of a decoding step, and of many positions at once with a vocabulary of odd size
        {"name": "choose_1", "kind": "choose", "rows": 1, "vocab": 32000},
        {"name": "choose_256", "kind": "choose", "rows": 256, "vocab": 50001},
    ]


HEADS = ((4, 4), (8, 2), (16, 16), (12, 4), (32, 32), (32, 8), (40, 8), (24, 1))


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "attend", "attend", "attend", "step", "counts", "choose"))
    heads, kv_heads = rng.choice(HEADS)
    d_head = rng.choice((64, 128))
    if kind == "append":
        new = _log(rng, 1, 16384)
        return {"kind": kind, "start": BLOCK * rng.randint(0, 32), "new": new, "piece": rng.choice((new, new, -(-new // 3))),
                "kv_heads": kv_heads, "d_head": d_head}
    if kind == "attend":
        rows = rng.choice((1, 1, rng.randint(2, 8), _log(rng, 9, 1500)))
        keys = _log(rng, max(rows, 1), 8192) if rows > 8 else _log(rng, rows, 65536 if kv_heads <= 8 else 16384)
        return {"kind": kind, "keys": keys, "rows": rows, "heads": heads, "kv_heads": kv_heads, "d_head": d_head}
    if kind == "step":
        keys = _log(rng, 1, 8192)
        # (a token that completes a block turns the tail into codes, and a second pass would have no tail to begin with)
        return {"kind": kind, "keys": keys + (keys % BLOCK == 0), "heads": heads, "kv_heads": kv_heads, "d_head": d_head}
    vocab = _log(rng, 700, 130000)
    rows = rng.choice((1, 1, _log(rng, 2, 128)))
    if kind == "counts":
        return {"kind": kind, "rows": rows, "tokens": _log(rng, 1, 16384), "vocab": vocab}
    return {"kind": kind, "rows": rows, "vocab": vocab}


# ---------------------------------------------------------------- inputs
def _keys_values(gen, n, heads, d):
    """bf16 [n, heads, d] keys and values: normal draws, a few columns of the keys larger, as trained decoders have them"""
    k = torch.randn(n, heads, d, generator=gen, device="cuda")
    k[..., :: 16] *= 4
    v = torch.randn(n, heads, d, generator=gen, device="cuda")
    return k.bfloat16(), v.bfloat16()


def _scales_codes(x):
    """fp32 [blocks, heads] and whole-valued fp64 [blocks, 64, heads, D] of bf16 [blocks, 64, heads, D]; quotients in 64 bits,
    because a value next to the border of two codes would else go to the wrong one"""
    s = (x.abs().amax(dim=(1, 3)).double().clamp(min=LEAST) / 127).float()
    return s, torch.round(x.double() / s.double()[:, None, :, None])


def _lay_k(x):
    """[.., 64, heads, D] -> [.., heads, D / 64, 64, 64]"""
    x = x.unflatten(-1, (-1, 64))
    n = x.dim()
    return x.permute(*range(n - 4), n - 3, n - 2, n - 4, n - 1).contiguous()


def _lay_v(x):
    """[.., 64, heads, D] -> [.., heads, D, 64]"""
    n = x.dim()
    return x.permute(*range(n - 3), n - 2, n - 1, n - 3).contiguous()


def _cache(gen, n, capacity, heads, d):
    """the cache of n tokens, with room for `capacity`; positions that hold no token are left as torch.empty gives them"""
    nb, full = -(-capacity // BLOCK), n // BLOCK
    c = {"k": torch.empty(nb, heads, d // 64, BLOCK, 64, dtype=torch.int8, device="cuda"),
         "v": torch.empty(nb, heads, d, BLOCK, dtype=torch.int8, device="cuda"),
         "k_scale": torch.empty(nb, heads, device="cuda"), "v_scale": torch.empty(nb, heads, device="cuda"),
         "k_tail": torch.zeros(heads, d // 64, BLOCK, 64, dtype=torch.bfloat16, device="cuda"),
         "v_tail": torch.zeros(heads, d, BLOCK, dtype=torch.bfloat16, device="cuda"), "n": n, "capacity": capacity}
    step = 256                              # blocks at a time: the 64-bit quotients of a long cache take room
    for b in range(0, full, step):
        m = min(step, full - b)
        for x, at, lay in zip(_keys_values(gen, m * BLOCK, heads, d), "kv", (_lay_k, _lay_v)):
            s, codes = _scales_codes(x.view(m, BLOCK, heads, d))
            c[at][b:b + m] = lay(codes.to(torch.int8))
            c[at + "_scale"][b:b + m] = s
    t = n - full * BLOCK
    if t:
        for x, at, lay in zip(_keys_values(gen, t, heads, d), "kv", (_lay_k, _lay_v)):
            c[at + "_tail"].copy_(lay(torch.cat([x, torch.zeros(BLOCK - t, heads, d, dtype=x.dtype, device="cuda")])))
    return c


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind in ("append", "attend", "step"):
        h, d = case["kv_heads"], case["d_head"]
    if kind == "append":
        n = case["new"]
        s["cache"] = _cache(gen, case["start"], case["start"] + n, h, d)
        s["k"], s["v"] = (x.view(n, h * d) for x in _keys_values(gen, n, h, d))
        s["k_out"], s["v_out"] = (torch.empty(n, h * d, device="cuda") for _ in range(2))
    elif kind in ("attend", "step"):
        rows = case.get("rows", 1)
        s["cache"] = _cache(gen, case["keys"] - (kind == "step"), case["keys"], h, d)
        s["q"] = torch.randn(rows, case["heads"] * d, generator=gen, device="cuda").bfloat16()
        s["o"] = torch.empty_like(s["q"])
        s["workspace"] = torch.empty(1 << 22, device="cuda")
        if kind == "step":
            s["k"], s["v"] = (x.view(1, h * d) for x in _keys_values(gen, 1, h, d))
    elif kind == "counts":
        R, n, V = case["rows"], case["tokens"], case["vocab"]
        s["tokens"] = _history(gen, R, n, V)
        s["counts"] = torch.empty(R, V, dtype=torch.int32, device="cuda")
    else:
        R, V = case["rows"], case["vocab"]
        s["logits"] = torch.randn(R, V, generator=gen, device="cuda") * 3
        s["counts"] = torch.zeros(R, V, dtype=torch.int32, device="cuda")
        tok = _history(gen, R, 2000, V).long()
        s["counts"].scatter_add_(1, tok.clamp(min=0), (tok >= 0).int())
        s["bias"] = torch.where(torch.rand(V, generator=gen, device="cuda") < 0.02, 2.0, 0.0) * torch.randn(V, generator=gen, device="cuda")
        # three in four tokens are allowed, one bit each
        words = [torch.randint(-2 ** 31, 2 ** 31, (R, -(-V // 32)), generator=gen, device="cuda", dtype=torch.int64) for _ in range(2)]
        s["allowed"] = (words[0] | words[1]).to(torch.int32)
        s["penalties"] = {"repetition": 1.2, "presence": 0.3, "frequency": 0.05}
        s["out"] = torch.empty_like(s["logits"])
        s["choice"] = torch.empty(R, dtype=torch.int32, device="cuda")
        s["workspace"] = torch.empty(1 << 16, device="cuda")
    return s


def _history(gen, R, n, V):
    """int32 [R, n] token ids: frequent ones often, as in text; rows but the first shorter, filled up with -1"""
    ids = (V * torch.rand(R, n, generator=gen, device="cuda") ** 4).int().clamp(max=V - 1)
    length = (n * (0.5 + 0.5 * torch.rand(R, 1, generator=gen, device="cuda"))).int()
    length[0] = n
    return torch.where(torch.arange(n, device="cuda") < length, ids, -1).contiguous()


# ---------------------------------------------------------------- the framework's calls
def _run_own(s):
    from paper_2401_11504_amd import api
    case, kind = s["case"], s["case"]["kind"]
    if "cache" in s:
        c = s["cache"]
        if "handle" not in c:      # a program makes it once, with the cache's memory
            c["handle"] = api.Cache8(c["k"], c["v"], c["k_scale"], c["v_scale"], c["k_tail"], c["v_tail"], c["capacity"])
        cache = c["handle"]
    if kind == "append":
        at, n = case["start"], case["new"]
        for i in range(0, n, case["piece"]):
            m = min(case["piece"], n - i)
            api.tl_k_cache8_append(cache, at + i, s["k"][i:i + m], s["v"][i:i + m])
        api.tl_k_cache8_read(cache, at + n, at, s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if kind == "step":
        api.tl_k_cache8_append(cache, case["keys"] - 1, s["k"], s["v"])
        api.tl_k_attention_cache8(cache, case["keys"], s["q"], s["o"], case["heads"], s["workspace"])
        return {"o": s["o"], "k_tail": c["k_tail"], "v_tail": c["v_tail"]}
    if kind == "attend":
        api.tl_k_attention_cache8(cache, case["keys"], s["q"], s["o"], case["heads"], s["workspace"])
        return {"o": s["o"]}
    if kind == "counts":
        api.tl_k_token_counts(s["tokens"], s["counts"])
        return {"counts": s["counts"]}
    api.tl_k_choose(s["logits"], s["counts"], s["out"], s["choice"], bias=s["bias"], allowed=s["allowed"],
                    workspace=s["workspace"], **s["penalties"])
    return {"out": s["out"], "choice": s["choice"]}


# ---------------------------------------------------------------- the plain form
def _append_plain(x, h, d):
    """the values that the cache holds of rows that begin at a block: fp32 [n, heads D]"""
    n = x.shape[0]
    full = n // BLOCK
    sc, codes = _scales_codes(x[:full * BLOCK].view(full, BLOCK, h, d))
    held = codes.float() * sc[:, None, :, None]
    return torch.cat([held.reshape(-1, h * d), x[full * BLOCK:].float()])


def _rows_of(c, at, n):
    """fp32 [heads, n, D] of the first n tokens of keys ("k") or values ("v")"""
    full = n // BLOCK
    x = c[at][:full].float() * c[at + "_scale"][:full].view(full, c[at].shape[1], *([1] * (c[at].dim() - 2)))
    x = torch.cat([x, c[at + "_tail"][None].float()])
    if at == "k":       # [blocks, heads, D / 64, 64, 64]
        x = x.permute(1, 0, 3, 2, 4)
    else:               # [blocks, heads, D, 64]
        x = x.permute(1, 0, 3, 2)
    return x.flatten(1, 2).flatten(2)[:, :n]


def _attend_plain(c, keys, q, heads):
    rows = q.shape[0]
    k, v = _rows_of(c, "k", keys), _rows_of(c, "v", keys)
    h, _, d = k.shape
    qf = q.float().view(rows, h, heads // h, d).permute(1, 2, 0, 3).reshape(h, heads // h * rows, d)
    x = (torch.bmm(qf, k.transpose(1, 2).contiguous()) / math.sqrt(d)).view(h, heads // h, rows, keys)
    last = torch.arange(rows, device=q.device) + keys - rows
    x = x.masked_fill(torch.arange(keys, device=q.device) > last[:, None], -math.inf)
    x = torch.exp(x - x.amax(dim=-1, keepdim=True))
    x = x / x.sum(dim=-1, keepdim=True)
    o = torch.bmm(x.view(h, -1, keys), v.contiguous()).view(h, heads // h, rows, d)
    return o.permute(2, 0, 1, 3).reshape(rows, heads * d).bfloat16()


def _allowed_bits(words, V):
    bits = words.long()[..., None] >> torch.arange(32, device=words.device)
    return (bits & 1).flatten(-2)[..., :V].bool()


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "append":
        h, d = case["kv_heads"], case["d_head"]
        return {"k": _append_plain(s["k"], h, d), "v": _append_plain(s["v"], h, d)}
    if kind == "attend":
        return {"o": _attend_plain(s["cache"], case["keys"], s["q"], case["heads"])}
    if kind == "step":
        c, h, d = s["cache"], case["kv_heads"], case["d_head"]
        slot = (case["keys"] - 1) % BLOCK
        c["k_tail"][:, :, slot] = s["k"].view(h, d // 64, 64)
        c["v_tail"][:, :, slot] = s["v"].view(h, d)
        return {"o": _attend_plain(c, case["keys"], s["q"], case["heads"]), "k_tail": c["k_tail"], "v_tail": c["v_tail"]}
    if kind == "counts":
        t = s["tokens"].long()
        return {"counts": torch.zeros_like(s["counts"]).scatter_add_(1, t.clamp(min=0), (t >= 0).int())}
    x, c, p = s["logits"], s["counts"], s["penalties"]
    seen, rep = c > 0, x.new_full((), p["repetition"])     # (a tensor: torch divides by a number through its reciprocal)
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(seen, x - (c.float() * p["frequency"] + p["presence"]), x) + s["bias"]
    x = x.masked_fill(~_allowed_bits(s["allowed"], x.shape[1]), -math.inf)
    best = x.amax(dim=1, keepdim=True)
    index = torch.arange(x.shape[1], device=x.device)
    return {"out": x, "choice": torch.where(x == best, index, x.shape[1]).amin(dim=1).int()}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind == "append":
        n = case["new"] * case["kv_heads"] * case["d_head"]
        # keys and values in, their codes and their values out
        return {"bytes": 2.0 * n * (2 + 1 + 4), "flops": 2.0 * n * 3}
    if kind in ("attend", "step"):
        keys, rows, d = case["keys"], case.get("rows", 1), case["d_head"]
        seen = rows * (keys - rows) + rows * (rows + 1) / 2
        return {"bytes": 2.0 * keys * case["kv_heads"] * d + 4.0 * rows * case["heads"] * d, "flops": 4.0 * seen * case["heads"] * d}
    if kind == "counts":
        return {"bytes": 4.0 * case["rows"] * (case["tokens"] + case["vocab"]), "flops": float(case["rows"] * case["tokens"])}
    R, V = case["rows"], case["vocab"]
    return {"bytes": R * V * 12.125 + 4.0 * V, "flops": 6.0 * R * V}


# ---------------------------------------------------------------- the definition in 64 bits
def _held(x, h, d):
    """block by block and head by head"""
    out = x.double().clone().view(-1, h, d)
    for b in range(x.shape[0] // BLOCK):
        blk = out[b * BLOCK:(b + 1) * BLOCK]
        top = blk.abs().amax(dim=2).amax(dim=0).clamp(min=LEAST)
        unit = (top / 127).float().double()[:, None]
        blk.copy_((blk / unit).round() * unit)
    return out.view(-1, h * d)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "append":
        return {x: _held(s[x], case["kv_heads"], case["d_head"]) for x in "kv"}
    if kind in ("attend", "step"):
        c, keys, H, h, d = s["cache"], case["keys"], case["heads"], case["kv_heads"], case["d_head"]
        q = s["q"].double().view(-1, H, d)
        rows, slot = q.shape[0], (keys - 1) % BLOCK
        if kind == "step":
            c["k_tail"][:, :, slot] = s["k"].view(h, d // 64, 64)
            c["v_tail"][:, :, slot] = s["v"].view(h, d)
        o = torch.empty_like(q)
        later = torch.arange(keys, device="cuda")[None] - torch.arange(rows, device="cuda")[:, None] > keys - rows
        for kh in range(h):
            k = (c["k"][:, kh].double() * c["k_scale"][:, kh].double()[:, None, None, None])[:keys // BLOCK]
            v = (c["v"][:, kh].double() * c["v_scale"][:, kh].double()[:, None, None])[:keys // BLOCK]
            k = torch.cat([k, c["k_tail"][kh][None].double()]).transpose(1, 2).reshape(-1, d)[:keys]
            v = torch.cat([v, c["v_tail"][kh][None].double()]).transpose(1, 2).reshape(-1, d)[:keys]
            for j in range(kh * (H // h), (kh + 1) * (H // h)):
                x = (q[:, j] @ k.T) * d ** -0.5
                x[later] = -math.inf
                o[:, j] = torch.exp(x - torch.logsumexp(x, dim=1, keepdim=True)) @ v
        o = o.view(rows, H * d)
        return {"o": o} if kind == "attend" else {"o": o, "k_tail": c["k_tail"].double(), "v_tail": c["v_tail"].double()}
    if kind == "counts":
        return None
    x = s["logits"].double().cpu().numpy()
    c = s["counts"].cpu().numpy()
    p = s["penalties"]
    y = np.where(c > 0, np.where(x > 0, x / p["repetition"], x * p["repetition"]) - p["presence"] - p["frequency"] * c, x)
    y += s["bias"].double().cpu().numpy()
    bits = np.unpackbits(s["allowed"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :x.shape[1]]
    y[bits == 0] = -np.inf
    return {"out": torch.from_numpy(y), "choice": None}
