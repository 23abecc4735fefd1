"""Plain 64-bit definitions of the calls on a key/value cache on pages and of the drawn token (CPU; loops over sequences and heads)."""
import math

import numpy as np
import torch

ONE = 2 ** 40


def page_of(table, n_pages, seq, slot, page):
    i = int(table[seq, slot // page])
    return i if 0 <= i < n_pages else -1


def append(k_pool, v_pool, table, lengths, k, v, first_row=None, pos=None, weights=None, positions=None):
    """in place on CPU tensors"""
    n_pages, heads, page, d = k_pool.shape
    n_seqs, n_table = table.shape
    for row in range(k.shape[0]):
        seq, i = row, 0
        if first_row is not None:
            owner = [s for s in range(n_seqs) if int(first_row[s]) <= row < int(first_row[s + 1])]
            if not owner:
                continue
            seq = owner[0]
            i = row - int(first_row[seq])
        slot = max(int(lengths[seq]), 0) + i
        if slot >= n_table * page:
            continue
        for t, value in ((weights, 0.0), (positions, slot if pos is None else int(pos[row]))):
            if t is not None and slot < t.shape[2]:
                t[seq, :, slot] = value
        at = page_of(table, n_pages, seq, slot, page)
        if at >= 0:
            k_pool[at, :, slot % page] = k[row].view(heads, d)
            v_pool[at, :, slot % page] = v[row].view(heads, d)


def attention(k_pool, v_pool, table, lengths, max_len, q, heads):
    """-> o fp64 [n_seqs, heads * d]; got fp64 [n_seqs, kv_heads, max_len]; how far 32 bits may be off: tol_o like o (before its rounding), tol_got like got"""
    n_pages, kv, page, d = k_pool.shape
    n_seqs, G = table.shape[0], heads // kv
    o, tol_o = (torch.zeros(n_seqs, heads, d, dtype=torch.float64) for _ in range(2))
    got, tol_got = (torch.zeros(n_seqs, kv, max_len, dtype=torch.float64) for _ in range(2))
    for s in range(n_seqs):
        n = min(max(int(lengths[s]), 0), max_len)
        slots = [j for j in range(n) if page_of(table, n_pages, s, j, page) >= 0]
        if not slots:
            continue
        pages = torch.tensor([page_of(table, n_pages, s, j, page) for j in slots])
        at, off = torch.tensor(slots), torch.tensor([j % page for j in slots])
        for h in range(kv):
            k, v = (x[pages, h, off].double() for x in (k_pool, v_pool))
            qq = q[s].view(heads, d)[h * G:(h + 1) * G].double()
            x = qq @ k.T / math.sqrt(d)
            p = torch.softmax(x, dim=1)
            o[s, h * G:(h + 1) * G] = p @ v
            got[s, h, at] = p.sum(dim=0)
            # a score is a sum of d products in fp32, scaled and shifted (three roundings of at most its size): off by (d + 3) 2^-24 of the sum of magnitudes;
            # a weight by twice that (its own score, the others' in the sum), two steps of the exponential (2^-23 each) and n 2^-24 for the sums
            size = (qq.abs() @ k.abs().T / math.sqrt(d)).amax()
            rel = 2 * (d + 3) * 2.0 ** -24 * size + 2 * 2.0 ** -23 + len(slots) * 2.0 ** -24
            # (fp32 has no normal number below 2^-126: a weight below it may become 0, and is off by no more than 2^-126 then)
            # outputs: weights in two bf16 parts, the first cut off after 8 bits (2^-7), the rest rounded (2^-8 of it): 2^-15; and a sum of n products
            tol_o[s, h * G:(h + 1) * G] = (p @ v.abs()) * (rel + 2.0 ** -15 + len(slots) * 2.0 ** -24) + 2.0 ** -126 * v.abs().sum(dim=0)
            tol_got[s, h, at] = p.sum(dim=0) * (rel + G * 2.0 ** -24) + G * 2.0 ** -126
    return o.view(n_seqs, -1), got, tol_o.view(n_seqs, -1), tol_got


def evict(k_pool, v_pool, table, lengths, budget, recent, weights, positions):
    """in place on CPU tensors; -> new lengths, weights, positions (copies)"""
    n_pages, kv, page, d = k_pool.shape
    weights_out, positions_out, after = weights.clone(), positions.clone(), []
    for s in range(table.shape[0]):
        n = min(max(int(lengths[s]), 0), weights.shape[2], table.shape[1] * page)
        after.append(min(n, budget))
        for h in range(kv):
            newest = max((int(positions[s, h, j]) for j in range(n)), default=0)

            def rank(j):
                if page_of(table, n_pages, s, j, page) < 0:
                    return (0 if j < budget else 3, 0, 0.0, j)
                w = float(weights[s, h, j])
                of_recent = 1 if int(positions[s, h, j]) > newest - recent else 2
                return (of_recent, 1, 0.0, j) if w != w else (of_recent, 0, -w, j)
            kept = sorted(range(n), key=rank)[:budget]
            src = sorted(j for j in kept if j >= budget)
            dst = sorted(set(range(min(n, budget))) - set(kept))
            assert len(src) == len(dst)
            for a, b in zip(src, dst):
                weights_out[s, h, b], positions_out[s, h, b] = weights[s, h, a], positions[s, h, a]
                pa, pb = page_of(table, n_pages, s, a, page), page_of(table, n_pages, s, b, page)
                assert pa >= 0 and pb >= 0                # nothing moves from or to where there is no page
                for x in (k_pool, v_pool):
                    x[pb, h, b % page] = x[pa, h, a % page]
    return torch.tensor(after, dtype=torch.int32), weights_out, positions_out


def column_sums(q, k, heads, kv, lse, first_row):
    """fp64 [kv, T], and how far 32 bits may be off"""
    T, d = q.shape[0], q.shape[1] // heads
    out, tol = (torch.zeros(kv, T, dtype=torch.float64) for _ in range(2))
    rows = torch.arange(T)[:, None]
    sees = (torch.arange(T) <= rows) & (rows >= first_row)
    for j in range(heads):
        h = j // (heads // kv)
        qq, kk = q.view(T, heads, d)[:, j].double(), k.view(T, kv, d)[:, h].double()
        x = torch.exp(qq @ kk.T / math.sqrt(d) - lse[j].double()[:, None]).masked_fill(~sees, 0.0)
        out[h] += x.sum(dim=0)
        # the score as above; lse in fp32 times log2(e), added: three roundings of at most its size
        size = (qq.abs() @ kk.abs().T / math.sqrt(d)).amax(dim=1, keepdim=True)
        rel = (d + 3) * 2.0 ** -24 * size + 3 * 2.0 ** -24 * lse[j].double().abs()[:, None] + 2 * 2.0 ** -23
        tol[h] += (x * (rel + T * 2.0 ** -24)).sum(dim=0)
    return out, tol + heads * 2.0 ** -24 * out + heads * T * 2.0 ** -126        # (weights below fp32's normal numbers may become 0)


def sample(logits, params, u):
    """-> choice, kept, prob: lists"""
    V = logits.shape[1]
    out = []
    for r in range(logits.shape[0]):
        x = logits[r].double().numpy().copy()
        x[np.isnan(x)] = -np.inf
        T, K, p, least = (float(t) for t in params[r])
        top = x.max()
        if top == -np.inf:
            out.append((-1, 0, 0.0))
            continue
        if not T > 0:
            out.append((int(np.argmax(x)), 1, 1.0))
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            w = np.rint(np.exp((x - top) / T) * ONE)
        w[x == top] = ONE
        w = [int(a) if a == a else 0 for a in w]
        order = sorted((i for i in range(V) if w[i] > 0), key=lambda i: (-x[i], i))
        if 1 <= K < V:
            order = order[:int(K)]
        if p < 1:
            limit = math.ceil(p * float(sum(w[i] for i in order)))
            before, n = 0, 0
            for i in order:
                if n and before >= limit:
                    break
                before += w[i]
                n += 1
            order = order[:n]
        if least > 0:
            order = [i for i in order if w[i] >= math.ceil(min(least, 1.0) * ONE)]
        S = sum(w[i] for i in order)
        t = min(math.floor(max(float(u[r]), 0.0) * float(S)), S - 1)
        upto = 0
        for i in sorted(order):
            upto += w[i]
            if upto > t:
                out.append((i, len(order), w[i] / S))
                break
    return [list(c) for c in zip(*out)]
