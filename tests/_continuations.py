"""Several continuations of a sequence: the operators' definitions, by lists and in 64 bits (CPU), for their tests."""
import math

import torch

import _serving as sv


# ------------------------------------------------------------------------------------------------ attention of drafted tokens
def random_tree(n, words, gen, roots=0.2):
    """bits [n, words] int64: of each drafted token those that it descends from and itself"""
    seen = []
    for i in range(n):
        parent = -1 if i == 0 or torch.rand((), generator=gen) < roots else int(torch.randint(i, (), generator=gen))
        seen.append((1 << i) | (seen[parent] if parent >= 0 else 0))
    return to_bits(seen, words)


def to_bits(seen, words):
    """rows of Python integers -> int64 [rows, words]"""
    out = torch.zeros(len(seen), words, dtype=torch.int64)
    for i, bits in enumerate(seen):
        for w in range(words):
            x = bits >> (64 * w) & (2 ** 64 - 1)
            out[i, w] = x - 2 ** 64 if x >= 2 ** 63 else x
    return out


def attention(q, k, v, seen, dtype):
    """One head: rows q [n, d], row i sees key j where seen[i, j].  (out, lse, bounds of their errors); the bounds are those of _serving.attention."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = k.shape
    if n == 0:
        z, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full((len(q),), -math.inf, dtype=torch.float64)
        return z, lse, z, torch.zeros_like(lse)
    score = (q @ k.nan_to_num(0.0, 0.0, 0.0).T / math.sqrt(d)).masked_fill(~seen, -math.inf)
    size = (q.abs() @ k.abs().nan_to_num(0.0, 0.0, 0.0).T / math.sqrt(d)).masked_fill(~seen, 0.0).amax(-1)
    lse = torch.logsumexp(score, -1)
    weight = (score - lse[:, None].nan_to_num(neginf=0.0)).exp().masked_fill(~seen, 0.0)
    clean = v.nan_to_num(0.0, 0.0, 0.0)
    out, absolute = weight @ clean, weight @ clean.abs()
    each = (d + 2) * 2.0 ** -24 * size + 2.0 ** -21 + (n + 8) * 2.0 ** -24
    return out, lse, sv.HALF[dtype] * out.abs() + (sv.HALF[dtype] + 2 * each)[:, None] * absolute, each + 2.0 ** -21 + 2.0 ** -22 * lse.abs().nan_to_num(posinf=0.0)


def tree_attention(q, kc, vc, table, lengths, cu, tree, max_len=None):
    """(out [rows, H, d], lse [rows, H], bounds); rows of no sequence NaN"""
    rows, H, d = q.shape
    n_pages, page, H_kv, _ = kc.shape
    out, lse, ob, lb = (torch.full(s, math.nan, dtype=torch.float64) for s in ((rows, H, d), (rows, H), (rows, H, d), (rows, H)))
    most = table.shape[1] * page if max_len is None else max_len
    for b in range(len(lengths)):
        begin, end = int(cu[b]), int(cu[b + 1])
        L, n = min(max(lengths[b], 0), most), end - begin
        if n == 0:
            continue
        keys = [j for j in range(L) if 0 <= int(table[b, j // page]) < n_pages]
        flat = torch.tensor([int(table[b, j // page]) * page + j % page for j in keys], dtype=torch.long)
        drafted = torch.tensor([j - (L - n) for j in keys], dtype=torch.long)
        i = torch.arange(n)[:, None]
        if tree is None:
            seen = drafted[None] <= i
        else:
            named = torch.zeros(n, n, dtype=torch.bool)
            for c in range(min(n, 64 * tree.shape[1])):
                named[:, c] = (tree[begin:end, c // 64] >> (c % 64)) & 1 != 0
            seen = torch.where(drafted[None] < 0, True, named[:, drafted.clamp(min=0)]) if len(keys) else torch.zeros(n, 0, dtype=torch.bool)
        for h in range(H):
            g = h // (H // H_kv)
            r = attention(q[begin:end, h], kc.view(-1, H_kv, d)[flat, g], vc.view(-1, H_kv, d)[flat, g], seen, q.dtype)
            out[begin:end, h], lse[begin:end, h], ob[begin:end, h], lb[begin:end, h] = r
    return out, lse, ob, lb


# ------------------------------------------------------------------------------------------------ pages
def fork(kc, vc, table, lengths, parents, room=None, held=None):
    """(k_cache, v_cache, table_out, lengths_out, missing) by the definition"""
    n_pages, page = kc.shape[:2]
    wide = table.shape[1]
    table = table.tolist()
    kc, vc = kc.clone(), vc.clone()
    result, out_lengths, writers, used = [], [], {}, set(i for i in range(n_pages) if held is not None and int(held[i]) != 0)
    read = set(used)
    for s, p in enumerate(parents):
        some = 0 <= p < len(lengths)
        n = min(max(lengths[p], 0), wide * page) if some else 0
        r = (1 if some else 0) if room is None else max(room[s], 0)
        mine = [x if 0 <= x < n_pages else -1 for x in table[p][:-(-n // page)]] if some else []
        result.append((n, r, mine))
        for nth, x in enumerate(mine):
            if x < 0:
                continue
            used.add(x)
            if nth == n // page and r > 0:
                writers.setdefault(x, []).append(s)
            else:
                read.add(x)
    free = [x for x in range(n_pages) if x not in used]
    new, missing, moves = [], 0, []
    for s, (n, r, mine) in enumerate(result):
        row = list(mine)
        if n % page and r > 0 and mine[-1] >= 0:
            x = mine[-1]
            if x in read or writers[x][0] != s:
                if free:
                    row[-1] = free.pop(0)
                    moves.append((x, row[-1], n % page))
                else:
                    row[-1], missing = -1, missing + 1
        wanted = -(-(n + r) // page)
        missing += max(0, wanted - wide)
        for _ in range(min(wanted, wide) - len(row)):
            if free:
                row.append(free.pop(0))
            else:
                row.append(-1)
                missing += 1
        new.append(row + [-1] * (wide - len(row)))
        out_lengths.append(min(n + r, wide * page))
    old_k, old_v = kc.clone(), vc.clone()
    for x, y, rows in moves:
        kc[y, :rows], vc[y, :rows] = old_k[x, :rows], old_v[x, :rows]
    return kc, vc, torch.tensor(new, dtype=torch.int32).view(len(parents), wide), torch.tensor(out_lengths, dtype=torch.int32), missing


def compact(kc, vc, table, lengths, cu, kept):
    """(k_cache, v_cache, lengths_out); kept: a list of ascending numbers for every sequence"""
    n_pages, page = kc.shape[:2]
    old_k, old_v, kc, vc = kc, vc, kc.clone(), vc.clone()
    out = []
    for b, path in enumerate(kept):
        base = min(max(lengths[b], 0), table.shape[1] * page) - int(cu[b + 1] - cu[b])

        def place(p):
            x = int(table[b, p // page]) if p >= 0 else -1
            return (x, p % page) if 0 <= x < n_pages else None

        for i, at in enumerate(path):
            frm, to = place(base + at), place(base + i)
            if frm and to:
                kc[to], vc[to] = old_k[frm], old_v[frm]
        out.append(max(0, base + len(path)))
    return kc, vc, torch.tensor(out, dtype=torch.int32)


# ------------------------------------------------------------------------------------------------ beam search's choice
# A row's sum is off by 2^-19 of itself at most (32 terms added in 32 bits, the lanes' sums in 64; 2^-21 for the exponentials and what they are taken of)
LSE_BOUND = 2.0 ** -19 + 2.0 ** -21


def select(logits, scores, n_out, finished=None, end_token=-1):
    """(scores_out in 64 bits, parents, tokens, finished_out, least distance of two totals of different beams that the choice rests on)"""
    B, K = scores.shape
    V = logits.shape[1]
    want = torch.full((B, n_out), -math.inf, dtype=torch.float64), torch.full((B, n_out), -1), torch.full((B, n_out), -1), torch.ones(B, n_out, dtype=torch.bool)
    margin = math.inf
    for b in range(B):
        all_of = []
        for k in range(K):
            score, x = float(scores[b, k]), logits[b * K + k].double()
            if not math.isfinite(score):
                continue
            if finished is not None and bool(finished[b, k]):
                all_of.append((-score, k, end_token, True))
                continue
            lse = float(torch.logsumexp(x, 0))
            if not math.isfinite(lse):
                continue
            # of equal logits the lower token first
            order = sorted(torch.topk(x, min(V, n_out)).values.tolist(), reverse=True)
            least = order[-1]
            some = [(-(float(x[v])), v) for v in (x >= least).nonzero()[:, 0].tolist() if float(x[v]) > -math.inf]
            for neg, v in sorted(some)[:n_out]:
                all_of.append((-(score + (-neg - lse)), k, v, v == end_token))
        all_of.sort()
        for one, two in zip(all_of[:n_out], all_of[1:n_out + 1]):
            if one[1] != two[1] and one[0] != two[0]:           # (alike to the last bit: rows that are, whose sums are too)
                margin = min(margin, two[0] - one[0])
        for i, (neg, k, v, ended) in enumerate(all_of[:n_out]):
            want[0][b, i], want[1][b, i], want[2][b, i], want[3][b, i] = -neg, b * K + k, v, ended
    return (*want, margin)
