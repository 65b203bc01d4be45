"""What is measured of the operators for several continuations of a sequence: beams, and trees of drafted tokens, over the paged cache.

Four kinds of pass, each one call of the public binding (`paper_2311_02382_amd.lss`) with the buffers such a program keeps:

  tree     the attention of drafted tokens over the cached ones and over those drafted ones that each descends from, or of a chunk of a
           long prompt over what is cached of it (lss_paged_attn_tree)
  select   beam search's choice over beams and vocabulary (lss_beam_select)
  fork     the sequences of the next step take on their parents' pages: shared where they are full, copied where two write, freed, new ones for new
           tokens (lss_paged_fork)
  compact  the accepted ones of the drafted tokens move to the front (lss_paged_compact)

With `own` false the same operators run in their plain form: elementary torch operations in 32 bits (64 for the totals that beams are chosen by).  Activations and
logits are i.i.d. Gaussian; a sequence's pages lie in the pool in random order, as they do after a while of serving.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _tree(B, drafted, length, H, H_kv, d, page, dtype="bf16", chain=False, ragged=1):
    """`drafted`: (least, most) drafted tokens of a sequence; `length`: (least, most) tokens in front of them; `chain`: each descends from the one before"""
    return {"kind": "tree", "B": B, "n_lo": drafted[0], "n_hi": drafted[1], "len_lo": length[0], "len_hi": length[1], "H": H, "H_kv": H_kv, "d": d, "page": page,
            "dtype": dtype, "chain": chain, "ragged": ragged}


def _select(B, K, N, V, dtype="bf16", spread=3.0, finished=False, ragged=1):
    """`spread`: of the logits; `finished`: some beams have ended"""
    return {"kind": "select", "B": B, "K": K, "N": N, "V": V, "dtype": dtype, "spread": spread, "finished": finished, "ragged": ragged}


def _fork(B, K, prompt, new, H_kv, d, page, dtype="bf16", ragged=1):
    """B prompts with K beams each; `prompt`: (least, most) tokens whose full pages the beams share; `new`: (least, most) tokens since"""
    return {"kind": "fork", "B": B, "K": K, "len_lo": prompt[0], "len_hi": prompt[1], "new_lo": new[0], "new_hi": new[1], "H_kv": H_kv, "d": d, "page": page,
            "dtype": dtype, "ragged": ragged}


def _compact(B, drafted, kept, length, H_kv, d, page, dtype="bf16", ragged=1):
    """`kept`: (least, most) of the drafted tokens are accepted"""
    return {"kind": "compact", "B": B, "n_lo": drafted[0], "n_hi": drafted[1], "kept_lo": kept[0], "kept_hi": kept[1], "len_lo": length[0], "len_hi": length[1],
            "H_kv": H_kv, "d": d, "page": page, "dtype": dtype, "ragged": ragged}


def listed():
    return [
        # one user, a short conversation, a small model: five drafted tokens, nothing but latency
        {"name": "tree token", **_tree(1, (5, 5), (77, 77), 4, 4, 64, 16)},
        # a server with two dozen sequences of very different lengths, small trees, groups of four heads
        {"name": "tree ragged", **_tree(24, (4, 12), (1, 8192), 32, 8, 128, 32, ragged=2)},
        # a busy server that drafts a lot: trees of 64 tokens, 256 rows to a head of keys
        {"name": "tree wide", **_tree(48, (64, 64), (2048, 6500), 32, 8, 128, 16, ragged=3)},
        # the next piece of a long prompt, an odd number of tokens over what is cached of it; no tree
        {"name": "tree chunk", **_tree(1, (1001, 1001), (23000, 23000), 16, 4, 64, 64, chain=True)},
        # single precision, every head with keys of its own, as the float training runs
        {"name": "tree f32", **_tree(6, (3, 21), (300, 4000), 8, 8, 64, 32, dtype="f32", ragged=4)},
        # one user, a few beams, characters: the first steps of a conversation
        {"name": "select characters", **_select(1, 4, 4, 256, dtype="f32")},
        # an ordinary service: eight prompts, eight beams each, some of which have ended; twice as many are chosen
        {"name": "select beams", **_select(8, 8, 16, 32001, finished=True, ragged=5)},
        # a full one: 32 prompts, a large vocabulary
        {"name": "select full", **_select(32, 8, 8, 128256, spread=2.0, ragged=6)},
        # one user, four beams
        {"name": "fork beams", **_fork(1, 4, (77, 77), (1, 40), 4, 64, 16)},
        # 48 prompts with eight beams each, long shared prompts
        {"name": "fork full", **_fork(48, 8, (300, 6000), (1, 700), 8, 128, 32, ragged=7)},
        # one user's tree of ten tokens, a path of which is accepted
        {"name": "compact token", **_compact(1, (10, 10), (3, 3), (77, 77), 4, 64, 16)},
        # a busy server's trees of up to 64 tokens
        {"name": "compact full", **_compact(192, (16, 64), (1, 12), (1, 6000), 8, 128, 32, ragged=8)},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_MOST = {"tree": {"bytes": 9e8, "flops": 2.0e11}, "select": {"bytes": 6.5e7, "flops": 1e12}, "fork": {"bytes": 8e7, "flops": 1}, "compact": {"bytes": 1.2e7, "flops": 1}}


def draw(rng):
    while True:
        kind = rng.choice(["tree", "tree", "select", "fork", "compact"])
        d, dtype = rng.choice([64, 64, 128, 128]), "f32" if rng.random() < 0.25 else "bf16"
        H_kv = rng.choice([1, 2, 3, 4, 6, 8, 8, 16])
        H = H_kv * rng.choice([1, 2, 3, 4, 5, 7, 8, 16])
        page, ragged = rng.choice([16, 32, 64, 128, 256]), rng.randint(10, 10 ** 6)
        if H > 64:
            continue
        if kind == "tree":
            hi, chain = _log_int(rng, 1, 30000), rng.random() < 0.3
            n = _log_int(rng, 1, 1200 if chain else 150)
            c = _tree(_log_int(rng, 1, 128 if n < 100 else 8), (_log_int(rng, 1, n), n), (_log_int(rng, 1, hi), hi), H, H_kv, d, page, dtype, chain, ragged)
        elif kind == "select":
            K = rng.choice([1, 2, 3, 4, 5, 8, 8, 16, 32])
            c = _select(_log_int(rng, 1, 64), K, min(64, K * rng.choice([1, 1, 2])), _log_int(rng, 64, 200000), dtype, rng.choice([0.5, 1.0, 2.0, 4.0]), rng.random() < 0.4, ragged)
        elif kind == "fork":
            hi, new = _log_int(rng, 1, 8000), _log_int(rng, 1, 1000)
            c = _fork(_log_int(rng, 1, 64), rng.choice([1, 2, 3, 4, 5, 8, 8, 16]), (_log_int(rng, 1, hi), hi), (_log_int(rng, 1, new), new), H_kv, d, page, dtype, ragged)
        else:
            n, hi = _log_int(rng, 1, 150), _log_int(rng, 1, 6000)
            kept = _log_int(rng, 1, min(n, 20))
            c = _compact(_log_int(rng, 1, 256), (_log_int(rng, kept, n), n), (_log_int(rng, 1, kept), kept), (_log_int(rng, 1, hi), hi), H_kv, d, page, dtype, ragged)
        w, most = work(c), _MOST[kind]
        # (a pass over float does six products where one over bf16 does one)
        if w["bytes"] <= most["bytes"] and w["flops"] * (4 if dtype == "f32" else 1) <= most["flops"] and _pool_bytes(c) <= 1.2e9:
            return c


def _lengths(c):
    """(tokens in front, drafted or new tokens) of every sequence, fork: of every prompt"""
    rng = random.Random(c["ragged"])
    lo, hi = (c["new_lo"], c["new_hi"]) if c["kind"] == "fork" else (c["n_lo"], c["n_hi"])
    return [(_log_int(rng, c["len_lo"], c["len_hi"]), _log_int(rng, lo, hi)) for _ in range(c["B"])]


def _kept(c):
    """numbers of drafted tokens that every sequence keeps, ascending"""
    rng = random.Random(c["ragged"] + 1)
    return [sorted(rng.sample(range(n), min(n, rng.randint(c["kept_lo"], c["kept_hi"])))) for _, n in _lengths(c)]


def _parents(c):
    """of every beam; the beams of a prompt are chosen from among its own, the better ones more often"""
    rng = random.Random(c["ragged"] + 2)
    return [b * c["K"] + min(rng.randrange(c["K"]), rng.randrange(c["K"])) for b in range(c["B"]) for _ in range(c["K"])]


def _pages(c):
    """pages of every sequence; fork: (shared, own) of every prompt's beams before the call"""
    if c["kind"] != "fork":
        return [-(-(old + new) // c["page"]) for old, new in _lengths(c)]
    return [(old // c["page"], -(-(old + new) // c["page"]) - old // c["page"]) for old, new in _lengths(c)]


def _n_pages(c):
    if c["kind"] != "fork":
        return sum(_pages(c)) + 3                               # a few pages belong to nobody
    return sum(shared + c["K"] * mine for shared, mine in _pages(c)) + 2 * c["B"] * c["K"] + 3


def _row_elements(c):
    return c["H_kv"] * c["d"]


def _element(c):
    return 4 if c["dtype"] == "f32" else 2


def _pool_bytes(c):
    return 0 if c["kind"] == "select" else 2 * _n_pages(c) * c["page"] * _row_elements(c) * _element(c)


def work(case):
    c = case
    eb = _element(c)
    if c["kind"] == "select":
        # logits in; scores in and out, parents and tokens out.  A subtraction, an exponential, a sum and a comparison each
        rows = c["B"] * c["K"]
        return {"bytes": rows * c["V"] * eb + 4 * rows + 12 * c["B"] * c["N"], "flops": 4 * rows * c["V"]}
    both = _lengths(c)
    if c["kind"] == "tree":
        H, H_kv, d = c["H"], c["H_kv"], c["d"]
        rows, words = sum(n for _, n in both), 0 if c["chain"] else -(-c["n_hi"] // 64)
        keys = sum(old + n for old, n in both)
        pairs = sum(n * old + (n * (n + 1) // 2 if c["chain"] else n * n) for old, n in both)
        return {"bytes": 2 * keys * H_kv * d * eb + rows * (H * (2 * d * eb + 4) + 8 * words) + 4 * sum(_pages(c)) + 8 * c["B"], "flops": 4 * pairs * H * d}
    row = 2 * 2 * _row_elements(c) * eb                           # of both caches, read and written
    if c["kind"] == "compact":
        moved = sum(i != at for path in _kept(c) for i, at in enumerate(path))
        return {"bytes": moved * row + 4 * sum(map(len, _kept(c))) + 16 * c["B"], "flops": 0}
    # the first beam with a parent keeps its partly filled page, the others copy what is in it
    parents, copied, table = _parents(c), 0, 0
    for b, (old, new) in enumerate(both):
        mine = parents[b * c["K"]:(b + 1) * c["K"]]
        copied += (c["K"] - len(set(mine))) * ((old + new) % c["page"])
        table += c["K"] * (-(-(old + new) // c["page"]))
    return {"bytes": copied * row + 2 * 4 * table + 4 * c["B"] * c["K"] * 3, "flops": 0}


# ------------------------------------------------------------------------------------------------ inputs
def _starts(counts):
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    return starts


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _trees(both, words, rng):
    """Of every drafted token, `words` words of bits: those that it sees, itself and what it descends from"""
    rows = []
    for _, n in both:
        seen = []
        for i in range(n):
            parent = rng.randrange(-1, i)                           # -1: the last token in front of the tree
            seen.append((1 << i) | (seen[parent] if parent >= 0 else 0))
        rows += seen
    signed = [[(bits >> (64 * w)) & (2 ** 64 - 1) for w in range(words)] for bits in rows]
    return torch.tensor([[x - 2 ** 64 if x >= 2 ** 63 else x for x in row] for row in signed], dtype=torch.int64, device="cuda")


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _DTYPES[c["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt)

    if c["kind"] == "select":
        B, K, N, V = c["B"], c["K"], c["N"], c["V"]
        s = {"case": c, "logits": normal(B * K, V).mul_(c["spread"]), "scores": -20 * torch.rand((B, K), generator=gen, device="cuda"),
             "scores_out": torch.empty((B, N), dtype=torch.float32, device="cuda"), "parents": torch.empty((B, N), dtype=torch.int32, device="cuda"),
             "tokens": torch.empty((B, N), dtype=torch.int32, device="cuda")}
        if c["finished"]:
            s["finished"] = torch.rand((B, K), generator=gen, device="cuda") < 0.2
            s["finished"][:, 0] = False                             # (a prompt all of whose beams have ended is not searched any more)
            s["finished_out"] = torch.empty((B, N), dtype=torch.bool, device="cuda")
        return s
    both, n_pages = _lengths(c), _n_pages(c)
    s = {"case": c, "both": both, "k_cache": normal(n_pages, c["page"], c["H_kv"], c["d"]), "v_cache": normal(n_pages, c["page"], c["H_kv"], c["d"])}
    order = torch.randperm(n_pages, generator=gen, device="cuda").tolist()
    if c["kind"] == "fork":
        # a page more than the longest sequence has: room for the next token
        wide, table, at = max(shared + mine for shared, mine in _pages(c)) + 1, [], 0
        for shared, mine in _pages(c):
            prompt, at = order[at:at + shared], at + shared
            for _ in range(c["K"]):
                table.append(prompt + order[at:at + mine] + [-1] * (wide - shared - mine))
                at += mine
        S = c["B"] * c["K"]
        s.update(table=_int32(table), lengths=_int32([old + new for old, new in both for _ in range(c["K"])]), parents=_int32(_parents(c)),
                 table_out=torch.empty((S, wide), dtype=torch.int32, device="cuda"), lengths_out=torch.empty(S, dtype=torch.int32, device="cuda"),
                 missing=torch.empty(1, dtype=torch.int32, device="cuda"))
        return s
    pages = _pages(c)
    table, at = [], 0
    for n in pages:
        table.append(order[at:at + n] + [0] * (max(pages) - n))
        at += n
    s.update(table=_int32(table), lengths=_int32([old + n for old, n in both]), cu=_int32(_starts([n for _, n in both])), longest=max(old + n for old, n in both))
    if c["kind"] == "compact":
        kept = _kept(c)
        most = max(map(len, kept))
        s.update(kept=_int32([path + [-1] * (most - len(path)) for path in kept]), n_kept=_int32([len(path) for path in kept]),
                 lengths_out=torch.empty(c["B"], dtype=torch.int32, device="cuda"))
        return s
    s["q"] = normal(sum(n for _, n in both), c["H"], c["d"])
    s.update(tree=None if c["chain"] else _trees(both, -(-c["n_hi"] // 64), random.Random(seed)), out=torch.empty_like(s["q"]),
             lse=torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda"))
    return s


# ------------------------------------------------------------------------------------------------ the calls
def _answer(s, *names):
    return {name: s[name] for name in names if name in s}


def _run_own(s):
    from paper_2311_02382_amd import lss
    kind = s["case"]["kind"]
    if kind == "tree":
        lss.lss_paged_attn_tree(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["cu"], tree=s["tree"], max_len=s["longest"], out=s["out"], lse=s["lse"])
        return _answer(s, "out", "lse")
    if kind == "select":
        lss.lss_beam_select(s["logits"], s["scores"], s["case"]["N"], finished=s.get("finished"), end_token=2, scores_out=s["scores_out"], parents=s["parents"],
                            tokens=s["tokens"], finished_out=s.get("finished_out"))
        return _answer(s, "scores_out", "parents", "tokens", "finished_out")
    if kind == "fork":
        lss.lss_paged_fork(s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["parents"], table_out=s["table_out"], lengths_out=s["lengths_out"],
                           missing=s["missing"])
        return _answer(s, "k_cache", "v_cache", "table_out", "lengths_out", "missing")
    lss.lss_paged_compact(s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["cu"], s["kept"], s["n_kept"], lengths_out=s["lengths_out"])
    return _answer(s, "k_cache", "v_cache", "lengths_out")


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_tree(s):
    c = s["case"]
    H, H_kv, d, page = c["H"], c["H_kv"], c["d"], c["page"]
    G = H // H_kv
    r0 = 0
    for b, (old, n) in enumerate(s["both"]):
        L = old + n
        pages = s["table"][b, :-(-L // page)].long()
        q = s["q"][r0:r0 + n].float().view(n, H_kv, G, d).permute(1, 2, 0, 3).contiguous()          # [H_kv, G, n, d]
        k = s["k_cache"][pages].flatten(0, 1)[:L].float().permute(1, 2, 0).contiguous()            # [H_kv, d, L]
        v = s["v_cache"][pages].flatten(0, 1)[:L].float().transpose(0, 1).contiguous()             # [H_kv, L, d]
        drafted = torch.arange(n, device="cuda")
        if s["tree"] is None:
            hidden = drafted > drafted[:, None]
        else:
            hidden = (s["tree"][r0:r0 + n][:, drafted // 64] >> (drafted % 64)) & 1 == 0              # [n, n]
        heads = max(1, min(H_kv, (1 << 28) // (G * n * L)))
        for h in range(0, H_kv, heads):
            some = slice(h, min(H_kv, h + heads))
            count = some.stop - h
            score = torch.matmul(q[some].reshape(count, G * n, d), k[some]).view(count, G, n, L) * d ** -0.5
            score[..., old:].masked_fill_(hidden, float("-inf"))
            top = score.amax(-1, keepdim=True)
            weight = (score - top).exp()
            total = weight.sum(-1, keepdim=True)
            out = torch.matmul(weight.view(count, G * n, L), v[some]).view(count, G, n, d) / total
            mine = slice(h * G, some.stop * G)
            s["out"][r0:r0 + n, mine] = out.permute(2, 0, 1, 3).reshape(n, count * G, d)
            s["lse"][r0:r0 + n, mine] = (total.log() + top).permute(2, 0, 1, 3).reshape(n, count * G)
        r0 += n
    return _answer(s, "out", "lse")


def _plain_select(s):
    c = s["case"]
    B, K, N, V = c["B"], c["K"], c["N"], c["V"]
    x = s["logits"].double()                                        # 64 bits: totals of two beams may lie next to each other
    top = x.amax(-1, keepdim=True)
    total = x - ((x - top).exp().sum(-1, keepdim=True).log() + top) + s["scores"].double().view(B * K, 1)
    if "finished" in s:
        ended = s["finished"].view(B * K, 1)
        total = torch.where(ended, float("-inf"), total)
        total[:, 2:3] = torch.where(ended, s["scores"].double().view(B * K, 1), total[:, 2:3])
    value, flat = total.view(B, K * V).sort(dim=-1, descending=True, stable=True)
    value, flat = value[:, :N], flat[:, :N]
    beam = torch.arange(B, device="cuda")[:, None] * K + flat // V
    s["scores_out"].copy_(value)
    s["parents"].copy_(beam)
    s["tokens"].copy_(flat % V)
    if "finished" in s:
        s["finished_out"].copy_(s["finished"].view(-1)[beam] | (flat % V == 2))
    return _answer(s, "scores_out", "parents", "tokens", "finished_out")


def _plain_fork(s):
    page, (n_pages, wide) = s["case"]["page"], (s["k_cache"].shape[0], s["table"].shape[1])
    p = s["parents"].long()
    S, length, table = p.shape[0], s["lengths"].long()[p], s["table"].long()[p]
    nth, each = torch.arange(wide, device="cuda"), torch.arange(S, device="cuda")
    full, part = (length // page)[:, None], (length % page)
    table = torch.where(nth < (length[:, None] + page - 1) // page, table, -1)
    tail = torch.where(part > 0, table.gather(1, full)[:, 0], n_pages)                            # (n_pages: none)
    reads = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    reads[torch.where((nth < full) & (table >= 0), table, n_pages)] = True
    first = torch.full((n_pages + 1,), S, device="cuda").scatter_reduce_(0, tail, each, "amin")
    copies = (part > 0) & (reads[tail] | (first[tail] != each))
    used = reads | (first < S)
    free = used[:n_pages].long().sort(stable=True)[1]                                             # the free ones first, in their order
    needs = copies | (part == 0)                                                                    # one more token each
    fresh = free[(needs.long().cumsum(0) - 1).clamp(min=0)]
    table.scatter_(1, full, torch.where(needs, fresh, table.gather(1, full)[:, 0])[:, None])
    move = copies[:, None] & (torch.arange(page, device="cuda") < part[:, None])
    who, slot = move.nonzero(as_tuple=True)
    for cache in (s["k_cache"], s["v_cache"]):
        cache[fresh[who], slot] = cache[tail[who], slot]
    s["table_out"].copy_(table)
    s["lengths_out"].copy_(length + 1)
    s["missing"].copy_((needs.sum() - (~used[:n_pages]).sum()).clamp(min=0))
    return _answer(s, "k_cache", "v_cache", "table_out", "lengths_out", "missing")


def _plain_compact(s):
    page = s["case"]["page"]
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    base = s["lengths"].long() - n
    seq, nth = (torch.arange(s["kept"].shape[1], device="cuda") < s["n_kept"][:, None]).nonzero(as_tuple=True)
    source, target = base[seq] + s["kept"].long()[seq, nth], base[seq] + nth
    table = s["table"].long()
    for cache in (s["k_cache"], s["v_cache"]):
        cache[table[seq, target // page], target % page] = cache[table[seq, source // page], source % page]
    s["lengths_out"].copy_(base + s["n_kept"])
    return _answer(s, "k_cache", "v_cache", "lengths_out")


def run(state):
    if own:
        return _run_own(state)
    return {"tree": _plain_tree, "select": _plain_select, "fork": _plain_fork, "compact": _plain_compact}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_tree(s, c):
    H, H_kv, d, page = c["H"], c["H_kv"], c["d"], c["page"]
    G = H // H_kv
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    r0 = 0
    for b, (old, n) in enumerate(s["both"]):
        p = torch.arange(old + n, device="cuda")
        flat = s["table"][b].long()[p // page] * page + p % page
        # what each row sees: bit by bit
        seen = torch.ones((n, old + n), dtype=torch.bool, device="cuda")
        for j in range(n):
            if c["chain"]:
                seen[:, old + j] = torch.arange(n, device="cuda") >= j
            else:
                seen[:, old + j] = torch.bitwise_and(s["tree"][r0:r0 + n, j // 64], torch.tensor(1 << (j % 64) if j % 64 < 63 else -2 ** 63, device="cuda")) != 0
        for g in range(H_kv):
            k, v = (s[name].view(-1, H_kv, d)[flat, g].double() for name in ("k_cache", "v_cache"))
            for h in range(g * G, (g + 1) * G):
                score = torch.where(seen, s["q"][r0:r0 + n, h].double() @ k.T / math.sqrt(d), -math.inf)
                log_sum = torch.logsumexp(score, -1)
                out[r0:r0 + n, h] = (score - log_sum[:, None]).exp() @ v
                lse[r0:r0 + n, h] = log_sum
        r0 += n
    return {"out": out, "lse": lse}


def _exact_select(s, c):
    scores = []
    for b in range(c["B"]):
        best = []
        for k in range(c["K"]):
            x, score = s["logits"][b * c["K"] + k].double(), s["scores"][b, k].double()
            if c["finished"] and bool(s["finished"][b, k]):
                best.append(score[None])
            else:
                best.append(score + torch.log_softmax(x, 0).topk(min(c["N"], c["V"]))[0])
        scores.append(torch.cat(best).topk(c["N"])[0])
    return {"scores_out": torch.stack(scores), "parents": None, "tokens": None, "finished_out": None}


def _exact_fork(s, c):
    """The same by lists: what is in a page after the call"""
    page, K = c["page"], c["K"]
    table, parents, lengths = s["table"].tolist(), s["parents"].tolist(), s["lengths"].tolist()
    used, writes = set(), {}
    for i, p in enumerate(parents):
        used.update(table[p][:-(-lengths[p] // page)])
        if lengths[p] % page:
            writes.setdefault(table[p][lengths[p] // page], []).append(i)
    free = iter(x for x in range(s["k_cache"].shape[0]) if x not in used)
    k, v = s["k_cache"].double(), s["v_cache"].double()
    for i, p in enumerate(parents):
        part = lengths[p] % page
        tail = table[p][lengths[p] // page]
        if part == 0:
            next(free)
        elif writes[tail][0] != i:
            to = next(free)
            k[to, :part], v[to, :part] = k[tail, :part], v[tail, :part]
    return {"k_cache": k, "v_cache": v, "table_out": None, "lengths_out": None, "missing": None}


def _exact_compact(s, c):
    k, v = s["k_cache"].double(), s["v_cache"].double()
    table = s["table"].tolist()
    for b, path in enumerate(_kept(c)):
        old = s["both"][b][0]
        for i, at in enumerate(path):                                # ascending: no row is overwritten before it is read
            (to_page, to), (from_page, frm) = divmod(old + i, c["page"]), divmod(old + at, c["page"])
            for cache in (k, v):
                cache[table[b][to_page], to] = cache[table[b][from_page], frm]
    return {"k_cache": k, "v_cache": v, "lengths_out": None}


def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "select": _exact_select, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](s, s["case"])
