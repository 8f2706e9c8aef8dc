"""What the speed of the attention operators and of the paged cache under them is
measured on: prompts in one call, single new tokens over a paged cache, and the
steps that a serving loop makes with both.

A case is a dict of plain values:

  op         what one pass calls
               prompt    Context.attention over packed sequences
               token     Context.cache_attention: one new token of every sequence
               step      cache_append of one token of every sequence, cache_attention, and
                         cache_trim back to the lengths before (a draft that was not taken)
               beams     cache_fork of every source to `beams` others, one token appended to each
                         of them all, cache_attention, and cache_trim of what was added
               turnover  one group of sequences in `groups` is freed (cache_trim to nothing), the
                         cache compacted, and the group's next prompts appended (cache_append)
  dtype      type of queries, keys and values
  seqs       sequences of a call
  shortest, longest   their lengths (of the new tokens where op is prompt), over a logarithmic scale
  cached     (prompt) most keys that a sequence has before its first new token; 0: none has any
  heads, kv_heads, dim   heads of the queries, of keys and values, and elements of a head
  causal, lse   (prompt) mask, and whether the log-sum-exp of each row is wanted
  page       tokens of a page
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DEV = "cuda:0"
_PLAIN = dict(op="prompt", dtype="bfloat16", seqs=1, shortest=1, longest=1, cached=0, heads=8, kv_heads=8, dim=64,
              causal=True, lse=False, page=16, beams=0, groups=1)


def _case(name, **kw):
    return dict(_PLAIN, name=name, **kw)


def listed():
    return [
        # one forward pass of a layer of the small language model that the paper profiles: four prompts of 128
        _case("prompt_4x128", seqs=4, shortest=128, longest=128, heads=12, kv_heads=12),
        # the paper's attention workload: eight sequences of 512, eight heads, every key visible
        _case("prompt_8x512", seqs=8, shortest=512, longest=512, causal=False, dtype="float16"),
        # the prompts of a batch, packed, short ones beside long ones; rows' log-sum-exp kept
        _case("prompt_ragged", seqs=37, shortest=1, longest=2500, heads=16, kv_heads=4, dim=128, lse=True),
        # pieces of long prompts whose first parts are cached already, heads of an uncommon width
        _case("prompt_pieces", seqs=5, shortest=60, longest=1021, cached=9001, heads=20, kv_heads=4, dim=96,
              dtype="float16"),
        # one long document
        _case("prompt_12k", shortest=12301, longest=12301, heads=32, kv_heads=8, dim=128),
        # one user's next token: latency
        _case("token_1x700", op="token", shortest=700, longest=700, heads=12, kv_heads=12),
        # a busy server's next tokens, from chats just begun to whole documents
        _case("token_64", op="token", seqs=64, shortest=1, longest=16001, heads=32, kv_heads=8, dim=128, page=32),
        # two very long contexts
        _case("token_2x260k", op="token", seqs=2, shortest=259_999, longest=262_000, heads=40, kv_heads=8, dim=128,
              page=64, dtype="float16"),
        # a draft's token, appended, attended and taken back
        _case("step_200", op="step", seqs=200, shortest=400, longest=2600, heads=16, kv_heads=16),
        # beam search: each source forked to five beams
        _case("beams_8x5", op="beams", seqs=8, beams=5, shortest=300, longest=2000, heads=32, kv_heads=8, dim=128,
              page=32),
        # a small server whose chats end and begin
        _case("turnover_24", op="turnover", seqs=24, groups=4, shortest=20, longest=300, heads=12, kv_heads=12),
        # a large one
        _case("turnover_400", op="turnover", seqs=400, groups=8, shortest=200, longest=3100, heads=32, kv_heads=8,
              dim=128, page=32),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    c = dict(_PLAIN)
    c["op"] = rng.choice(["prompt", "prompt", "prompt", "token", "token", "step", "beams", "turnover"])
    c["dtype"] = rng.choice(["bfloat16", "bfloat16", "float16"])
    c["kv_heads"], group = rng.choice([(1, 1), (1, 7), (2, 4), (4, 4), (4, 5), (8, 4), (8, 5), (12, 1), (8, 1), (16, 1), (3, 2)])
    c["heads"] = c["kv_heads"] * group
    c["dim"] = rng.choice([64, 64, 128, 128, 128, 32, 80, 96])
    c["page"] = rng.choice([16, 16, 32, 64, 128])
    if c["op"] == "prompt":
        c["seqs"] = _log_int(rng, 1, 48)
        # scores of a padded batch are what the plain form holds
        most = int(math.sqrt(1.2e9 / (c["seqs"] * c["heads"])))
        c["longest"] = _log_int(rng, 16, min(most, 8000))
        c["shortest"] = rng.choice([1, c["longest"], max(1, c["longest"] // 3)])
        c["causal"] = rng.random() < 0.75
        c["lse"] = rng.random() < 0.4
        if rng.random() < 0.35:
            c["cached"] = _log_int(rng, 16, max(17, most * most // c["longest"]))
    elif c["op"] == "token":
        c["seqs"] = _log_int(rng, 1, 300)
        most = int(6e8 / (c["seqs"] * c["kv_heads"] * c["dim"]))
        c["longest"] = _log_int(rng, 16, min(most, 300_000))
        c["shortest"] = rng.choice([1, c["longest"], max(1, c["longest"] // 3)])
    else:
        c["seqs"] = _log_int(rng, 4, 40 if c["op"] == "beams" else 300)
        c["beams"] = rng.randint(1, 6) if c["op"] == "beams" else 0
        c["groups"] = rng.choice([2, 3, 4, 8]) if c["op"] == "turnover" else 1
        c["seqs"] = max(c["seqs"], c["groups"])
        most = int(4e8 / (c["seqs"] * (1 + c["beams"]) * c["kv_heads"] * c["dim"]))
        c["longest"] = _log_int(rng, 20, min(most, 6000))
        c["shortest"] = rng.choice([1, max(1, c["longest"] // 4)])
    return c


# ---------------------------------------------------------------- inputs
def _lengths(case):
    """Lengths of the sequences (of the new tokens), and keys before them: the case's alone."""
    rs = np.random.RandomState((case["seqs"] * 7919 + case["longest"] * 31 + case["heads"]) % (2**31))
    lo, hi = math.log(case["shortest"]), math.log(case["longest"])
    n = np.rint(np.exp(rs.uniform(lo, hi, case["seqs"]))).astype(np.int64).clip(case["shortest"], case["longest"])
    n[rs.randint(case["seqs"])] = case["longest"]
    before = rs.randint(case["cached"] // 4, case["cached"] + 1, case["seqs"]) if case["cached"] else np.zeros_like(n)
    return n, before.astype(np.int64)


def _offsets(n):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(_DEV)


def _rows(gen, dtype, n, heads, dim, spread=1.0, shift=0.0):
    """Rows as a projection gives them: unit-sized, with channels that lean to one side."""
    lean = torch.randn((1, heads, dim), generator=gen, device=_DEV) * shift
    x = torch.empty((n, heads, dim), dtype=dtype, device=_DEV)
    per = max(1, (1 << 26) // (heads * dim))
    for at in range(0, n, per):
        m = min(per, n - at)
        x[at:at + m] = torch.randn((m, heads, dim), generator=gen, device=_DEV) * spread + lean
    return x


def _pages_of(n, page):
    return -(-n // page)


def prepare(case, seed):
    """A call's tensors, a cache with its sequences where the case has one, and a context."""
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(seed)
    dtype = getattr(torch, case["dtype"])
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    n, before = _lengths(case)
    st = dict(case=case, scale=1.0 / math.sqrt(D), turn=0)
    if case["op"] == "prompt":
        st.update(q=_rows(gen, dtype, int(n.sum()), H, D, 1.5), k=_rows(gen, dtype, int((n + before).sum()), G, D, 1.0, 0.5),
                  v=_rows(gen, dtype, int((n + before).sum()), G, D), q_offsets=_offsets(n),
                  k_offsets=_offsets(n + before), max_q=int(n.max()), max_k=int((n + before).max()))
    else:
        rs = np.random.RandomState(seed % (2**32 - 1))
        page, S = case["page"], case["seqs"] * (1 + case["beams"])
        per_seq = _pages_of(int(n.max()) + 1, page)
        need = int(_pages_of(n, page).sum())
        # pages beyond those in use: a new one for every sequence, and a group's next prompts
        pool = need + S + (need // 2 if case["op"] == "turnover" else 0) + 3
        place = rs.permutation(pool)[:need].astype(np.int32)
        table = np.full((S, per_seq), -1, np.int32)
        at = 0
        for b in range(case["seqs"]):
            m = int(_pages_of(int(n[b]), page))
            table[b, :m] = place[at:at + m]
            at += m
        refs = np.zeros(pool, np.int32)
        refs[place] = 1
        length = np.zeros(S, np.int32)
        length[:case["seqs"]] = n
        up = lambda a: torch.from_numpy(a).to(_DEV)  # noqa: E731
        pools = [_rows(gen, dtype, pool * page, G, D, 1.0, shift).view(pool, page, G, D).transpose(1, 2).contiguous()
                 for shift in (0.5, 0.0)]
        st.update(k_pages=pools[0], v_pages=pools[1], table=up(table), length=up(length), refs=up(refs), page=page,
                  low=torch.zeros(1, dtype=torch.int32, device=_DEV))
        if case["op"] in ("token", "step", "beams"):
            st.update(q=_rows(gen, dtype, S, H, D, 1.5), seqs=torch.arange(S, dtype=torch.int32, device=_DEV))
        if case["op"] in ("step", "beams"):
            st.update(k=_rows(gen, dtype, S, G, D, 1.0, 0.5), v=_rows(gen, dtype, S, G, D), offsets=_offsets(np.ones(S, np.int64)))
        if case["op"] == "step":
            st["back"] = up(length)
        if case["op"] == "beams":
            # beam j of source b is sequence seqs + b * beams + j; after the pass the sources are as before
            st["src"] = up(np.repeat(np.arange(case["seqs"], dtype=np.int32), case["beams"]))
            st["dst"] = up(np.arange(case["seqs"], S, dtype=np.int32))
            st["back"] = up(length)
        if case["op"] == "turnover":
            which = np.array_split(rs.permutation(S).astype(np.int32), case["groups"])
            st["turns"] = [dict(seqs=up(w), offsets=_offsets(n[w]), k=_rows(gen, dtype, int(n[w].sum()), G, D, 1.0, 0.5),
                                v=_rows(gen, dtype, int(n[w].sum()), G, D)) for w in which]
    if own:
        import paper_2609_11938_gb300 as opa
        st["ctx"] = opa.Context(0)
        if case["op"] != "prompt":
            st["cache"] = opa.KVCache(st["k_pages"], st["v_pages"], st["table"], st["length"], st["refs"], st["low"])
    return st


# ---------------------------------------------------------------- one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _state_of(st):
    return dict(k_pages=st["k_pages"], v_pages=st["v_pages"], table=st["table"], length=st["length"], refs=st["refs"])


def _next_turn(st):
    t = st["turns"][st["turn"] % len(st["turns"])]
    st["turn"] += 1
    return t


def _run_own(st):
    ctx, op = st["ctx"], st["case"]["op"]
    if op == "prompt":
        _, out, lse = ctx.attention(st["q"], st["k"], st["v"], st["q_offsets"], st["k_offsets"],
                                    causal=st["case"]["causal"], scale=st["scale"], need_lse=st["case"]["lse"])
        return dict(out=out, lse=lse)
    cache = st["cache"]
    if op == "token":
        _, out, _ = ctx.cache_attention(cache, st["seqs"], st["q"], scale=st["scale"])
        return dict(out=out)
    if op == "turnover":
        t = _next_turn(st)
        ctx.cache_trim(cache, t["seqs"])
        _, live = ctx.cache_compact(cache)
        ctx.cache_append(cache, t["seqs"], t["offsets"], t["k"], t["v"])
        return dict(_state_of(st), live=live)
    if op == "beams":
        ctx.cache_fork(cache, st["src"], st["dst"])
    ctx.cache_append(cache, st["seqs"], st["offsets"], st["k"], st["v"])
    _, out, _ = ctx.cache_attention(cache, st["seqs"], st["q"], scale=st["scale"])
    ctx.cache_trim(cache, st["seqs"], st["back"])
    return dict(_state_of(st), out=out)


# the plain forms: torch operations over padded batches, 32 bits
def _run_plain(st):
    op = st["case"]["op"]
    if op == "prompt":
        return _plain_prompt(st)
    if op == "token":
        return dict(out=_plain_token(st))
    if op == "turnover":
        t = _next_turn(st)
        _plain_trim(st, t["seqs"], torch.zeros_like(t["seqs"]))
        live = _plain_compact(st)
        _plain_append(st, t["seqs"], t["offsets"], t["k"], t["v"])
        return dict(_state_of(st), live=live)
    if op == "beams":
        _plain_fork(st, st["src"], st["dst"])
    _plain_append(st, st["seqs"], st["offsets"], st["k"], st["v"])
    out = _plain_token(st)
    _plain_trim(st, st["seqs"], st["back"])
    return dict(_state_of(st), out=out)


def _softmax_rows(s, seen):
    """exp of the scores over the seen keys (in place), the rows' sums and the log of them."""
    s.masked_fill_(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    s.sub_(m).exp_()
    total = s.sum(-1, keepdim=True)
    return s, total, (total.log() + m).squeeze(-1)


def _plain_prompt(st):
    q, k, v, qo, ko = st["q"], st["k"], st["v"], st["q_offsets"].long(), st["k_offsets"].long()
    H, G, D = q.shape[1], k.shape[1], q.shape[2]
    lq, lk = qo.diff(), ko.diff()
    iq, ik = torch.arange(st["max_q"], device=_DEV), torch.arange(st["max_k"], device=_DEV)
    at_q = (qo[:-1, None] + iq).clamp_(max=q.shape[0] - 1)
    at_k = (ko[:-1, None] + ik).clamp_(max=k.shape[0] - 1)
    Q = q[at_q].float().view(len(lq), -1, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(len(lq), G, -1, D)
    K = k[at_k].float().permute(0, 2, 3, 1)
    V = v[at_k].float().permute(0, 2, 1, 3)
    s = torch.matmul(Q, K).mul_(st["scale"]).view(len(lq), G, H // G, len(iq), len(ik))
    seen = (ik < lk[:, None])[:, None, :].expand(-1, len(iq), -1)
    if st["case"]["causal"]:
        seen = seen & (ik <= iq[:, None] + (lk - lq)[:, None, None])
    p, total, lse = _softmax_rows(s, seen[:, None, None])
    o = torch.matmul(p.view(len(lq), G, -1, len(ik)), V).view(len(lq), G, H // G, len(iq), D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    row = torch.arange(q.shape[0], device=_DEV)
    b = torch.searchsorted(qo[1:], row, right=True)
    i = row - qo[b]
    out = o.reshape(len(lq), H, len(iq), D)[b, :, i].to(q.dtype)
    return dict(out=out, lse=lse.reshape(len(lq), H, len(iq))[b, :, i] if st["case"]["lse"] else None)


def _plain_token(st):
    q, table, length = st["q"], st["table"][st["seqs"].long()].long(), st["length"][st["seqs"].long()].long()
    G, page, D = st["k_pages"].shape[1:]
    B, H = q.shape[:2]
    get = lambda x: x[table.clamp(min=0)].float().permute(0, 2, 1, 3, 4).reshape(B, G, -1, D)  # noqa: E731
    s = torch.matmul(q.float().view(B, G, H // G, D), get(st["k_pages"]).transpose(2, 3)).mul_(st["scale"])
    seen = torch.arange(s.shape[-1], device=_DEV) < length[:, None]
    p, total, _ = _softmax_rows(s, seen[:, None, None])
    o = torch.matmul(p, get(st["v_pages"]))
    return torch.where(total > 0, o / total, torch.zeros_like(o)).view(B, H, D).to(q.dtype)


def _plain_append(st, seqs, offsets, k, v):
    """New rows of `seqs`, one sequence after another: a partly filled page that others hold too is
    copied first, and pages are taken from the lowest free ones on."""
    table, length, refs, page = st["table"], st["length"], st["refs"], st["page"]
    s, off = seqs.long(), offsets.long()
    old, new = length[s].long(), off.diff()
    have, want = (old + page - 1) // page, (old + new + page - 1) // page
    last = table[s].gather(1, (have - 1).clamp(min=0)[:, None])[:, 0].long()
    part = (old % page != 0) & (new > 0)
    last = torch.where(part, last, -1 - torch.arange(len(s), device=_DEV))
    before = ((last[:, None] == last[None]) & part[None]).tril(-1).sum(1)
    copied = part & (refs[last.clamp(min=0)] - before > 1)
    count = want - have + copied
    first = count.cumsum(0) - count
    free = torch.argsort((refs != 0).to(torch.int8), stable=True)
    taken = torch.arange(len(free), device=_DEV) < count.sum()
    refs.index_add_(0, last.clamp(min=0), -copied.int())
    refs[free] = torch.where(taken, 1, refs[free])
    j = torch.arange(table.shape[1], device=_DEV)
    rank = first[:, None] + torch.where(j == have[:, None] - 1, 0, copied[:, None] + j - have[:, None])
    fresh = ((j >= have[:, None]) & (j < want[:, None])) | ((j == have[:, None] - 1) & copied[:, None])
    table[s] = torch.where(fresh, free[rank.clamp(0, len(free) - 1)].int(), table[s])
    c = copied.nonzero()[:, 0]
    to, keep = table[s[c]].gather(1, (have[c] - 1)[:, None])[:, 0].long(), torch.arange(page, device=_DEV) < (old[c] % page)[:, None]
    row = torch.arange(k.shape[0], device=_DEV)
    b = torch.searchsorted(off[1:], row, right=True)
    pos = old[b] + row - off[b]
    where = table[s[b], pos // page].long()
    length[s] += new.int()
    st["k_pages"][to] = torch.where(keep[:, None, :, None], st["k_pages"][last[c]], st["k_pages"][to])
    st["v_pages"][to] = torch.where(keep[:, None, :, None], st["v_pages"][last[c]], st["v_pages"][to])
    st["k_pages"][where, :, pos % page] = k
    st["v_pages"][where, :, pos % page] = v


def _plain_fork(st, src, dst):
    s, d = src.long(), dst.long()
    rows = st["table"][s]
    st["table"][d] = rows
    st["length"][d] = st["length"][s]
    held = rows >= 0
    st["refs"].index_add_(0, rows.clamp(min=0).flatten().long(), held.int().flatten())


def _plain_trim(st, seqs, lengths):
    s = seqs.long()
    keep = (lengths.long() + st["page"] - 1) // st["page"]
    rows = st["table"][s]
    drop = (torch.arange(rows.shape[1], device=_DEV) >= keep[:, None]) & (rows >= 0)
    st["refs"].index_add_(0, rows.clamp(min=0).flatten().long(), -drop.int().flatten())
    st["table"][s] = torch.where(drop, -1, rows)
    st["length"][s] = lengths


def _plain_compact(st):
    """The live pages past the first `live` ones fill the free ones among these, in order."""
    refs, table = st["refs"], st["table"]
    used = refs > 0
    live = used.sum()
    at = torch.arange(len(refs), device=_DEV)
    hole, last = (~used & (at < live)).nonzero()[:, 0], (used & (at >= live)).nonzero()[:, 0]
    to = at.clone()
    to[last] = hole
    for name in ("k_pages", "v_pages"):
        st[name][hole] = st[name][last]
    refs[hole] = refs[last]
    refs[last] = 0
    st["table"].copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    return live.int().view(1)


# ---------------------------------------------------------------- what a pass cannot do without
def _pairs(case, n, before):
    """Pairs of a query and a key that it sees."""
    if not case["causal"]:
        return int((n * (n + before)).sum())
    return int((n * before + n * (n + 1) // 2).sum())


def work(case):
    n, before = _lengths(case)
    H, G, D, S = case["heads"], case["kv_heads"], case["dim"], case["seqs"] * (1 + case["beams"])
    if case["op"] == "prompt":
        b = 2 * D * (2 * H * int(n.sum()) + 2 * G * int((n + before).sum())) + 8 * (len(n) + 1)
        return {"bytes": b + (4 * H * int(n.sum()) if case["lse"] else 0), "flops": 4 * D * H * _pairs(case, n, before)}
    row, page = 4 * G * D, case["page"]                                      # bytes of a token's key and value
    pages = int(_pages_of(n, page).sum())
    if case["op"] == "turnover":
        # a group's pages leave and as many are filled; as many again move into the gaps
        share = 1.0 / case["groups"]
        return {"bytes": int(share * (2 * row * int(n.sum()) + 2 * row * page * pages) + 4 * pages * (2 + 2 * share)), "flops": 0}
    more = 0 if case["op"] == "token" else 1                                 # the new token
    seen = int((n + more).sum())
    # forked sequences read what they share once
    b = row * (seen + (S - case["seqs"]) * more) + 4 * H * D * S + 4 * pages + more * 2 * row * S
    seen_by = seen * (1 + case["beams"])
    if case["op"] == "beams":
        b += 2 * row * int((n % page).sum()) * case["beams"] + 8 * pages * case["beams"]
    return {"bytes": b, "flops": 4 * D * H * seen_by}


# ---------------------------------------------------------------- the same from the definition, 64 bits
def _exact_rows(q, k, v, scale, first):
    """Attention of q [n, H, D] over k, v [m, G, D], query i over the keys up to first + i."""
    n, H, D = q.shape
    m, G = k.shape[:2]
    out = torch.zeros((n, H, D), dtype=torch.float64, device=_DEV)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64, device=_DEV)
    for g in range(G):
        K, V = k[:, g].double(), v[:, g].double()
        for h in range(g * (H // G), (g + 1) * (H // G)):
            for at in range(0, n, 2048):
                last = min(at + 2048, n)
                top = min(m, first + last)
                if top <= 0:
                    continue
                x = scale * (q[at:last, h].double() @ K[:top].T)
                rows = torch.arange(at, last, device=_DEV)[:, None]
                x = torch.where(torch.arange(top, device=_DEV) <= first + rows, x, -math.inf)
                lse[at:last, h] = torch.logsumexp(x, 1)
                some = lse[at:last, h] > -math.inf
                out[at:last, h] = torch.where(some[:, None], torch.exp(x - torch.where(some, lse[at:last, h], 0.0)[:, None]) @ V[:top], 0.0)
    return out, lse


def exact(case, seed):
    n, before = _lengths(case)
    H, D = case["heads"], case["dim"]
    if case["op"] == "turnover":
        return None                                              # pages are copied, not computed
    if 4 * D * H * int((n * (n + before) if case["op"] == "prompt" else n).sum()) > 6e12:
        return None
    st = prepare(case, seed)
    if case["op"] == "prompt":
        qo, ko = st["q_offsets"].tolist(), st["k_offsets"].tolist()
        got = []
        for b in range(case["seqs"]):
            first = (ko[b + 1] - ko[b]) - (qo[b + 1] - qo[b]) if case["causal"] else 1 << 40
            got.append(_exact_rows(st["q"][qo[b]:qo[b + 1]], st["k"][ko[b]:ko[b + 1]], st["v"][ko[b]:ko[b + 1]], st["scale"], first))
        return dict(out=torch.cat([o for o, _ in got]), lse=torch.cat([x for _, x in got]) if case["lse"] else None)
    table, length, out = st["table"].tolist(), st["length"].tolist(), []
    for b in range(len(length)):
        held = b if b < case["seqs"] else (b - case["seqs"]) // case["beams"]         # the source of a beam
        at = torch.tensor([p for p in table[held] if p >= 0], dtype=torch.long, device=_DEV)
        rows = [st[x][at].transpose(1, 2).reshape(-1, *st[x].shape[1::2])[:length[held]] for x in ("k_pages", "v_pages")]
        if case["op"] != "token":
            rows = [torch.cat([r, st[x][b:b + 1]]) for r, x in zip(rows, "kv")]
        out.append(_exact_rows(st["q"][b:b + 1], rows[0], rows[1], st["scale"], 1 << 40)[0])
    out = torch.cat(out)
    return dict(out=out) if case["op"] == "token" else dict({x: None for x in ("k_pages", "v_pages", "table", "length", "refs")}, out=out)
