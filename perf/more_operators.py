"""What the speed of attention with a sliding window and of the cache in 8 bits is
measured on: prompts and single tokens that see their last keys and a few first ones,
and a paged cache whose keys and values are held in e4m3 with a scale for each 16
tokens of a head, filled, read, forked and grown.

A case is a dict of plain values:

  op         what one pass calls
               prompt    Context.attention over packed sequences, with a window
               token     Context.cache_attention: one new token of every sequence
               fill      Context.cache_append of prompts to empty sequences, which cache_trim frees again
               step      cache_append of one token of every sequence, cache_attention, and
                         cache_trim back to the lengths before (a draft that was not taken)
               beams     cache_fork of every source to `beams` others, one token appended to each
                         of them all, cache_attention, and cache_trim of what was added
  bits       (but prompt) 16, or 8: what an element of the cache is held in
  dtype      type of queries, of keys and values that are appended, and of results
  window, sinks   a query sees the last `window` keys up to its own, and the first `sinks`;
             window 0: all up to its own
  seqs       sequences of a call
  shortest, longest   their lengths (of the new tokens where op is prompt), over a logarithmic scale
  cached     (prompt) most keys that a sequence has before its first new token; 0: none has any
  heads, kv_heads, dim   heads of the queries, of keys and values, and elements of a head
  lse        whether the log-sum-exp of each row is wanted
  page       tokens of a page
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DEV = "cuda:0"
_E4M3 = torch.float8_e4m3fn
_BLOCK = 16                                                          # tokens that share a scale
_PLAIN = dict(op="prompt", bits=16, dtype="bfloat16", window=0, sinks=0, seqs=1, shortest=1, longest=1, cached=0, heads=8,
              kv_heads=8, dim=64, lse=False, page=16, beams=0)


def _case(name, **kw):
    return dict(_PLAIN, name=name, **kw)


def listed():
    return [
        # short prompts of a small model that attends to its near past: latency
        _case("prompt_4x128", window=64, sinks=4, seqs=4, shortest=128, longest=128, heads=12, kv_heads=12),
        # the prompts of a batch, packed, short ones beside long ones; rows' log-sum-exp kept
        _case("prompt_ragged", window=512, sinks=4, seqs=31, shortest=1, longest=3300, heads=16, kv_heads=4, dim=128, lse=True),
        # pieces of long prompts whose first parts are cached already, an odd window, heads of an uncommon width
        _case("prompt_pieces", window=1001, sinks=1, seqs=5, shortest=60, longest=1021, cached=9001, heads=20, kv_heads=4,
              dim=96, dtype="float16"),
        # one long document under a wide window
        _case("prompt_14k", window=4096, sinks=4, shortest=14001, longest=14001, heads=32, kv_heads=8, dim=128),
        # one user's next token in a long chat: latency
        _case("token_1x5k", op="token", window=1024, sinks=4, shortest=5003, longest=5003, heads=12, kv_heads=12),
        # a busy server's next tokens, from chats just begun to whole documents
        _case("token_96", op="token", window=4096, sinks=4, seqs=96, shortest=1, longest=20001, heads=32, kv_heads=8, dim=128,
              page=32),
        # one user's next token over a cache in 8 bits: latency
        _case("token8_1x700", op="token", bits=8, shortest=700, longest=700, heads=12, kv_heads=12),
        # a busy server's, over a cache in 8 bits
        _case("token8_64", op="token", bits=8, seqs=64, shortest=1, longest=16001, heads=32, kv_heads=8, dim=128, page=32),
        # two very long contexts that fit because they are held in 8 bits
        _case("token8_2x500k", op="token", bits=8, seqs=2, shortest=499_999, longest=502_000, heads=40, kv_heads=8, dim=128,
              page=64, dtype="float16"),
        # prompts that come in: rounded to 8 bits on their way into the pages
        _case("fill8_50", op="fill", bits=8, seqs=50, shortest=200, longest=3100, heads=32, kv_heads=8, dim=128, page=32),
        # a draft's token over a window, appended, attended and taken back
        _case("step8_200", op="step", bits=8, window=1024, sinks=4, seqs=200, shortest=400, longest=2600, heads=16, kv_heads=16),
        # beam search: each source forked to five beams, part-filled pages copied
        _case("beams8_8x5", op="beams", bits=8, seqs=8, beams=5, shortest=300, longest=2000, heads=32, kv_heads=8, dim=128,
              page=32, dtype="float16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    c = dict(_PLAIN)
    c["op"] = rng.choice(["prompt", "prompt", "prompt", "token", "token", "token", "fill", "step", "step", "beams"])
    c["dtype"] = rng.choice(["bfloat16", "bfloat16", "float16"])
    c["kv_heads"], group = rng.choice([(1, 1), (1, 7), (2, 4), (4, 4), (4, 5), (8, 4), (8, 5), (12, 1), (8, 1), (16, 1), (3, 2), (2, 12)])
    c["heads"] = c["kv_heads"] * group
    c["dim"] = rng.choice([64, 64, 128, 128, 128, 32, 80, 96])
    c["page"] = rng.choice([16, 16, 32, 64, 128])
    if c["op"] != "prompt":
        c["bits"] = 8 if c["op"] == "fill" else rng.choice([8, 8, 16])
    if c["op"] != "fill" and (c["bits"] == 16 or rng.random() < 0.4):
        c["window"] = _log_int(rng, 1, 8000)
        c["sinks"] = rng.choice([0, 1, 4, 4, 16, 130])
    if c["op"] == "prompt":
        c["seqs"] = _log_int(rng, 1, 48)
        # scores of a padded batch are what the plain form holds
        most = int(math.sqrt(1.2e9 / (c["seqs"] * c["heads"])))
        c["longest"] = _log_int(rng, 16, min(most, 8000))
        c["shortest"] = rng.choice([1, c["longest"], max(1, c["longest"] // 3)])
        c["lse"] = rng.random() < 0.4
        if rng.random() < 0.35:
            c["cached"] = _log_int(rng, 16, max(17, most * most // c["longest"]))
    elif c["op"] == "token":
        c["seqs"] = _log_int(rng, 1, 300)
        most = int(6e8 / (c["seqs"] * c["kv_heads"] * c["dim"]))
        c["longest"] = _log_int(rng, 16, min(most, 300_000))
        c["shortest"] = rng.choice([1, c["longest"], max(1, c["longest"] // 3)])
    else:
        c["seqs"] = _log_int(rng, 1 if c["op"] == "fill" else 4, 40 if c["op"] == "beams" else 300)
        c["beams"] = rng.randint(1, 6) if c["op"] == "beams" else 0
        most = int(1.5e8 / (c["seqs"] * (1 + c["beams"]) * c["kv_heads"] * c["dim"]))
        c["longest"] = _log_int(rng, 20, max(20, min(most, 6000)))
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


def _pool(gen, dtype, case, pages, shift):
    """Pages as appending left them, and their scales (None in 16 bits)."""
    G, D, page = case["kv_heads"], case["dim"], case["page"]
    if case["bits"] == 16:
        return _rows(gen, dtype, pages * page, G, D, 1.0, shift).view(pages, page, G, D).transpose(1, 2).contiguous(), None
    codes = torch.empty((pages, G, page, D), dtype=_E4M3, device=_DEV)
    scales = torch.empty((pages, G, page // _BLOCK), dtype=torch.float32, device=_DEV)
    lean = torch.randn((1, G, 1, 1, D), generator=gen, device=_DEV) * shift
    per = max(1, (1 << 26) // (G * page * D))
    for at in range(0, pages, per):
        m = min(per, pages - at)
        x = (torch.randn((m, G, page // _BLOCK, _BLOCK, D), generator=gen, device=_DEV) + lean).to(dtype).float()
        s = _need(x.abs().amax((3, 4)))
        codes[at:at + m] = _code(x / s[..., None, None]).view(m, G, page, D)
        scales[at:at + m] = s
    return codes, scales


def prepare(case, seed):
    """A call's tensors, a cache with its sequences where the case has one, and a context."""
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(seed)
    dtype = getattr(torch, case["dtype"])
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    n, before = _lengths(case)
    st = dict(case=case, scale=1.0 / math.sqrt(D))
    if case["op"] == "prompt":
        st.update(q=_rows(gen, dtype, int(n.sum()), H, D, 1.5), k=_rows(gen, dtype, int((n + before).sum()), G, D, 1.0, 0.5),
                  v=_rows(gen, dtype, int((n + before).sum()), G, D), q_offsets=_offsets(n),
                  k_offsets=_offsets(n + before), max_q=int(n.max()), max_k=int((n + before).max()))
    else:
        rs = np.random.RandomState(seed % (2**32 - 1))
        page, S, fill = case["page"], case["seqs"] * (1 + case["beams"]), case["op"] == "fill"
        per_seq = _pages_of(int(n.max()) + 1, page)
        need = int(_pages_of(n, page).sum())
        pool = need + S + 3                                          # a new page for every sequence
        place = rs.permutation(pool)[:need].astype(np.int32)
        table = np.full((S, per_seq), -1, np.int32)
        refs, length = np.zeros(pool, np.int32), np.zeros(S, np.int32)
        if fill:
            refs[rs.permutation(pool)[:S]] = 1                       # held by sequences that are not of this call
        else:
            at = 0
            for b in range(case["seqs"]):
                m = int(_pages_of(int(n[b]), page))
                table[b, :m] = place[at:at + m]
                at += m
            refs[place] = 1
            length[:case["seqs"]] = n
        up = lambda a: torch.tensor(a, device=_DEV)  # noqa: E731
        (kp, ks), (vp, vs) = (_pool(gen, dtype, case, pool, shift) for shift in (0.5, 0.0))
        st.update(k_pages=kp, v_pages=vp, k_scales=ks, v_scales=vs, table=up(table), length=up(length), refs=up(refs), page=page,
                  low=torch.zeros(1, dtype=torch.int32, device=_DEV), seqs=torch.arange(S, dtype=torch.int32, device=_DEV))
        if not fill:
            st["q"] = _rows(gen, dtype, S, H, D, 1.5)
        if case["op"] != "token":
            new = n if fill else np.ones(S, np.int64)
            st.update(k=_rows(gen, dtype, int(new.sum()), G, D, 1.0, 0.5), v=_rows(gen, dtype, int(new.sum()), G, D),
                      offsets=_offsets(new), back=up(length), most_new=int(new.max()))
        if case["op"] == "beams":
            # beam j of source b is sequence seqs + b * beams + j; after the pass the sources are as before
            st["src"] = up(np.repeat(np.arange(case["seqs"], dtype=np.int32), case["beams"]))
            st["dst"] = up(np.arange(case["seqs"], S, dtype=np.int32))
    if own:
        import paper_2609_11938_gb300 as opa
        st["ctx"] = opa.Context(0)
        if case["op"] != "prompt":
            more = dict(k_scales=st["k_scales"], v_scales=st["v_scales"]) if case["bits"] == 8 else {}
            st["cache"] = opa.KVCache(st["k_pages"], st["v_pages"], st["table"], st["length"], st["refs"], st["low"], **more)
    return st


# ---------------------------------------------------------------- one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _state_of(st):
    return {x: st[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales", "table", "length", "refs")}


def _run_own(st):
    ctx, c = st["ctx"], st["case"]
    seen = dict(window=c["window"], sinks=c["sinks"]) if c["window"] else {}
    if c["op"] == "prompt":
        _, out, lse = ctx.attention(st["q"], st["k"], st["v"], st["q_offsets"], st["k_offsets"], scale=st["scale"],
                                    need_lse=c["lse"], **seen)
        return dict(out=out, lse=lse)
    cache = st["cache"]
    if c["op"] == "token":
        _, out, lse = ctx.cache_attention(cache, st["seqs"], st["q"], scale=st["scale"], need_lse=c["lse"], **seen)
        return dict(out=out, lse=lse)
    if c["op"] == "beams":
        ctx.cache_fork(cache, st["src"], st["dst"])
    ctx.cache_append(cache, st["seqs"], st["offsets"], st["k"], st["v"])
    out = None
    if c["op"] != "fill":
        _, out, _ = ctx.cache_attention(cache, st["seqs"], st["q"], scale=st["scale"], **seen)
    ctx.cache_trim(cache, st["seqs"], st["back"])
    return dict(_state_of(st), out=out)


# the plain forms: torch operations over padded batches, 32 bits
def _run_plain(st):
    c = st["case"]
    if c["op"] == "prompt":
        return _plain_prompt(st)
    if c["op"] == "token":
        return _plain_token(st)
    if c["op"] == "beams":
        _plain_fork(st, st["src"], st["dst"])
    _plain_append(st)
    out = _plain_token(st)["out"] if c["op"] != "fill" else None
    _plain_trim(st, st["seqs"], st["back"])
    return dict(_state_of(st), out=out)


def _near(case, key, pos):
    """Whether a query at `pos` sees a key: one of the last ones, or of the first."""
    seen = key <= pos
    return seen & ((key > pos - case["window"]) | (key < case["sinks"])) if case["window"] else seen


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
    seen = (ik < lk[:, None])[:, None, :] & _near(st["case"], ik, iq[:, None] + (lk - lq)[:, None, None])
    p, total, lse = _softmax_rows(s, seen[:, None, None])
    o = torch.matmul(p.view(len(lq), G, -1, len(ik)), V).view(len(lq), G, H // G, len(iq), D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    row = torch.arange(q.shape[0], device=_DEV)
    b = torch.searchsorted(qo[1:], row, right=True)
    i = row - qo[b]
    out = o.reshape(len(lq), H, len(iq), D)[b, :, i].to(q.dtype)
    return dict(out=out, lse=lse.reshape(len(lq), H, len(iq))[b, :, i] if st["case"]["lse"] else None)


def _values(st, which, pages):
    """What the pages stand for, in 32 bits: [.., G, page, D]."""
    x, s = st[which + "_pages"], st[which + "_scales"]
    if s is None:
        return x[pages].float()
    y = x.view(torch.uint8)[pages].view(_E4M3).float()
    return y.unflatten(-2, (-1, _BLOCK)).mul_(s[pages][..., None, None]).flatten(-3, -2)


def _plain_token(st):
    q, table, length = st["q"], st["table"][st["seqs"].long()].long(), st["length"][st["seqs"].long()].long()
    G, _, D = st["k_pages"].shape[1:]
    B, H = q.shape[:2]
    get = lambda x: _values(st, x, table.clamp(min=0)).permute(0, 2, 1, 3, 4).reshape(B, G, -1, D)  # noqa: E731
    s = torch.matmul(q.float().view(B, G, H // G, D), get("k").transpose(2, 3)).mul_(st["scale"])
    seen = _near(st["case"], torch.arange(s.shape[-1], device=_DEV), length[:, None] - 1)
    p, total, lse = _softmax_rows(s, seen[:, None, None])
    o = torch.matmul(p, get("v"))
    out = torch.where(total > 0, o / total, torch.zeros_like(o)).view(B, H, D).to(q.dtype)
    return dict(out=out, lse=lse.reshape(B, H) if st["case"]["lse"] else None)


def _need(top):
    """The least power of two, from 2^-126 to 2^119, that takes a block's largest element to 448 at most."""
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 9 + (m > 0.875).int(), -126).clamp_(-126, 119)
    return ((e + 127) << 23).view(torch.float32)


def _code(x):
    return torch.where(torch.isfinite(x), x.clamp(-448.0, 448.0), math.nan).to(_E4M3)


def _plain_append(st):
    """New rows of `seqs`, one sequence after another: a partly filled page that others hold too is
    copied first, and pages are taken from the lowest free ones on."""
    table, length, refs, page = st["table"], st["length"], st["refs"], st["page"]
    s, off = st["seqs"].long(), st["offsets"].long()
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
    to = table[s[c]].gather(1, (have[c] - 1)[:, None])[:, 0].long()
    filled = (old[c] % page)[:, None]
    keep = torch.arange(page, device=_DEV) < filled
    length[s] += new.int()
    for x in ("k", "v"):
        pages, scales = st[x + "_pages"].view(torch.uint8 if st["case"]["bits"] == 8 else st[x].dtype), st[x + "_scales"]
        pages[to] = torch.where(keep[:, None, :, None], pages[last[c]], pages[to])
        if scales is None:
            row = torch.arange(st[x].shape[0], device=_DEV)
            b = torch.searchsorted(off[1:], row, right=True)
            pos = old[b] + row - off[b]
            pages[table[s[b], pos // page].long(), :, pos % page] = st[x]
        else:
            some = torch.arange(page // _BLOCK, device=_DEV) * _BLOCK < filled
            scales[to] = torch.where(some[:, None], scales[last[c]], scales[to])
            _plain_round(st, pages, scales, st[x], s, off, old, new)


def _plain_round(st, pages, scales, rows, s, off, old, new):
    """Rows into pages of 8 bits, 16 tokens of a head to a scale; a scale that grows takes the codes before it along."""
    page = st["page"]
    block = old[:, None] // _BLOCK + torch.arange((st["most_new"] + 2 * _BLOCK - 2) // _BLOCK, device=_DEV)
    block = block.clamp(max=(old + new - 1).clamp(min=0)[:, None] // _BLOCK)       # (the last one again: the same stores)
    pos = block[..., None] * _BLOCK + torch.arange(_BLOCK, device=_DEV)
    at = (off[:-1, None, None] + pos - old[:, None, None])
    mine = (pos >= old[:, None, None]) & (pos < (old + new)[:, None, None])
    x = rows[at.clamp(0, rows.shape[0] - 1)].float().permute(0, 1, 3, 2, 4)         # [n, blocks, G, 16, D]
    mine = mine[:, :, None, :, None].expand_as(x)
    need = _need(torch.where(mine & torch.isfinite(x), x.abs(), 0.0).amax((3, 4)))
    where, sub = table_at(st, s, block * _BLOCK // page), block * _BLOCK % page // _BLOCK
    all_codes = pages.unflatten(2, (-1, _BLOCK))
    was, codes = scales[where, :, sub], all_codes[where, :, sub].view(_E4M3).float()
    held = (block * _BLOCK < old[:, None])[..., None]
    now = torch.where(held, torch.maximum(was, need), need)
    moved = _code(codes * (was / now)[..., None, None])
    before = (pos < old[:, None, None])[:, :, None, :, None] & (was < now)[..., None, None]
    got = torch.where(mine, _code(x / now[..., None, None]).view(torch.uint8),
                      torch.where(before, moved.view(torch.uint8), all_codes[where, :, sub]))
    live = (new > 0)[:, None].expand_as(block)
    all_codes[where[live], :, sub[live]] = got[live]
    scales[where[live], :, sub[live]] = now[live]


def table_at(st, s, j):
    return st["table"][s].long().gather(1, j).clamp(min=0)


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


# ---------------------------------------------------------------- what a pass cannot do without
def _seen_of(case, pos):
    """How many keys the queries at `pos` see."""
    w, s = case["window"], case["sinks"]
    return np.minimum(pos + 1, w + np.clip(pos + 1 - w, 0, s)) if w else pos + 1


def work(case):
    n, before = _lengths(case)
    H, G, D, S = case["heads"], case["kv_heads"], case["dim"], case["seqs"] * (1 + case["beams"])
    if case["op"] == "prompt":
        pairs = sum(int(_seen_of(case, np.arange(b, b + m)).sum()) for m, b in zip(n, before))
        keys = int((n - 1 + _seen_of(case, before)).sum())           # those that any query sees
        b = 2 * D * (2 * H * int(n.sum()) + 2 * G * keys) + 8 * (len(n) + 1)
        return {"bytes": b + (4 * H * int(n.sum()) if case["lse"] else 0), "flops": 4 * D * H * pairs}
    # bytes of a token's key and value, and of the same as they come in
    row, given = (4 * G * D if case["bits"] == 16 else 2 * G * D + 8 * G / _BLOCK), 4 * G * D
    if case["op"] == "fill":
        return {"bytes": int((row + given) * int(n.sum()) + 12 * int(_pages_of(n, case["page"]).sum())), "flops": 0}
    more = 0 if case["op"] == "token" else 1                         # the new token
    seen = _seen_of(case, n + more - 1)
    # forked sequences read what they share once
    b = row * (int(seen.sum()) + (S - case["seqs"]) * more) + 4 * H * D * S + 4 * int(_pages_of(seen, case["page"]).sum())
    b += more * (row + given) * S
    if case["op"] == "beams":
        b += 2 * row * int((n % case["page"]).sum()) * case["beams"] + 8 * int(_pages_of(n, case["page"]).sum()) * case["beams"]
    return {"bytes": int(b), "flops": 4 * D * H * int(seen.sum()) * (1 + case["beams"])}


# ---------------------------------------------------------------- the same from the definition, 64 bits
def _exact_rows(case, q, k, v, scale, first):
    """Attention of q [n, H, D] over k, v [m, G, D]; query i stands at first + i."""
    n, H, D = q.shape
    m, G = k.shape[:2]
    W, S = case["window"] or 1 << 40, case["sinks"]
    out = torch.zeros((n, H, D), dtype=torch.float64, device=_DEV)
    lse = torch.full((n, H), -math.inf, dtype=torch.float64, device=_DEV)
    for at in range(0, n, 1024):
        end = min(at + 1024, n)
        lo, top = max(0, first + at - W + 1), min(m, first + end)
        if top <= 0:
            continue
        place = torch.cat([torch.arange(min(S, lo), device=_DEV), torch.arange(lo, top, device=_DEV)])
        p = first + torch.arange(at, end, device=_DEV)[:, None]
        hidden = (place > p) | ((place <= p - W) & (place >= S))
        for h in range(H):
            K, V = k[place, h * G // H].double(), v[place, h * G // H].double()
            x = (scale * (q[at:end, h].double() @ K.T)).masked_fill_(hidden, -math.inf)
            lse[at:end, h] = torch.logsumexp(x, 1)
            some = (lse[at:end, h] > -math.inf)[:, None]
            out[at:end, h] = torch.where(some, torch.exp(x - torch.where(some, lse[at:end, h, None], 0.0)) @ V, 0.0)
    return out, lse


def _exact_append(codes, scales, have, x):
    """A head's codes [have, D] and scales, as numbers, and rows x [n, D] after them, block by block:
    all codes (in units of their scale, as the sums of attention take them) and scales."""
    n = x.shape[0]
    codes, scales = codes[:have].double(), scales[:-(-have // _BLOCK)].double()
    total = have + n
    blocks = -(-total // _BLOCK)
    got = torch.zeros((blocks * _BLOCK, x.shape[1]), dtype=torch.float64, device=_DEV)
    got[:have], got[have:total] = codes, x.double()
    fresh = torch.zeros(blocks * _BLOCK, dtype=torch.bool, device=_DEV)
    fresh[have:total] = True
    top = torch.where(fresh[:, None], got.abs(), 0.0).view(blocks, -1).amax(1)
    s = torch.exp2((torch.log2(top / 448).round() - 1).clamp(-126, 119))
    s = torch.where(448 * s < top, 2 * s, s)
    s = torch.where(448 * s < top, 2 * s, s).clamp(max=2.0 ** 119)
    was = torch.zeros(blocks, dtype=torch.float64, device=_DEV)
    was[:len(scales)] = scales
    now = torch.where((torch.arange(blocks, device=_DEV) * _BLOCK >= have), s, torch.where(fresh.view(blocks, -1).any(1), torch.maximum(was, s), was))
    each = now.repeat_interleave(_BLOCK)[:, None]
    got = torch.where(fresh[:, None], got / each, got * was.repeat_interleave(_BLOCK)[:, None] / each)
    return got[:total].to(torch.float32).to(_E4M3).double(), now


def exact(case, seed):
    n, before = _lengths(case)
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "fill" and case["seqs"] * G > 500:
        return None
    if 4 * D * H * int((n * (n + before) if case["op"] == "prompt" else n).sum()) > 6e12:
        return None
    st = prepare(case, seed)
    if case["op"] == "prompt":
        qo, ko = st["q_offsets"].tolist(), st["k_offsets"].tolist()
        got = [_exact_rows(case, st["q"][qo[b]:qo[b + 1]], st["k"][ko[b]:ko[b + 1]], st["v"][ko[b]:ko[b + 1]], st["scale"], int(before[b]))
               for b in range(case["seqs"])]
        return dict(out=torch.cat([o for o, _ in got]), lse=torch.cat([x for _, x in got]) if case["lse"] else None)
    nothing = {x: None for x in ("k_pages", "v_pages", "k_scales", "v_scales", "table", "length", "refs")}
    table, length, out, lse = st["table"].tolist(), st["length"].tolist(), [], []
    if case["op"] == "fill":
        # sequence after sequence takes the lowest free pages
        free, off = [i for i, r in enumerate(st["refs"].tolist()) if r == 0], st["offsets"].tolist()
        for x in ("k", "v"):
            pages, scales, at = st[x + "_pages"].to(torch.float64), st[x + "_scales"].double(), 0
            for b in range(case["seqs"]):
                m = off[b + 1] - off[b]
                mine = torch.tensor(free[at:at + _pages_of(m, st["page"])], device=_DEV)
                at += len(mine)
                for g in range(G):
                    c, s = _exact_append(pages[:0, 0, 0], scales[:0, 0, 0], 0, st[x][off[b]:off[b + 1], g])
                    t = torch.arange(m, device=_DEV)
                    pages[mine[t // st["page"]], g, t % st["page"]] = c
                    t = torch.arange(len(s), device=_DEV) * _BLOCK
                    scales[mine[t // st["page"]], g, t % st["page"] // _BLOCK] = s
            nothing[x + "_pages"], nothing[x + "_scales"] = pages, scales
        return dict(nothing, out=None)
    for b in range(len(length)):
        held = b if b < case["seqs"] else (b - case["seqs"]) // case["beams"]         # the source of a beam
        at = torch.tensor([p for p in table[held] if p >= 0], dtype=torch.long, device=_DEV)
        rows = []
        for x in ("k", "v"):
            y = st[x + "_pages"].view(torch.uint8 if case["bits"] == 8 else st["q"].dtype)[at].transpose(1, 2).reshape(-1, G, D)[:length[held]]
            if case["bits"] == 8:
                s = st[x + "_scales"][at].transpose(1, 2).reshape(-1, G)
                y = y.contiguous().view(_E4M3).to(torch.float32)
                if case["op"] == "token":
                    y = y.double() * s.double().repeat_interleave(_BLOCK, 0)[:length[held], :, None]
                else:
                    full = length[held] // _BLOCK * _BLOCK                            # blocks that stay
                    z = [y[:full].double() * s.double().repeat_interleave(_BLOCK, 0)[:full, :, None]]
                    ends = [_exact_append(y[full:, g], s[full // _BLOCK:, g], length[held] - full, st[x][b:b + 1, g]) for g in range(G)]
                    z.append(torch.stack([c * w for c, w in ends], 1))
                    y = torch.cat(z)
            elif case["op"] != "token":
                y = torch.cat([y, st[x][b:b + 1]])
            rows.append(y)
        o, x = _exact_rows(case, st["q"][b:b + 1], rows[0], rows[1], st["scale"], len(rows[0]) - 1)
        out.append(o)
        lse.append(x)
    if case["op"] == "token":
        return dict(out=torch.cat(out), lse=torch.cat(lse) if case["lse"] else None)
    return dict(nothing, out=torch.cat(out))
