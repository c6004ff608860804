"""Verification of drafted tokens, and the pages of a K/V cache, as measurable cases.

What serving needs around the attention over a paged cache: deciding which of a chunk's drafted
tokens hold against the target's logits and drawing the next token, and the pages behind the
sequences: growing rows (a page that rows share is copied before one of them writes it), branching
and trimming and dropping rows, moving pages together.  Each operator in its plain form (elementary
torch operations; the probabilities in 64 bits, because a drawn token depends on which side of a
border a sum lies), as the calls that a program makes of this framework, and from its definition.
"""
import math

import torch

own = False

BT = 16   # positions per block
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # ---- drafted tokens against the target's logits
        # one user of a small decoder (GPT-2-small's vocabulary), four tokens drafted: latency is all there is
        dict(name="verify_one", kind="verify", seqs=1, drafts=4, ragged=False, vocab=50257, target="f32", draft="f32", mode="sample"),
        # eight users, greedy: the drafts have to be the target's own best tokens
        dict(name="verify_greedy", kind="verify", seqs=8, drafts=6, ragged=True, vocab=32000, target="f32", draft="none", mode="greedy"),
        # a serving batch: 16 users of different temperatures (some greedy), none to seven drafts each
        dict(name="verify_batch", kind="verify", seqs=16, drafts=7, ragged=True, vocab=32000, target="f32", draft="bf16", mode="mixed"),
        # drafts looked up in the text so far, without probabilities of their own
        dict(name="verify_lookup", kind="verify", seqs=32, drafts=10, ragged=True, vocab=50257, target="bf16", draft="none", mode="sample"),
        # a large batch over a large vocabulary
        dict(name="verify_wide", kind="verify", seqs=64, drafts=8, ragged=False, vocab=131072, target="f32", draft="bf16", mode="sample"),
        # ---- a round of drafts: rows cut back to what was accepted, and grown for the next drafts
        dict(name="round_few", kind="round", seqs=4, cols=24, blocks=128, step=9),
        # 256 users of up to 32768 positions
        dict(name="round_many", kind="round", seqs=256, cols=2048, blocks=60000, step=9),
        # ---- branches of prompts that stay: rows branch off, grow, and get their own copy of the page they write
        # four samples of one prompt, all layers of a GPT-2-small decoder
        dict(name="branch_samples", kind="branch", kv="bf16", layers=12, kv_heads=12, head_dim=64, prompts=1, branches=4, prompt=333, grow=30, cols=64),
        # eight beams of 16 prompts each, 8-bit cache of a grouped-query decoder
        dict(name="branch_beams", kind="branch", kv="e4m3", layers=8, kv_heads=8, head_dim=128, prompts=16, branches=8, prompt=700, grow=1, cols=128),
        # 32 samples of eight prompts each
        dict(name="branch_wide", kind="branch", kv="bf16", layers=4, kv_heads=32, head_dim=128, prompts=8, branches=32, prompt=1000, grow=20, cols=256),
        # ---- pages moved together
        # a small pool after some users left
        dict(name="compact_few", kind="compact", kv="f32", layers=4, kv_heads=4, head_dim=64, seqs=6, cols=16, blocks=150, held=0.4),
        # a large pool, so that its last part can be given away
        dict(name="compact_pool", kind="compact", kv="bf16", layers=4, kv_heads=32, head_dim=128, seqs=64, cols=128, blocks=4096, held=0.6),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "verify", "round", "branch", "branch", "compact"])
    if kind == "verify":
        vocab = _log_int(rng, 1000, 131072)
        drafts = rng.randint(0, 12)
        seqs = _log_int(rng, 1, max(1, min(128, 64 * 9 * 131072 // (vocab * (drafts + 1)))))
        return dict(kind="verify", seqs=seqs, drafts=drafts, ragged=rng.random() < 0.7, vocab=vocab, target=rng.choice(["f32", "f32", "bf16"]),
                    draft=rng.choice(["f32", "bf16", "none"]), mode=rng.choice(["sample", "sample", "mixed", "greedy"]))
    if kind == "round":
        seqs, cols = _log_int(rng, 1, 512), _log_int(rng, 4, 1000)
        return dict(kind="round", seqs=seqs, cols=cols, blocks=max(8, int(seqs * cols * rng.uniform(0.3, 1.0))), step=rng.randint(1, 40))
    kv, (hk, dh) = rng.choice(["bf16", "e4m3", "f32"]), rng.choice([(12, 64), (32, 128), (8, 128), (2, 32), (25, 64)])
    if kind == "branch":
        prompts, branches = _log_int(rng, 1, 8), _log_int(rng, 1, 24)
        prompt, grow = _log_int(rng, 1, 1500), _log_int(rng, 1, 200)
        return dict(kind="branch", kv=kv, layers=rng.randint(1, 4), kv_heads=hk, head_dim=dh, prompts=prompts, branches=branches, prompt=prompt,
                    grow=grow, cols=(prompt + grow) // BT + 1 + rng.randint(0, 20))
    seqs, cols = _log_int(rng, 1, 64), _log_int(rng, 2, 96)
    return dict(kind="compact", kv=kv, layers=rng.randint(1, 2), kv_heads=hk, head_dim=dh, seqs=seqs, cols=cols,
                blocks=max(8, seqs * cols * rng.randint(5, 10) // 8), held=rng.uniform(0.1, 0.6))


# ---------------------------------------------------------------------------
# the sizes that follow from a case (lengths and rows are the same for every seed)
# ---------------------------------------------------------------------------

def _drafts(case):
    """Drafts per sequence."""
    n, d = case["seqs"], case["drafts"]
    return [(b * 5 + 3) % (d + 1) if case["ragged"] else d for b in range(n)]


def _lengths(case):
    """Round: positions accepted per row (step more are asked for)."""
    most = min(case["cols"] * BT - case["step"], (case["blocks"] // case["seqs"] - 1) * BT - case["step"])
    return [max(0, most * ((b * 7 + 5) % 11 + 3) // 13) for b in range(case["seqs"])]


def _prompts(case):
    return [max(1, case["prompt"] - (37 * b) % max(1, case["prompt"] // 2)) for b in range(case["prompts"])]


def _up(n):
    return (n + BT - 1) // BT


def _block_bytes(case):
    """K and V of a block in one layer."""
    el = case["kv_heads"] * BT * case["head_dim"]
    return 2 * {"f32": 4 * el, "bf16": 2 * el, "e4m3": el + case["kv_heads"] * BT}[case["kv"]]


def _compact_moves(case):
    """Blocks held, and (about: the mean over the draws) blocks to move."""
    held = min(case["blocks"] - 1, case["seqs"] * case["cols"], int(case["blocks"] * case["held"]))
    return held, held * (case["blocks"] - held) // case["blocks"]


def work(case):
    if case["kind"] == "verify":
        d = _drafts(case)
        t, q = sum(d) + len(d), sum(d) if case["draft"] != "none" and case["mode"] != "greedy" else 0
        size = {"f32": 4, "bf16": 2, "none": 0}
        # a maximum, an exponential and a sum for each element
        return {"bytes": case["vocab"] * (t * size[case["target"]] + q * size[case["draft"]]) + 16 * t + 20 * len(d), "flops": 4 * case["vocab"] * (t + q)}
    if case["kind"] == "round":
        # counts read once; the rows' entries behind what stays, read; entries of blocks that change, written
        tail = sum(case["cols"] - _up(n) for n in _lengths(case))
        return {"bytes": 4 * (case["blocks"] + tail + 4 * case["seqs"] * (1 + case["step"] // BT)) + 24 * case["seqs"], "flops": 0}
    if case["kind"] == "branch":
        copies = sum(case["branches"] for n in _prompts(case) if n % BT)
        rows = case["prompts"] * (1 + case["branches"])
        blocks = sum(_up(n) * (1 + case["branches"]) for n in _prompts(case))
        return {"bytes": 2 * copies * case["layers"] * _block_bytes(case) + 4 * (2 * blocks + rows * 8), "flops": 0}
    held, moves = _compact_moves(case)
    return {"bytes": 2 * moves * case["layers"] * _block_bytes(case) + 4 * (2 * case["blocks"] + 2 * held), "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 6271 + 41)
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_verify(case, g):
    d, v = _drafts(case), case["vocab"]
    rows = sum(d) + len(d)
    start = [0]
    for n in d:
        start.append(start[-1] + n + 1)
    # logits as a decoder's: a normal bulk, and a few tokens that stand out
    logits = 2.0 * torch.randn(rows, v, generator=g, device="cuda")
    top = torch.randint(v, (rows, 12), generator=g, device="cuda")
    logits.scatter_add_(1, top, 5.0 + 6.0 * torch.rand(rows, 12, generator=g, device="cuda"))
    near = logits + 0.5 * torch.randn(rows, v, generator=g, device="cuda")   # a draft model's
    # drafts drawn from the draft model (an exponential race); greedy or without probabilities: often the target's best tokens
    if case["mode"] == "greedy" or case["draft"] == "none":
        pick = (logits + 0.3 * torch.randn(rows, v, generator=g, device="cuda")).argmax(1)
    else:
        pick = (near - torch.empty_like(near).exponential_(generator=g).log_()).argmax(1)
    tokens = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), pick[:-1]]).to(torch.int32)
    temp = None
    if case["mode"] == "greedy":
        temp = torch.zeros(len(d), device="cuda")
    elif case["mode"] == "mixed":
        temp = torch.tensor([0.0, 0.7, 1.0, 1.3], device="cuda").repeat(len(d) // 4 + 1)[:len(d)].contiguous()
    return dict(target=logits.to(TYPES[case["target"]]), draft=None if case["draft"] == "none" else near.to(TYPES[case["draft"]]), tokens=tokens,
                start=_i32(start), temp=temp, u=torch.rand(rows, generator=g, device="cuda"),
                logprob=torch.zeros(rows, device="cuda"))


def _fill_rows(case, lens, blocks, g):
    """A table whose rows hold the blocks of lens positions each, scattered over the pool, and the counts."""
    need = [_up(n) for n in lens]
    order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    held = torch.arange(case["cols"], device="cuda")[None, :] < _i32(need)[:, None]
    table = torch.full(held.shape, -1, dtype=torch.int32, device="cuda")
    table[held] = order[:sum(need)]
    ref = torch.zeros(blocks, dtype=torch.int32, device="cuda")
    ref[order[:sum(need)].long()] = 1
    return table, ref


def _pools(case, blocks, g):
    """Per layer K, V (and exponents)."""
    shape = (blocks, case["kv_heads"], BT, case["head_dim"])
    out = []
    for _ in range(case["layers"]):
        if case["kv"] == "e4m3":
            out.append([torch.randint(0, 120, s, generator=g, device="cuda", dtype=torch.uint8) for s in (shape, shape, shape[:3], shape[:3])])
        else:
            out.append([torch.empty(shape, dtype=TYPES[case["kv"]], device="cuda").normal_(generator=g) for _ in range(2)])
    return out


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    if case["kind"] == "verify":
        st.update(_prepare_verify(case, g))
        if own:
            import paper_2601_03700_gb300 as adept
            st["ws"] = adept.verify_workspace(st["tokens"].numel())
        return st
    if case["kind"] == "round":
        lens, n_rows, blocks = _lengths(case), case["seqs"], case["blocks"]
        # as the last round left them: rows of up to `step` positions more
        more = [n + (b * 3) % (case["step"] + 1) for b, n in enumerate(lens)]
        table, ref = _fill_rows(case, more, blocks, g)
        st.update(source=torch.arange(n_rows, dtype=torch.int32, device="cuda"), length=_i32(lens), want=_i32([n + case["step"] for n in lens]))
    elif case["kind"] == "branch":
        prompts = _prompts(case)
        n_rows = len(prompts) * (1 + case["branches"])
        blocks = sum(_up(n) + case["branches"] * (_up(n + case["grow"]) - n // BT) for n in prompts) + 5
        lens = prompts + [0] * (n_rows - len(prompts))
        table, ref = _fill_rows(case, lens, blocks, g)
        src = list(range(len(prompts))) + [b for b in range(len(prompts)) for _ in range(case["branches"])]
        length = [prompts[b] for b in src]
        st.update(source=_i32(src), length=_i32(length), want=_i32([n + (case["grow"] if r >= len(prompts) else 0) for r, n in enumerate(length)]))
    else:
        held, _ = _compact_moves(case)
        n_rows, blocks = case["seqs"], case["blocks"]
        lens = [min(case["cols"], held // n_rows + (b < held % n_rows)) * BT for b in range(n_rows)]
        table, ref = _fill_rows(case, lens, blocks, g)
        if n_rows > 1:   # the second row shares its first blocks with the first
            n = min(lens[0], lens[1]) // BT // 2
            ref[table[1, :n].long()] -= 1
            table[1, :n] = table[0, :n]
            ref[table[0, :n].long()] += 1
    st.update(pools=[] if case["kind"] == "round" else _pools(case, blocks, g))
    if own:
        import paper_2601_03700_gb300 as adept
        p = adept.KVPages(blocks, n_rows, case["cols"], block_tokens=BT)
        p.block_table.copy_(table)
        p.ref.copy_(ref)
        st["pages"], st["ws"], st["state0"] = p, p.workspace(), p.state.clone()
        if st["pools"]:
            layers = [adept.KVCache(blocks, case["kv_heads"], case["head_dim"], n_rows, case["cols"], dtype=case["kv"], block_tokens=BT, pages=p)
                      for _ in st["pools"]]
            for c, pool in zip(layers, st["pools"]):
                for to, x in zip((c.k, c.v, c.k_exp, c.v_exp), pool):
                    to.copy_(x)
            st["pools"] = [[x for x in (c.k, c.v, c.k_exp, c.v_exp) if x is not None] for c in layers]
            st["layers"] = adept.KVLayers(layers)
    else:
        st["table"], st["ref"] = table, ref
        st["state0"] = (table.clone(), ref.clone())
    n_pairs = blocks // 2 if case["kind"] == "compact" else n_rows
    st["got"] = torch.zeros(1 if case["kind"] == "compact" else n_rows, dtype=torch.int32, device="cuda")
    st["src"], st["dst"] = (torch.zeros(n_pairs, dtype=torch.int32, device="cuda") for _ in range(2))
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _plain_verify(st):
    target, draft, start, u = st["target"], st["draft"], st["start"].long(), st["u"]
    n, rows = start.numel() - 1, target.shape[0]
    # the sequence of each row, and the next row's token (the last row of a sequence has none)
    seq = torch.searchsorted(start[1:].contiguous(), torch.arange(rows, device="cuda"), right=True)
    temp = torch.ones(n, device="cuda") if st["temp"] is None else st["temp"]
    greedy = temp == 0
    scale = torch.where(greedy, torch.ones_like(temp), temp).double()[seq][:, None]
    x = st["tokens"].long().roll(-1)[:, None]
    lp = torch.log_softmax(target.double() / scale, 1)
    best = target.float().argmax(1)
    if draft is None:
        lq = torch.full_like(lp, -math.inf).scatter_(1, x, 0.0)
    else:
        lq = torch.log_softmax(draft.double() / scale, 1)
    holds = u.double().log() + lq.gather(1, x)[:, 0] < lp.gather(1, x)[:, 0]
    holds = torch.where(greedy[seq], best == x[:, 0], holds)
    # drafts accepted: rows from the first one on that all hold
    row = torch.arange(rows, device="cuda")
    last = row == start[1:][seq] - 1
    first_bad = torch.full((n,), rows, device="cuda").scatter_reduce_(0, seq, torch.where(holds & ~last, torch.full_like(row, rows), row), "amin")
    accepted = first_bad - start[:-1]
    at = first_bad
    p = lp[at].exp()
    q = torch.where(last[at][:, None], torch.zeros_like(p), lq[at].exp())
    w = (p - q).clamp_(min=0)
    w = torch.where(w.sum(1, keepdim=True) < 2.0 ** -20, p, w)
    c = w.cumsum(1)
    drawn = (c <= (u[start[1:] - 1].double()[:, None] + 2.0 ** -25) * w.sum(1, keepdim=True)).sum(1)
    nxt = torch.where(greedy, best[at], drawn)
    # log probabilities of the tokens that were taken (rows behind them stay as they are)
    taken = torch.where(row == at[seq], nxt[seq], x[:, 0])
    st["logprob"].copy_(torch.where(row <= at[seq], lp.gather(1, taken[:, None])[:, 0].float(), st["logprob"]))
    return [accepted.int(), nxt.int(), st["logprob"]]


def _plain_fork(table, ref, source, length):
    """Row b: the first length[b] positions of row source[b] (< 0: none)."""
    cols = torch.arange(table.shape[1], device="cuda")[None, :]
    keep = (cols < (length[:, None] + BT - 1) // BT) & (source[:, None] >= 0)
    new = torch.where(keep, table[source.long().clamp(min=0)], torch.full_like(table, -1))
    for x, by in ((new, 1), (table, -1)):
        ref.index_add_(0, x.reshape(-1).long().clamp(min=0), (x.reshape(-1) >= 0).int() * by)
    table.copy_(new)


def _plain_reserve(table, ref, length, want):
    """(positions that each row may write up to, blocks to copy from, to)."""
    n, nb = table.shape[0], ref.numel()
    row, cols = torch.arange(n, device="cuda"), torch.arange(table.shape[1], device="cuda")[None, :]
    asks = want > length
    j0 = length // BT
    inside = asks[:, None] & (cols >= j0[:, None]) & (cols < (want[:, None] + BT - 1) // BT)
    e = table.long().clamp(min=0)
    shared = inside & (table >= 0) & (ref[e] > 1)
    # blocks that are written in part, held by several rows: the last of these keeps it where all of them ask
    at = cols == j0[:, None]
    part = (shared & at).any(1) & (length % BT > 0)
    pe = e.gather(1, j0.long().clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    asking = torch.zeros(nb + 1, dtype=torch.int32, device="cuda").index_add_(0, torch.where(part, pe, torch.full_like(pe, nb)), torch.ones_like(row).int())
    final = torch.full((nb + 1,), -1, device="cuda").scatter_reduce_(0, torch.where(part, pe, torch.full_like(pe, nb)), row, "amax")
    keeps = part & (asking[pe] == ref[pe]) & (final[pe] == row)
    need = inside & ((table < 0) | shared) & ~(at & keeps[:, None])
    ask = need.sum(1)
    free = ref == 0
    served = asks & ((ask.cumsum(0) <= free.sum()) | ((ask == 0) & ~keeps))
    need &= served[:, None]
    # the free blocks in ascending order
    ids = torch.zeros(nb + 1, dtype=torch.int32, device="cuda")
    ids[torch.where(free, free.long().cumsum(0) - 1, torch.full_like(ref, nb).long())] = torch.arange(nb, dtype=torch.int32, device="cuda")
    new = torch.where(need, ids[(need.reshape(-1).long().cumsum(0) - 1).clamp(0, nb).view(need.shape)], table)
    copy = part & ~keeps & served
    none = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    src = torch.where(copy, pe.int(), none)
    dst = torch.where(copy, new.gather(1, j0.long().clamp(max=table.shape[1] - 1)[:, None])[:, 0], none)
    ref.index_add_(0, e.reshape(-1), -(need & shared).reshape(-1).int())
    ref.index_add_(0, new.reshape(-1).long().clamp(min=0), need.reshape(-1).int())
    table.copy_(new)
    return torch.where(served, want, length), src, dst


def _plain_compact(table, ref):
    """(blocks in use, blocks moved from, to)."""
    nb = ref.numel()
    ids = torch.arange(nb, device="cuda")
    used = ref > 0
    count = used.sum()
    hole, mover = ~used & (ids < count), used & (ids >= count)
    pairs = []
    for m in (mover, hole):
        to = torch.full((nb + 1,), -1, dtype=torch.int32, device="cuda")
        to[torch.where(m, m.long().cumsum(0) - 1, torch.full_like(ids, nb))] = ids.int()
        k = torch.arange(nb // 2, device="cuda")
        pairs.append(torch.where(k < m.sum(), to[:nb // 2], torch.full_like(to[:nb // 2], -1)))
    src, dst = pairs
    s, d = (torch.where(x >= 0, x, torch.full_like(x, nb)).long() for x in pairs)
    remap = torch.cat([ids, ids[:1]]).int()
    remap[s] = torch.where(dst >= 0, dst, remap[s])
    table.copy_(torch.where(table >= 0, remap[table.long().clamp(min=0)], table))
    full = torch.cat([ref, ref[:1]])
    full[d] = full[s]
    full[s] = 0
    ref.copy_(full[:nb])
    return count.int().view(1), src, dst


def _plain_copy(pools, src, dst):
    """Blocks src[i] to dst[i] in every layer (-1: none).  A pair of none is made the first live pair, or block 0 onto itself."""
    live = src >= 0
    first = live.int().argmax()
    s, d = (torch.where(live, x, torch.where(live.any(), x[first], torch.zeros_like(x[first]))).long() for x in (src, dst))
    for pool in pools:
        for x in pool:
            x[d] = x[s]


def run(state):
    case = state["case"]
    if case["kind"] == "verify":
        if not own:
            return _plain_verify(state)
        import paper_2601_03700_gb300 as adept
        accepted, nxt = (torch.empty(case["seqs"], dtype=torch.int32, device="cuda") for _ in range(2))
        adept.adept_verify_drafts(state["target"], state["draft"], state["tokens"], state["start"], state["u"], accepted, nxt,
                                  logprob=state["logprob"], temperature=state["temp"], workspace=state["ws"])
        return [accepted, nxt, state["logprob"]]
    if not own:
        table, ref = state["table"], state["ref"]
        if case["kind"] == "compact":
            table.copy_(state["state0"][0])   # a pool with holes again
            ref.copy_(state["state0"][1])
            got, src, dst = _plain_compact(table, ref)
        else:
            _plain_fork(table, ref, state["source"], state["length"])
            got, src, dst = _plain_reserve(table, ref, state["length"], state["want"])
        if state["pools"]:
            _plain_copy(state["pools"], src, dst)
        return [table, ref, got, src, dst, state["pools"]]
    import paper_2601_03700_gb300 as adept
    pages, got, src, dst = state["pages"], state["got"], state["src"], state["dst"]
    if case["kind"] == "compact":
        pages.state.copy_(state["state0"])
        adept.adept_kv_compact(pages, got, src, dst, workspace=state["ws"])
    else:
        adept.adept_kv_fork(pages, state["source"], state["length"], workspace=state["ws"])
        adept.adept_kv_reserve(pages, state["length"], state["want"], got, src, dst, workspace=state["ws"])
    if state["pools"]:
        adept.adept_kv_copy_blocks(state["layers"], src, dst)
    return [pages.block_table, pages.ref, got, src, dst, state["pools"]]


# ---------------------------------------------------------------------------
# from the definitions
# ---------------------------------------------------------------------------

def _exact_verify(st):
    accepted, nxt, logprob = [], [], torch.zeros(st["u"].numel(), dtype=torch.float64)
    start, tokens = st["start"].tolist(), st["tokens"].tolist()
    for b in range(len(start) - 1):
        t = 1.0 if st["temp"] is None else float(st["temp"][b])
        r, end = start[b], start[b + 1] - 1
        logs = lambda x: x.double() / (t or 1.0) - torch.logsumexp(x.double() / (t or 1.0), 0)  # noqa: E731
        probs = lambda x: torch.exp(logs(x))  # noqa: E731
        p = q = None
        while True:
            if t == 0:
                x = st["target"][r].double()
                p, q = (x == x.max()), None
                if r == end or int(p.int().argmax()) != tokens[r + 1]:
                    break
            else:
                p, q = probs(st["target"][r]), None
                if r == end:
                    break
                if st["draft"] is None:
                    q = torch.zeros_like(p)
                    q[tokens[r + 1]] = 1.0
                else:
                    q = probs(st["draft"][r])
                if not float(st["u"][r]) * float(q[tokens[r + 1]]) < float(p[tokens[r + 1]]):
                    break
            logprob[r] = logs(st["target"][r])[tokens[r + 1]]
            r += 1
        accepted.append(r - start[b])
        if t == 0:
            nxt.append(int(p.int().argmax()))
            logprob[r] = logs(st["target"][r])[nxt[-1]]
            continue
        w = p if q is None or float(torch.relu(p - q).sum()) < 2.0 ** -20 else torch.relu(p - q)
        c = torch.cumsum(w, 0)
        nxt.append(int(torch.searchsorted(c, ((float(st["u"][end]) + 2.0 ** -25) * w.sum()).view(1), right=True)))
        logprob[r] = logs(st["target"][r])[nxt[-1]]
    return [_i32(accepted), _i32(nxt), logprob.cuda()]


def _exact_pages(st):
    case, table, ref = st["case"], st["table"].tolist(), st["ref"].tolist()
    n_pairs = st["src"].numel()
    src, dst = [-1] * n_pairs, [-1] * n_pairs
    if case["kind"] == "compact":
        used = [i for i, r in enumerate(ref) if r]
        got, moved = [len(used)], {}
        holes = [i for i in range(len(used)) if not ref[i]]
        for k, (s, d) in enumerate(zip([i for i in used if i >= len(used)], holes)):
            src[k], dst[k], moved[s] = s, d, d
            ref[d], ref[s] = ref[s], 0
        table = [[moved.get(e, e) for e in row] for row in table]
    else:
        source, length, want = (st[k].tolist() for k in ("source", "length", "want"))
        old = table
        table = [(old[s][:_up(n)] if s >= 0 else []) for s, n in zip(source, length)]
        table = [row + [-1] * (case["cols"] - len(row)) for row in table]
        for rows, by in ((old, -1), (table, 1)):
            for e in (e for row in rows for e in row if e >= 0):
                ref[e] += by
        free = [i for i, r in enumerate(ref) if not r]
        got, before, enough = list(length), list(ref), True
        part = [table[b][n // BT] if want[b] > n and n % BT and before[table[b][n // BT]] > 1 else -1 for b, n in enumerate(length)]
        for b, (n, w) in enumerate(zip(length, want)):
            if w <= n:
                continue
            keep = part[b] >= 0 and part.count(part[b]) == before[part[b]] and part[b] not in part[b + 1:]
            need = [j for j in range(n // BT, _up(w)) if table[b][j] < 0 or (before[table[b][j]] > 1 and not (keep and j == n // BT))]
            enough = enough and len(need) <= len(free)
            if not enough and (need or keep):
                continue
            got[b] = w
            for j in need:
                e, table[b][j] = table[b][j], free.pop(0)
                ref[table[b][j]] = 1
                if e >= 0:
                    ref[e] -= 1
                    if j == n // BT and n % BT:
                        src[b], dst[b] = e, table[b][j]
    pools = []
    s, d = (torch.tensor([i for i in x if i >= 0], dtype=torch.int64, device="cuda") for x in (src, dst))
    for pool in st["pools"]:
        pools.append([])
        for x in pool:
            y = x.double() if x.is_floating_point() else x.clone()
            y[d] = y[s]
            pools[-1].append(y)
    return [_i32(table), _i32(ref), _i32(got), _i32(src), _i32(dst), pools]


def exact(case, seed):
    global own
    held, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = held
    return _exact_verify(st) if case["kind"] == "verify" else _exact_pages(st)
